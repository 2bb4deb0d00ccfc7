// New tokens' keys and values into the paged 8-bit cache, with rotary positions, and the table of cosines and sines.
//
// One launch; a workgroup has one job:
//   keys    of one page and head: rotate, find the largest magnitude, take the page's scale, write [token][dim];
//   values  of one page and head: the same without the rotation, written [dim][token] through LDS;
//   queries of one token row, 16 or 32 heads: rotate.
// A page's scale depends on nothing but the page's own tokens, so no two workgroups share one.  The values of a page are held
// in registers between the search for the largest and the writing (eight neighbouring dimensions of a token to a thread).
// 2048 rows of 56 + 8 heads of 128: 16.2 us, 4.4 TB/s; 64 single tokens of 64 + 8 heads: 6.4 - 6.8 us.  Bound by memory for prompts, by the latency of its dependent loads (lengths, table and positions, values, old scale) for
// single tokens.
#include <algorithm>

#include "ccq_layer.h"

namespace ccq {

namespace {

struct AppendArgs {
  uint8_t *kc, *vc, *ks, *vs;
  const uint16_t *k, *v, *q;
  uint16_t* q_out;
  int64_t k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;
  const int32_t *offsets, *lens, *table;
  int64_t ld_table;
  const float* rope;
  const int32_t* positions;
  int32_t rope_rows, dims, interleaved;
  int32_t pages, kv_heads, q_heads, table_width, tokens, max_new, max_len;
  int32_t page_slots;         // pages that the new tokens of a sequence may touch
  int32_t kv_groups, query_groups, total;   // workgroups of keys (as many of values); a token row's queries; of the call
  int32_t first;              // workgroup of the call that is the launch's first
};

struct Sequence {
  int first, n, old;   // first token row, new tokens (within bounds), tokens before them
};
__device__ __forceinline__ Sequence sequence_of(const AppendArgs& a, int b) {
  Sequence s;
  const int end = min(a.offsets[b + 1], a.tokens);
  s.first = max(a.offsets[b], 0);
  s.n = end - s.first;
  s.old = a.lens[b] - s.n;
  s.n = min(s.n, a.max_new);
  return s;
}

// The rope table's row of a token, or NULL.
__device__ __forceinline__ const float* angles(const AppendArgs& a, int token, int position) {
  if (!a.rope) return nullptr;
  const int p = a.positions ? a.positions[token] : position;
  return a.rope + (int64_t)min(max(p, 0), a.rope_rows - 1) * a.dims;
}

__device__ __forceinline__ void unpack8(u32x4_t v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(v[i]);
    x[2 * i + 1] = bf16_hi(v[i]);
  }
}

// Cosines and sines for the eight dimensions from d0 on (sine with the sign that the partner's product has).
struct Turn {
  float c[8], s[8];
};
__device__ __forceinline__ void load_turn(const AppendArgs& a, const float* row, int d0, Turn& t) {
  const int half = a.dims >> 1;
  if ((half & 7) == 0 && d0 < a.dims) {   // eight pairs, or four, that lie side by side (one number at a time: 20 us instead of 17 for 2048 rows of 56 + 8 heads of 128)
    const float* from = row + (a.interleaved ? d0 >> 1 : d0 < half ? d0 : d0 - half);
    const float sign = d0 < half ? -1.f : 1.f;
    f32x4_t c[2], s[2];
    __builtin_memcpy(&c[0], from, 16);
    __builtin_memcpy(&s[0], from + half, 16);
    if (!a.interleaved) {
      __builtin_memcpy(&c[1], from + 4, 16);
      __builtin_memcpy(&s[1], from + half + 4, 16);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t.c[i] = a.interleaved ? c[0][i >> 1] : c[i >> 2][i & 3];
      t.s[i] = a.interleaved ? ((i & 1) ? s[0][i >> 1] : -s[0][i >> 1]) : s[i >> 2][i & 3] * sign;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int d = d0 + i;
    t.c[i] = 1.f;
    t.s[i] = 0.f;
    if (d < a.dims) {
      const int pair = a.interleaved ? d >> 1 : (d < half ? d : d - half);
      const bool second = a.interleaved ? (d & 1) : d >= half;
      const float s = row[half + pair];
      t.c[i] = row[pair];
      t.s[i] = second ? s : -s;
    }
  }
}
// x: dimensions d0 .. d0 + 7 of the head at `head` (bf16).  Products and sum are each rounded: c a - s b and c b + s a.
// `partner`: what load_partner gave.
__device__ __forceinline__ u32x4_t load_partner(const AppendArgs& a, const uint16_t* head, int d0) {
  const int half = a.dims >> 1;
  if (a.interleaved || (half & 7) || d0 >= a.dims) return u32x4_t{0, 0, 0, 0};
  return *reinterpret_cast<const u32x4_t*>(head + (d0 < half ? d0 + half : d0 - half));
}
__device__ __forceinline__ void rotate8(const AppendArgs& a, const uint16_t* head, int d0, const Turn& t, u32x4_t partner, float (&x)[8]) {
#pragma clang fp contract(off)
  if (d0 >= a.dims) return;
  float other[8];
  const int half = a.dims >> 1;
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) other[i] = x[i ^ 1];
  } else if ((half & 7) == 0) {
    unpack8(partner, other);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      other[i] = d < a.dims ? bf16_lo(head[d < half ? d + half : d - half]) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float p = x[i] * t.c[i], q = other[i] * t.s[i];
    if (d0 + i < a.dims) x[i] = p + q;
  }
}

// Largest over the workgroup's 256 threads.
__device__ __forceinline__ uint32_t max_of_block(uint32_t v) {
  __shared__ uint32_t parts[4];
  v = max16(v);
  v = max(v, xor16(v));
  v = max(v, xor32(v));
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(parts[0], parts[1]), max(parts[2], parts[3]));
}

// Four e4m3 values times f (a power of two up to 1).
__device__ __forceinline__ uint32_t rescale4(uint32_t v, float f) {
  return pack_e4m3(__builtin_amdgcn_cvt_f32_fp8((int)v, 0) * f, __builtin_amdgcn_cvt_f32_fp8((int)v, 1) * f, __builtin_amdgcn_cvt_f32_fp8((int)v, 2) * f,
                   __builtin_amdgcn_cvt_f32_fp8((int)v, 3) * f);
}

__device__ __forceinline__ bool finite_bits(uint32_t magnitude) { return magnitude < kInfBits; }
// Whether one of eight bf16 values is NaN or infinite.
__device__ __forceinline__ bool any_bad(u32x4_t v) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) bad |= (v[i] & 0x7F80u) == 0x7F80u || (v[i] & 0x7F800000u) == 0x7F800000u;
  return bad;
}

// D: head dimension; P: tokens of a page.  KEYS or values of page slot `slot` of sequence b, head h.
template <int D, int P, bool KEYS>
__device__ __forceinline__ void append_page(const AppendArgs& a, int b, int slot, int h, uint8_t* lds) {
  constexpr int kPieces = D / 8, kTokens = 256 / kPieces, IT = (P + kTokens - 1) / kTokens;   // threads of a token, tokens at a time
  const Sequence s = sequence_of(a, b);
  if (s.n <= 0) return;
  const int page_no = max(s.old, 0) / P + slot;
  const int lo = max(max(s.old, 0), page_no * P), hi = min(min(s.old + s.n, a.max_len), (page_no + 1) * P);   // positions of the page's new tokens
  if (lo >= hi || page_no >= a.table_width) return;
  const int page = a.table[b * a.ld_table + page_no];   // (first looked at when the tokens are loaded: one wait for memory, not two)
  const int d0 = (threadIdx.x % kPieces) * 8, t0 = threadIdx.x / kPieces;
  const int row0 = s.first + (lo - s.old);   // token row of position lo

  float x[IT][8];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < IT; ++j) {
    const int t = t0 + j * kTokens;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
    if (t >= hi - lo) continue;
    const int row = row0 + t;
    const u32x4_t vv = *reinterpret_cast<const u32x4_t*>(a.v + row * a.v_token + h * a.v_head + d0);
    const uint16_t* head = a.k + row * a.k_token + h * a.k_head;
    const float* angle = nullptr;
    u32x4_t kk, partner;
    Turn turn;
    if (KEYS) {
      kk = *reinterpret_cast<const u32x4_t*>(head + d0);
      angle = angles(a, row, lo + t);
      if (angle) {
        partner = load_partner(a, head, d0);
        load_turn(a, angle, d0, turn);
      }
    }
    bool bad = any_bad(vv);   // of the token: its threads stand side by side in a wavefront
    const uint64_t votes = __ballot(bad);
    bad = (votes >> ((threadIdx.x & 63) / kPieces * kPieces) & ((1ull << kPieces) - 1)) != 0;
    if (KEYS) {
      unpack8(kk, x[j]);
      if (angle) rotate8(a, head, d0, turn, partner, x[j]);
      if (bad) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = __builtin_nanf("");
      }
    } else {
      unpack8(vv, x[j]);
      if (bad) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = __builtin_bit_cast(uint32_t, x[j][i]) & 0x7FFFFFFFu;
      if (finite_bits(m)) top = max(top, m);
    }
  }
  if (page < 0 || page >= a.pages) return;
  const int older = lo - page_no * P;   // slots that hold older tokens
  const int64_t tile = (int64_t)page * a.kv_heads + h;
  uint8_t* scale_at = (KEYS ? a.ks : a.vs) + tile;
  const int old_byte = older > 0 ? *scale_at : 0;
  uint8_t* codes = (KEYS ? a.kc : a.vc) + tile * (P * D);
  int byte = scale_byte(max_of_block(top), 127 - kCacheExp, 127 + kCacheExp);
  if (older > 0 && old_byte > byte) byte = min(old_byte, 254);
  const float inv = inverse_of_byte(min(byte, 253));
  if (threadIdx.x == 0) *scale_at = (uint8_t)byte;

  if (older > 0 && old_byte < byte) {
    const float f = __builtin_amdgcn_ldexpf(1.f, old_byte - byte);
    if (KEYS) {
      for (int i = threadIdx.x; i < older * D / 16; i += 256) {
        u32x4_t v = reinterpret_cast<const u32x4_t*>(codes)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = rescale4(v[e], f);
        reinterpret_cast<u32x4_t*>(codes)[i] = v;
      }
    } else {
      // 16 slots of a dimension at a time; of the last piece only the older tokens' bytes are written
      const int pieces = (older + 15) / 16;
      for (int i = threadIdx.x; i < pieces * D; i += 256) {
        const int d = i / pieces, p = i % pieces;
        uint8_t* at = codes + d * P + p * 16;
        u32x4_t v = *reinterpret_cast<const u32x4_t*>(at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = rescale4(v[e], f);
        if (p * 16 + 16 <= older) {
          *reinterpret_cast<u32x4_t*>(at) = v;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (p * 16 + e < older) at[e] = (uint8_t)(v[e >> 2] >> (8 * (e & 3)));
        }
      }
    }
  }

  constexpr int kPitch = P + 4;   // bytes between dimensions in LDS
#pragma unroll
  for (int j = 0; j < IT; ++j) {
    const int t = t0 + j * kTokens;
    if (t >= hi - lo) continue;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = x[j][i] * inv;
      const uint32_t m = __builtin_bit_cast(uint32_t, x[j][i]) & 0x7FFFFFFFu;
      y[i] = finite_bits(m) ? fminf(fmaxf(y[i], -448.f), 448.f) : __builtin_nanf("");
    }
    const u32x2_t q = {pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7])};
    if (KEYS) {
      *reinterpret_cast<u32x2_t*>(codes + (older + t) * D + d0) = q;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) lds[(d0 + i) * kPitch + older + t] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
    }
  }
  if constexpr (!KEYS) {
    __syncthreads();
    const int first = older / 4, words = (older + hi - lo + 3) / 4 - first;   // words of four slots that hold new tokens
    for (int i = threadIdx.x; i < words * D; i += 256) {
      const int d = i / words, w = first + i % words;
      const uint32_t v = *reinterpret_cast<const uint32_t*>(lds + d * kPitch + 4 * w);
      uint8_t* at = codes + d * P + 4 * w;
      if (4 * w >= older && 4 * w + 4 <= older + hi - lo) {
        *reinterpret_cast<uint32_t*>(at) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (4 * w + e >= older && 4 * w + e < older + hi - lo) at[e] = (uint8_t)(v >> (8 * e));
      }
    }
  }
}

template <int D>
constexpr int kQueryHeads = 256 / (D / 8);   // of a workgroup
template <int D>
__device__ __forceinline__ void rotate_queries(const AppendArgs& a, int b, int i, int heads) {
  const Sequence s = sequence_of(a, b);
  if (i >= s.n) return;
  const int row = s.first + i, d0 = (threadIdx.x % (D / 8)) * 8, own = threadIdx.x / (D / 8);
  auto head_at = [&](int h) { return a.q + row * a.q_token + min(h, a.q_heads - 1) * a.q_head; };
  u32x4_t q = *reinterpret_cast<const u32x4_t*>(head_at(heads * kQueryHeads<D> + own) + d0);
  const float* angle = angles(a, row, s.old + i);
  Turn turn;
  if (angle) load_turn(a, angle, d0, turn);
  for (int h0 = heads * kQueryHeads<D>; h0 < a.q_heads; h0 += a.query_groups * kQueryHeads<D>) {
    const int h = h0 + own;
    float x[8];
    unpack8(q, x);
    if (angle) rotate8(a, head_at(h), d0, turn, load_partner(a, head_at(h), d0), x);
    q = *reinterpret_cast<const u32x4_t*>(head_at(h + a.query_groups * kQueryHeads<D>) + d0);   // the next heads'
    __syncthreads();   // every thread's partner dimensions are read before anything of their head is written: q_out may be q
    if (h >= a.q_heads) continue;
    u32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
    *reinterpret_cast<u32x4_t*>(a.q_out + row * a.o_token + h * a.o_head + d0) = v;
  }
}

template <int D, int P>
__global__ __launch_bounds__(256) void ccq_append_kernel(AppendArgs a) {
  __shared__ __align__(16) uint8_t lds[D * (P + 4)];
  int g = a.first + blockIdx.x;
  if (g < 2 * a.kv_groups) {
    const bool keys = g < a.kv_groups;
    if (!keys) g -= a.kv_groups;
    const int h = g % a.kv_heads, r = g / a.kv_heads;
    if (keys) append_page<D, P, true>(a, r / a.page_slots, r % a.page_slots, h, lds);
    else append_page<D, P, false>(a, r / a.page_slots, r % a.page_slots, h, lds);
  } else {
    g -= 2 * a.kv_groups;
    const int heads = g % a.query_groups, r = g / a.query_groups;
    rotate_queries<D>(a, r / a.max_new, r % a.max_new, heads);
  }
}

struct TableArgs {
  float* table;
  double base, factor, low, high, magnitude;
  int32_t kind, rows, dims;
  int64_t first;   // pair of the table that is the launch's first
};
__global__ __launch_bounds__(256) void ccq_rope_table_kernel(TableArgs a) {
  const int half = a.dims / 2;
  const int64_t at = a.first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)a.rows * half) return;
  const int p = (int)(at / half), i = (int)(at % half);
  double f = pow(a.base, -2.0 * i / a.dims);
  if (a.kind == 1) f /= a.factor;
  if (a.kind == 3) {
    const double mix = fmin(fmax((i - a.low) / fmax(a.high - a.low, 1e-3), 0.0), 1.0);
    f = f * (1.0 - mix) + f / a.factor * mix;
  }
  double s, c;
  sincos(p * f, &s, &c);
  a.table[(int64_t)p * a.dims + i] = (float)(c * a.magnitude);
  a.table[(int64_t)p * a.dims + half + i] = (float)(s * a.magnitude);
}

template <int D, int P>
void launch(const AppendArgs& a, hipStream_t s) {
  AppendArgs part = a;
  for (int64_t first = 0; first < a.total; first += most_groups(256)) {
    part.first = (int)first;
    hipLaunchKernelGGL((ccq_append_kernel<D, P>), dim3((unsigned)std::min<int64_t>(a.total - first, most_groups(256))), dim3(256), 0, s, part);
  }
}
template <int D>
int launch_d(const AppendArgs& a, int page_tokens, hipStream_t s) {
  switch (page_tokens) {
    case 16: launch<D, 16>(a, s); break;
    case 32: launch<D, 32>(a, s); break;
    case 64: launch<D, 64>(a, s); break;
    case 128: launch<D, 128>(a, s); break;
    case 256: launch<D, 256>(a, s); break;
    default: return CCQ_ERR_UNSUPPORTED;
  }
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace

int launch_rope_table(const ccq_rope_scaling* s, int rows, int dims, float* table, void* stream) {
  TableArgs a;
  a.table = table;
  a.kind = s->kind, a.rows = rows, a.dims = dims;
  a.base = s->base, a.factor = s->factor, a.magnitude = s->magnitude == 0.0 ? 1.0 : s->magnitude;
  a.low = a.high = 0.0;
  if (s->kind == 2) a.base = s->base * pow(s->factor, (double)dims / (dims - 2));
  if (s->kind == 3) {
    const double scale = dims / (2.0 * log(s->base)), turn = 2.0 * 3.14159265358979323846;
    a.low = fmax(floor(scale * log(s->original_length / (turn * s->fast))), 0.0);
    a.high = fmin(ceil(scale * log(s->original_length / (turn * s->slow))), dims - 1.0);
  }
  const int64_t blocks = ((int64_t)rows * (dims / 2) + 255) / 256;
  for (int64_t first = 0; first < blocks; first += most_groups(256)) {
    a.first = first * 256;
    hipLaunchKernelGGL(ccq_rope_table_kernel, dim3((unsigned)std::min(blocks - first, most_groups(256))), dim3(256), 0, static_cast<hipStream_t>(stream), a);
  }
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

int launch_cache_append(const ccq_cache* c, const ccq_batch* b, const ccq_rope* rope, const ccq_heads* k, const ccq_heads* v, const ccq_heads* q,
                        const ccq_heads* q_out, int q_heads, void* stream) {
  AppendArgs a = {};
  a.kc = static_cast<uint8_t*>(c->k), a.vc = static_cast<uint8_t*>(c->v), a.ks = c->k_scales, a.vs = c->v_scales;
  if (k) {
    a.k = static_cast<const uint16_t*>(k->data), a.k_token = k->token_stride, a.k_head = k->head_stride;
    a.v = static_cast<const uint16_t*>(v->data), a.v_token = v->token_stride, a.v_head = v->head_stride;
  }
  if (q) {
    a.q = static_cast<const uint16_t*>(q->data), a.q_token = q->token_stride, a.q_head = q->head_stride;
    a.q_out = static_cast<uint16_t*>(q_out->data), a.o_token = q_out->token_stride, a.o_head = q_out->head_stride;
  }
  a.offsets = b->offsets, a.lens = b->lens, a.table = b->table, a.ld_table = b->ld_table;
  if (rope) a.rope = rope->table, a.positions = rope->positions, a.rope_rows = rope->rows, a.dims = rope->dims, a.interleaved = rope->interleaved;
  a.pages = c->pages, a.kv_heads = c->kv_heads, a.q_heads = q_heads, a.table_width = b->table_width;
  a.tokens = b->tokens, a.max_new = b->max_new, a.max_len = b->max_len;
  const int P = c->page_tokens;
  a.page_slots = (int)(((int64_t)b->max_new + P - 2) / P + 1);
  const int64_t groups = k ? (int64_t)b->batch * a.page_slots * c->kv_heads : 0;
  // Few token rows: a workgroup to every 16 heads of 128; many: one to a row.  By workgroups that the first makes, us with it / with one to a row: 32 rows of 64 heads (128 groups) 4.5 / 5.3, 64 of
  // 64 (256) 6.1 / 7.3, 128 of 128 (1024) 10.8 / 12.1, 256 of 64 (1024) 16.3 / 16.0, 512 of 64 (2048) 7.7 / 7.8, 1024 of 64 (4096) 13.6 / 10.9, 2048 of 64 (8192) 24.3 / 18.1.
  const int64_t rows = (int64_t)b->batch * b->max_new, heads_at_once = c->head_dim == 64 ? kQueryHeads<64> : kQueryHeads<128>;
  const int64_t head_groups = (q_heads + heads_at_once - 1) / heads_at_once;
  a.query_groups = rows * head_groups <= 1024 ? (int)std::max<int64_t>(head_groups, 1) : 1;
  const int64_t total = 2 * groups + (q ? (int64_t)b->batch * b->max_new * a.query_groups : 0);
  if (total > 0x7FFFFFFF) return CCQ_ERR_BAD_PARAM;
  if (total == 0) return CCQ_OK;
  a.kv_groups = (int)groups, a.total = (int)total;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return c->head_dim == 64 ? launch_d<64>(a, P, s) : launch_d<128>(a, P, s);
}

}  // namespace ccq
