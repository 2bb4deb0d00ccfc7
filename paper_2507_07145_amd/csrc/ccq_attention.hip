// Attention over the paged 8-bit cache for few rows: single new tokens, and the join of splits.
//
// A wavefront walks tiles of 64 cached tokens on its own (the four of a workgroup take them in turn) and holds up to 16 or 32 rows:
//   scores^T = K q^T   MFMA 16x16x32 bf16, cached tokens as rows: e4m3 is exact in bf16
//   out^T    = V^T p^T MFMA 16x16x32 f16, dimensions as rows: e4m3 is exact in fp16
// Tokens are dealt to the first product's rows so that a lane's 16 scores are those of 16 neighbouring tokens, in the order in which
// the second product wants its operand: the weights go from one to the other in registers, and the values of a dimension, stored
// token after token, are 16-byte loads that need no transposition either.  Nothing passes LDS until the wavefronts' results
// are joined.  A lane's 16 tokens lie in one page (pages hold multiples of 16): its scales are one value each.
// Bound by memory: 16 KB a tile (128 dimensions) against 32 MFMAs; keys and scales are asked for a tile ahead, table entries two, values while the scores
// are formed.  64 sequences of up to 8192 tokens (687 MB): 130 - 133 us, 5.2 TB/s; one of 131072 (268 MB): 55 - 57 us with the join.
#include <algorithm>

#include "ccq_attention.h"

namespace ccq {

namespace {

constexpr int kTile = 64, kWaves = 4;

// The sums of weights of a wavefront's rows once more, from the keys alone, with the references that are in `stats`.  Takes its arguments from memory again: kept in registers through the
// main loop, they made the compiler ask for that loop's values behind its products (64 sequences of 8192: 143 us instead of 132).
template <int D, int NT>
__device__ __forceinline__ void weights_again(float* stats) {
  constexpr int STEPS = D / 32;
  const AttnArgs* args = (const AttnArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  int thread = threadIdx.x;
  asm volatile("" : "+s"(args), "+v"(thread));
  const AttnArgs& a = *args;
  const int lane = thread & 63, wave = thread >> 6, r16 = lane & 15, g = lane >> 4, quarter_k = r16 >> 2;
  const int h = blockIdx.x % a.kv_heads, tile = (blockIdx.x / a.kv_heads) % a.row_tiles, split = blockIdx.x / (a.kv_heads * a.row_tiles), b = blockIdx.y;
  const AttnSequence s = attn_sequence(a, b);
  const AttnTile t = attn_tile(a, s, tile * (16 * NT), 16 * NT);
  const int from = t.begin + split * t.chunk, to = from + min(t.chunk, t.any_hi - from), in_page = (1 << a.page_shift) - 1;
  if (!tiny_pages(a, b, h, lane, from, to)) return;
  const int32_t* pages = a.table + b * a.ld_table;
  for (int nt = 0; nt < NT; ++nt) {
    const int row = min(t.first_row + nt * 16 + r16, t.last_row), token = row / a.group;
    const uint16_t* at = a.q + (int64_t)(s.first + token) * a.q_token + (int64_t)(h * a.group + row % a.group) * a.q_head;
    bf16x8_t q[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at + 64 * (i >> 1) + 16 * g + 8 * (i & 1)));
    const int lo = first_seen(a, s.old + token), hi = min(to, seen_end(a, s, s.old + token));
    __builtin_amdgcn_wave_barrier();   // (written by the lanes of the first 16)
    float* stat = stats + ((wave * NT + nt) * 16 + r16) * 2;
    const float m = stat[0];
    float l = 0.f;
    for (int t0 = from + wave * kTile; t0 < to; t0 += kWaves * kTile) {
      const int page_k = pages[min(t0 + 16 * quarter_k, to - 1) >> a.page_shift], page = pages[min(t0 + 16 * g, to - 1) >> a.page_shift];
      const bool there = page >= 0 && page < a.pages;
      const float ck = a.c * pow2_of_byte(cache_byte(a.ks[(int64_t)(there ? page : 0) * a.kv_heads + h]));
      const int slot = ((t0 + 16 * quarter_k) & in_page) + (r16 & 3);
      const uint8_t* keys = a.k + ((((int64_t)(page_k >= 0 && page_k < a.pages ? page_k : 0) * a.kv_heads + h) << a.page_shift) + slot) * D + 16 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
          const u32x4_t w = *reinterpret_cast<const u32x4_t*>(keys + (8 * (i >> 1) + 4 * (i & 1)) * D + 64 * (step >> 1));
          sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values_bf16(w[2 * (step & 1)], w[2 * (step & 1) + 1], 1.f), q[step], sc, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int token = t0 + 16 * g + 4 * i + e;
          if (there && token >= lo && token < hi) l += __builtin_amdgcn_exp2f(fmaf(sc[e], ck, -m));
        }
      }
    }
    l += xor16(l);
    l += xor32(l);
    if (g == 0) stat[1] = l;
  }
}

template <int D, int NT>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void ccq_attention_few_kernel(AttnArgs a) {
  constexpr int KP = D / 64;     // 16-byte pieces of a key in a lane: dimensions 64 p + 16 g .. + 15
  constexpr int DT = D / 16;     // tiles of dimensions
  constexpr int STEPS = D / 32;
  constexpr int kPitch = D + 4;
  __shared__ __align__(16) float joined[kWaves * 16 * NT * kPitch];
  __shared__ float stats[kWaves * 16 * NT * 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % a.kv_heads, tile = (blockIdx.x / a.kv_heads) % a.row_tiles, split = blockIdx.x / (a.kv_heads * a.row_tiles), b = blockIdx.y;
  const AttnSequence s = attn_sequence(a, b);
  const int rows = s.n * a.group, row0 = tile * (16 * NT);
  if (row0 >= rows) return;
  const AttnTile t = attn_tile(a, s, row0, 16 * NT);
  if (split >= t.splits) return;
  const int begin = t.begin + split * t.chunk, from = begin, to = begin + min(t.chunk, t.any_hi - begin);

  // queries: the same dimensions as a lane's pieces of the keys
  bf16x8_t q[NT][STEPS];
  int lo[NT], hi[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = min(row0 + nt * 16 + r16, t.last_row), token = row / a.group;
    const uint16_t* at = a.q + (int64_t)(s.first + token) * a.q_token + (int64_t)(h * a.group + row % a.group) * a.q_head;
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      q[nt][i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at + 64 * (i >> 1) + 16 * g + 8 * (i & 1)));
    lo[nt] = first_seen(a, s.old + token);
    hi[nt] = seen_end(a, s, s.old + token);
  }

  f32x4_t o[NT][DT];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt] = kLowest;
    l[nt] = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[nt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* pages = a.table + b * a.ld_table;
  const int in_page = (1 << a.page_shift) - 1;
  // Table entry of a quarter of the tile at t0; looked at a tile later (its page, -1 where there is none), so that nothing waits for it.
  auto entry_at = [&](int t0, int quarter) { return pages[min(t0 + 16 * quarter, to - 1) >> a.page_shift]; };
  auto page_of = [&](int entry) { return entry < a.pages ? entry : -1; };
  const int quarter_k = r16 >> 2;
  u32x4_t kr[4][KP], vr[DT];
  auto load_keys = [&](int t0, int page) {
    const int slot = ((t0 + 16 * quarter_k) & in_page) + (r16 & 3);
    const uint8_t* at = a.k + ((((int64_t)max(page, 0) * a.kv_heads + h) << a.page_shift) + slot) * D + 16 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int p = 0; p < KP; ++p) kr[i][p] = *reinterpret_cast<const u32x4_t*>(at + (8 * (i >> 1) + 4 * (i & 1)) * D + 64 * p);
  };
  auto load_values = [&](int t0, int page) {
    const int slot = (t0 + 16 * g) & in_page;
    const uint8_t* at = a.v + ((((int64_t)max(page, 0) * a.kv_heads + h) * D + r16) << a.page_shift) + slot;
#pragma unroll
    for (int i = 0; i < DT; ++i) vr[i] = *reinterpret_cast<const u32x4_t*>(at + ((int64_t)(16 * i) << a.page_shift));
  };

  int t0 = from + wave * kTile;
  bool tiny = false;
  const int stride = kWaves * kTile;
  if (t0 < to) {
    int pv = page_of(entry_at(t0, g)), next_k = entry_at(t0 + stride, quarter_k), next_v = entry_at(t0 + stride, g);
    load_keys(t0, page_of(entry_at(t0, quarter_k)));
    int64_t scale_at = (int64_t)max(pv, 0) * a.kv_heads + h;
    int k_byte = a.ks[scale_at], v_byte = a.vs[scale_at];
    for (; t0 < to; t0 += stride) {
      load_values(t0, pv);
      f32x4_t sc[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[nt][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
          const u32x4_t w = kr[i][step >> 1];
          const bf16x8_t key = values_bf16(w[2 * (step & 1)], w[2 * (step & 1) + 1], 1.f);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) sc[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[nt][step], sc[nt][i], 0, 0, 0);
        }
      const int v_scale = cache_byte(v_byte);
      tiny |= v_scale < 127 + kTiny;
      const float ck = a.c * pow2_of_byte(cache_byte(k_byte)), ev = (float)(v_scale - 127), inv_v = inverse_of_byte(v_scale);
      const int pv_next = page_of(next_v);
      load_keys(t0 + stride, page_of(next_k));   // (past the end the last page's, never used)
      scale_at = (int64_t)max(pv_next, 0) * a.kv_heads + h;
      k_byte = a.ks[scale_at];
      v_byte = a.vs[scale_at];
      next_k = entry_at(t0 + 2 * stride, quarter_k);
      next_v = entry_at(t0 + 2 * stride, g);
      const bool whole = t0 >= t.all_lo && t0 + kTile <= min(t.all_hi, to) && __all(pv >= 0);
      if (!whole) {
        const int token0 = t0 + 16 * g;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int first = pv >= 0 ? lo[nt] : 0x7FFFFFFF, last = min(hi[nt], to);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int token = token0 + 4 * i + e;
              if (token < first || token >= last) sc[nt][i][e] = -__builtin_inff();
            }
        }
#pragma unroll
        for (int i = 0; i < DT; ++i) vr[i] = keep_tokens(vr[i], token0, pv >= 0 ? t.any_lo : 0x7FFFFFFF, to);
      }
      f16x8_t w[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float top = sc[nt][0][0];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[nt][i][e]);
        top = fmaf(top, ck, ev);
        top = fmaxf(top, xor16(top));
        top = fmaxf(top, xor32(top));
        if (__any(top > m[nt] + kRise)) {
          const float next = top > m[nt] + kRise ? top : m[nt];
          const float f = __builtin_amdgcn_exp2f(m[nt] - next);
          m[nt] = next;
          l[nt] *= f;
#pragma unroll
          for (int i = 0; i < DT; ++i) o[nt][i] *= f;
        }
        const float bias = ev - m[nt];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(sc[nt][i][e], ck, bias));
            sum += p;
            w[nt][i >> 1][4 * (i & 1) + e] = (_Float16)p;
          }
        l[nt] = fmaf(sum, inv_v, l[nt]);
      }
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const f16x8_t val = values_f16(vr[i][2 * half], vr[i][2 * half + 1]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(val, w[nt][half], o[nt][i], 0, 0, 0);
        }
      pv = pv_next;
    }
  }

  // join the wavefronts
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += xor16(l[nt]);
    l[nt] += xor32(l[nt]);
    float* at = joined + ((wave * NT + nt) * 16 + r16) * kPitch + 4 * g;
#pragma unroll
    for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4_t*>(at + 16 * i) = o[nt][i];
    if (g == 0) {
      stats[((wave * NT + nt) * 16 + r16) * 2] = m[nt];
      stats[((wave * NT + nt) * 16 + r16) * 2 + 1] = l[nt];
    }
  }
  if (__any(tiny)) weights_again<D, NT>(stats);
  __syncthreads();
  constexpr int kQuads = D / 4;   // four dimensions to a thread
  for (int i = threadIdx.x; i < 16 * NT * kQuads; i += 64 * kWaves) {
    const int r = i / kQuads, d = i % kQuads * 4, row = row0 + r;
    if (row >= rows) continue;
    float top = kLowest;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stats[(w * 16 * NT + r) * 2]);
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(stats[(w * 16 * NT + r) * 2] - top);
      total += rescaled(stats[(w * 16 * NT + r) * 2 + 1], stats[(w * 16 * NT + r) * 2] - top);
      const f32x4_t part = *reinterpret_cast<const f32x4_t*>(joined + (w * 16 * NT + r) * kPitch + d);
      sum += part * f;
    }
    const int64_t token = s.first + row / a.group;
    const int head = h * a.group + row % a.group;
    if (a.splits > 1) {
      const int64_t at = ((int64_t)split * a.tokens + token) * a.q_heads + head;
      *reinterpret_cast<f32x4_t*>(a.part_o + at * D + d) = sum;
      if (d == 0) {
        a.part_ml[at * 2] = top;
        a.part_ml[at * 2 + 1] = total;
      }
    } else {
      const float inv = total == 0.f ? 0.f : 1.f / total;
      const u32x2_t v = {pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
      *reinterpret_cast<u32x2_t*>(a.out + token * a.o_token + head * a.o_head + d) = v;
    }
  }
}

// out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s, splits in a fixed order.  Of up to kFewSplits a thread adds four dimensions of a row, split
// after split (2 splits of 16384 rows of 128 dimensions: 15 us less than with a workgroup to a row).
constexpr int kFewSplits = 8;
__device__ __forceinline__ int splits_of(const AttnArgs& a, const AttnSequence& s, int r) {   // r: new token * q_heads + q head
  const int row = r / a.q_heads * a.group + r % a.q_heads % a.group;
  return attn_tile(a, s, row / a.tile_rows * a.tile_rows, a.tile_rows).splits;
}
template <int D>
__global__ __launch_bounds__(256) void ccq_attention_join_few_kernel(AttnArgs a) {
  constexpr int kQuads = D / 4;
  const int b = blockIdx.y, r = blockIdx.x * (256 / kQuads) + threadIdx.x / kQuads, quad = threadIdx.x % kQuads;
  const AttnSequence s = attn_sequence(a, b);
  if (r / a.q_heads >= s.n) return;
  const int64_t row = (int64_t)s.first * a.q_heads + r, rows_all = (int64_t)a.tokens * a.q_heads;
  const int splits = splits_of(a, s, r);
  float m[kFewSplits], l[kFewSplits];
  f32x4_t o[kFewSplits];
  float top = kLowest;
#pragma unroll
  for (int i = 0; i < kFewSplits; ++i) {   // (of splits that there are not: the last one's, not added)
    const int64_t at = min(i, splits - 1) * rows_all + row;
    m[i] = a.part_ml[at * 2];
    l[i] = a.part_ml[at * 2 + 1];
    o[i] = *reinterpret_cast<const f32x4_t*>(a.part_o + at * D + 4 * quad);
    top = fmaxf(top, m[i]);
  }
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < kFewSplits; ++i) {
    if (i >= splits) continue;
    const float f = __builtin_amdgcn_exp2f(m[i] - top);
    total += rescaled(l[i], m[i] - top);
    sum += o[i] * f;
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint16_t* out = a.out + (s.first + r / a.q_heads) * a.o_token + (int64_t)(r % a.q_heads) * a.o_head + 4 * quad;
  *reinterpret_cast<u32x2_t*>(out) = u32x2_t{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
}

// Of more, a workgroup has a row, its threads side by side over four dimensions each and over the splits (86 splits of one long sequence: 5.5 us, with a
// wavefront to a row, one split after the other, 27).
constexpr int kMostSplits = 1024;
template <int D>
__global__ __launch_bounds__(256) void ccq_attention_join_kernel(AttnArgs a) {
  constexpr int kQuads = D / 4, kGroups = 256 / kQuads;
  __shared__ float weight[kMostSplits], tops[4], totals[4];
  __shared__ __align__(16) float sums[kGroups * D];
  const int b = blockIdx.y, r = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const AttnSequence s = attn_sequence(a, b);
  if (r / a.q_heads >= s.n) return;
  const int64_t row = (int64_t)s.first * a.q_heads + r, rows_all = (int64_t)a.tokens * a.q_heads;
  const int splits = splits_of(a, s, r);
  float top = kLowest;
  for (int i = threadIdx.x; i < splits; i += 256) top = fmaxf(top, a.part_ml[(i * rows_all + row) * 2]);
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float total = 0.f;
  for (int i = threadIdx.x; i < splits; i += 256) {
    const float d = a.part_ml[(i * rows_all + row) * 2] - top;
    weight[i] = __builtin_amdgcn_exp2f(d);
    total += rescaled(a.part_ml[(i * rows_all + row) * 2 + 1], d);
  }
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
  if (lane == 0) totals[wave] = total;
  __syncthreads();
  total = (totals[0] + totals[1]) + (totals[2] + totals[3]);
  const int group = threadIdx.x / kQuads, quad = threadIdx.x % kQuads;
  f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = group; i < splits; i += kGroups) sum += *reinterpret_cast<const f32x4_t*>(a.part_o + (i * rows_all + row) * D + 4 * quad) * weight[i];
  *reinterpret_cast<f32x4_t*>(sums + group * D + 4 * quad) = sum;
  __syncthreads();
  if (group > 0) return;
  for (int i = 1; i < kGroups; ++i) sum += *reinterpret_cast<const f32x4_t*>(sums + i * D + 4 * quad);
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint16_t* out = a.out + (s.first + r / a.q_heads) * a.o_token + (int64_t)(r % a.q_heads) * a.o_head + 4 * quad;
  *reinterpret_cast<u32x2_t*>(out) = u32x2_t{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
}

// How a call is cut.
struct Plan {
  bool many = false;   // the kernel for many rows
  int nt = 0;          // the one for few: 16-row tiles of a workgroup
  int tile_rows = 0, row_tiles = 0, splits = 0;
  int image_tiles = 0;   // of a sequence
};
constexpr int64_t kMostImages = int64_t(4) << 30;   // bytes of workspace; past it the kernel for few rows
int64_t image_tiles(const ccq_batch* b, const ccq_attn* at) {   // of a sequence
  return (at->window > 0 ? std::min<int64_t>(b->max_len, (int64_t)at->window + b->max_new) : b->max_len) / kTile + 2;
}
thread_local int forced = -1;   // (tests: 1 the kernel for many rows, 0 the one for few)
Plan plan_of(const ccq_cache* c, const ccq_batch* b, const ccq_attn* at) {
  Plan p;
  const int64_t rows = (int64_t)b->max_new * (at->q_heads / c->kv_heads), pairs = (int64_t)b->batch * c->kv_heads;
  // The kernels for many rows take 0.02 us of the chip for an image, read by every 256 rows, and 1.7 us of a CU for a tile of 256 rows; the one for few takes 3 us
  // for that, but in pieces of 32 rows and of single wavefronts.  The first win where an image is read six times and every CU gets eight tiles (2048 rows of
  // 32 / 8 heads, 16384 tokens: 441 against 670 us; 512 rows, 2048 tokens: 42 against 32; measured over 366 shapes, 1 % from the better of the two on average).  Heads of 64 dimensions
  // leave the kernel for few three wavefronts a SIMD: it then keeps up (4 times 512 rows, 16384 tokens: 244 us against 379).
  if (c->head_dim == 128) {
    const int64_t mean = at->window > 0 ? std::min<int64_t>(at->window, b->max_len) : at->causal ? b->max_len - b->max_new / 2 : b->max_len;
    const int64_t tiles = (rows + kManyRows - 1) / kManyRows;
    p.many = tiles >= 6 && tiles * pairs * (mean / kTile) >= 8 * 256 && image_tiles(b, at) * pairs * kImageBytes <= kMostImages;
  }
  if (forced >= 0) p.many = forced == 1 && c->head_dim == 128;
  if (!p.many) p.nt = rows <= 16 ? 1 : 2;
  p.tile_rows = p.many ? kManyRows : 16 * p.nt;
  p.row_tiles = (int)((rows + p.tile_rows - 1) / p.tile_rows);
  // tokens that a tile of rows can see
  int64_t range = b->max_len;
  if (at->window > 0) range = std::min<int64_t>(range, (int64_t)at->window + std::min<int64_t>(b->max_new, p.tile_rows / (at->q_heads / c->kv_heads) + 1) + 63);
  static_assert(kUnit == kWaves * kTile, "");
  const int64_t units = std::max<int64_t>(1, (range + kUnit - 1) / kUnit), groups = pairs * p.row_tiles;
  // Split so far that every place for a workgroup has one (one a CU for many rows, two for few): further, the parts and the second launch cost more than
  // shorter pieces bring (64 sequences of up to 8192, 8 heads: 131 us whole, 135 in two, 144 in four; 131072 tokens of 8 heads: 55 us in 32 or 64 pieces, 60 in
  // 86; 16 sequences of up to 2048: 20 us whole, 16.5 in four; for many rows
  // 240 workgroups: 50 us whole, 74 in two).  Up to 768 tokens the second launch alone costs more (one sequence of 512: 7.5 us against 9.1).
  const int64_t places = p.many ? 256 : 2 * 256;
  int64_t splits = groups >= places || units <= 3 ? 1 : std::min((places + (p.many ? 0 : groups - 1)) / groups, units);
  splits = std::min<int64_t>(splits, kMostSplits);
  const int64_t per = (units + splits - 1) / splits;
  p.splits = (int)((units + per - 1) / per);
  if (p.many) p.image_tiles = (int)image_tiles(b, at);
  return p;
}

template <int D>
int launch_join(const AttnArgs& a, hipStream_t s) {
  const unsigned rows = (unsigned)(a.max_new * a.q_heads), at_once = 256 / (D / 4);
  if (a.splits <= kFewSplits) hipLaunchKernelGGL((ccq_attention_join_few_kernel<D>), dim3((rows + at_once - 1) / at_once, (unsigned)a.batch), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((ccq_attention_join_kernel<D>), dim3(rows, (unsigned)a.batch), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

template <int D>
int launch_few(const AttnArgs& a, const Plan& p, hipStream_t s) {
  const dim3 grid((unsigned)(a.kv_heads * a.row_tiles * a.splits), (unsigned)a.batch);
  if (p.nt == 1) hipLaunchKernelGGL((ccq_attention_few_kernel<D, 1>), grid, dim3(64 * kWaves), 0, s, a);
  else hipLaunchKernelGGL((ccq_attention_few_kernel<D, 2>), grid, dim3(64 * kWaves), 0, s, a);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

// Partial results of the splits.
int64_t parts_bytes(const Plan& p, const ccq_cache* c, const ccq_batch* b, const ccq_attn* at) {
  return p.splits > 1 ? ((int64_t)p.splits * b->tokens * at->q_heads * (c->head_dim + 2) * 4 + 255) / 256 * 256 : 0;
}

}  // namespace

int64_t attention_workspace(const ccq_cache* c, const ccq_batch* b, const ccq_attn* at) {
  if (b->batch == 0 || b->max_new == 0) return 0;
  const Plan p = plan_of(c, b, at);
  return parts_bytes(p, c, b, at) + (int64_t)p.image_tiles * b->batch * c->kv_heads * (kImageBytes + 32);
}

int launch_attention(const ccq_cache* c, const ccq_batch* b, const ccq_attn* at, const ccq_heads* q, const ccq_heads* out, void* workspace, void* stream) {
  if (b->batch == 0 || b->max_new == 0) return CCQ_OK;
  const Plan p = plan_of(c, b, at);
  const int threads = p.many ? 2 * kManyRows : 64 * kWaves;
  if (b->batch > 65535 || (int64_t)c->kv_heads * p.image_tiles > most_groups(threads) || (int64_t)c->kv_heads * p.row_tiles * p.splits > most_groups(threads)) return CCQ_ERR_BAD_PARAM;
  AttnArgs a = {};
  a.k = static_cast<const uint8_t*>(c->k), a.v = static_cast<const uint8_t*>(c->v), a.ks = c->k_scales, a.vs = c->v_scales;
  a.q = static_cast<const uint16_t*>(q->data), a.q_token = q->token_stride, a.q_head = q->head_stride;
  a.out = static_cast<uint16_t*>(out->data), a.o_token = out->token_stride, a.o_head = out->head_stride;
  a.offsets = b->offsets, a.lens = b->lens, a.table = b->table, a.ld_table = b->ld_table;
  a.pages = c->pages, a.page_shift = __builtin_ctz((unsigned)c->page_tokens), a.kv_heads = c->kv_heads, a.q_heads = at->q_heads;
  a.group = at->q_heads / c->kv_heads, a.table_width = b->table_width, a.batch = b->batch, a.tokens = b->tokens, a.max_new = b->max_new, a.max_len = b->max_len;
  a.causal = at->causal, a.window = at->window, a.c = at->scale * 1.4426950408889634f;
  a.splits = p.splits, a.row_tiles = p.row_tiles, a.tile_rows = p.tile_rows;
  if (p.splits > 1) {
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o + (int64_t)p.splits * b->tokens * at->q_heads * c->head_dim;
  }
  if (p.many) {
    a.images = static_cast<uint8_t*>(workspace) + parts_bytes(p, c, b, at);
    a.image_tiles = p.image_tiles;
    a.image_scales = reinterpret_cast<float*>(a.images + (int64_t)p.image_tiles * b->batch * c->kv_heads * kImageBytes);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rc = p.many ? launch_attention_rows(a, stream) : c->head_dim == 64 ? launch_few<64>(a, p, s) : launch_few<128>(a, p, s);
  if (rc != CCQ_OK || p.splits == 1) return rc;
  return c->head_dim == 64 ? launch_join<64>(a, s) : launch_join<128>(a, s);
}

// For tests, no part of the interface: all calls of this thread from now on take the kernel for many rows (1), the one for few (0), or (-1) what the rule says.
extern "C" void ccq_attention_force(int32_t kernel) { forced = kernel; }

}  // namespace ccq
