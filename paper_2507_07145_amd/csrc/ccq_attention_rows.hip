// Attention over the paged 8-bit cache for many rows: chunks of prompts.
//
// A wavefront holds 32 rows, a workgroup eight of them; the workgroup walks the cached tokens that its rows see in tiles of 64.  Keys and values of
// the next tile are converted on their way to LDS (keys to bf16 with their scale, values to fp16), once for all rows:
//   scores^T = K q^T   MFMA 32x32x16 bf16, cached tokens as rows
//   out^T    = V^T p^T MFMA 32x32x16 f16, dimensions as rows
// As in the kernel for few rows, tokens are dealt to the first product's rows so that a lane's scores lie in the order in which the second product wants
// its operand: the weights stay in registers.  Scales of values and pages that are not there enter as the exponent added to a score
// (-inf for the latter).  Only tiles that not all of a wavefront's rows see whole are masked.
// A tile costs a wavefront 32 MFMAs (1024 cycles) and 1350 cycles of the vector unit (32 scores a lane: largest, multiply-add, exp2, sum, fp16; its share of
// the conversions), and the two wavefronts of a SIMD overlap only a part of them: 2.1 us a tile.  A chunk of 2048 after 2048 tokens (56 / 8 heads): 217 us, 0.84
// PFLOP/s; counters say 35% of the time in MFMAs, 55% of vector instructions, LDS 25%.  Tried and no faster: half of the wavefronts half a tile behind, with
// barriers between (225 us), conversions and exp2 dealt out between the MFMAs (211 to 231).  Slower: four wavefronts of 64 rows, whose accumulators
// leave the registers that vector instructions reach.
#include "ccq_attention.h"

namespace ccq {

namespace {

constexpr int D = 128, kTile = 64;

__global__ __launch_bounds__(2 * kManyRows) __attribute__((amdgpu_waves_per_eu(2, 2))) void ccq_attention_rows_kernel(AttnArgs a) {
  constexpr int DT = D / 32, STEPS = D / 16;
  constexpr int kKeyRow = 2 * D, kKeys = kTile * kKeyRow, kValues = D * kTile * 2, kStage = kKeys + kValues;
  constexpr int kPieces = kTile * D / 16;   // 16-byte pieces of a tile's keys, and of its values
  static_assert(kPieces == 2 * kManyRows, "a piece to a thread");
  __shared__ __align__(256) uint8_t lds[2 * kStage];
  __shared__ float exponents[2][4], inverses[2][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
  const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, tile = a.row_tiles - 1 - rest % a.row_tiles, split = rest / a.row_tiles, b = blockIdx.y;
  const AttnSequence s = attn_sequence(a, b);
  const int rows = s.n * a.group, row0 = tile * kManyRows;
  if (row0 >= rows) return;
  const AttnTile w = attn_tile(a, s, row0, kManyRows);   // of the workgroup
  if (split >= w.splits(a)) return;
  const int from = w.begin + split * a.chunk, to = from + min(a.chunk, w.any_hi - from);
  const AttnTile own = attn_tile(a, s, min(row0 + wave * 32, w.last_row), 32);   // of the wavefront
  const int all_lo = own.all_lo, all_hi = own.all_hi, any_lo = w.any_lo, wave_lo = own.any_lo, wave_hi = min(to, own.any_hi), last_row = w.last_row;

  const int row = min(row0 + wave * 32 + l32, last_row), token = row / a.group, q_head = head * a.group + row % a.group;
  const int lo = first_seen(a, s.old + token), hi = min(to, seen_end(a, s, s.old + token));
  bf16x8_t q[STEPS];
  {
    const uint16_t* at = a.q + (int64_t)(s.first + token) * a.q_token + (int64_t)q_head * a.q_head + 8 * h;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at + 16 * i));
  }

  // staging: piece p of the keys is 16 dimensions of a token, of the values 16 tokens of a dimension
  const int32_t* pages = a.table + b * a.ld_table;
  const int in_page = (1 << a.page_shift) - 1;
  constexpr int kTokenPieces = D / 16;
  const int piece = threadIdx.x, key_piece_token = piece / kTokenPieces;
  u32x4_t kr, vr;
  int k_page, v_page, k_byte, v_byte, k_next, v_next;   // of what kr and vr hold; pages of the tile after it
  auto find_pages = [&](int t0) {   // looked at a tile later: no wait for memory here
    k_next = pages[min(t0 + key_piece_token, to - 1) >> a.page_shift];
    v_next = pages[min(t0 + 16 * (piece & 3), to - 1) >> a.page_shift];
  };
  const uint32_t page_bytes = (uint32_t)D << a.page_shift;   // of a head
  const uint32_t k_inner = piece % kTokenPieces * 16, v_inner = (uint32_t)(piece >> 2) << a.page_shift;
  auto load = [&](int t0) {   // of pages found before; past the end page 0, never stored
    k_page = k_next < a.pages ? k_next : -1, v_page = v_next < a.pages ? v_next : -1;
    const uint32_t k_tile = (uint32_t)max(k_page, 0) * a.kv_heads + head, v_tile = (uint32_t)max(v_page, 0) * a.kv_heads + head;
    kr = *reinterpret_cast<const u32x4_t*>(a.k + ((uint64_t)k_tile * page_bytes + (((t0 + key_piece_token) & in_page) * D + k_inner)));
    vr = *reinterpret_cast<const u32x4_t*>(a.v + ((uint64_t)v_tile * page_bytes + (((t0 + 16 * (piece & 3)) & in_page) + v_inner)));
    k_byte = a.ks[k_tile];
    v_byte = a.vs[v_tile];
  };
  auto store = [&](int t0, int stage) {   // what kr and vr hold, the tile at t0
    const int t = key_piece_token, c = piece % kTokenPieces * 2, d = piece >> 2, v = (piece & 3) * 2;
    uint8_t* keys = lds + stage * kStage + t * kKeyRow;
    uint8_t* values = lds + stage * kStage + kKeys + d * (2 * kTile);
    u32x4_t k = kr, x = vr;
    if (__any(k_page < 0)) k = k_page < 0 ? u32x4_t{0, 0, 0, 0} : k;
    const float scale = pow2_of_byte(k_byte);
    const int k_swizzle = t & 15, v_swizzle = (d ^ (d >> 3 & 1)) & 7;
    *reinterpret_cast<bf16x8_t*>(keys + ((c ^ k_swizzle) * 16)) = values_bf16(k[0], k[1], scale);
    *reinterpret_cast<bf16x8_t*>(keys + (((c + 1) ^ k_swizzle) * 16)) = values_bf16(k[2], k[3], scale);
    if (t0 < any_lo || t0 + kTile > to || __any(v_page < 0)) x = keep_tokens(x, t0 + 16 * (piece & 3), v_page < 0 ? 0x7FFFFFFF : any_lo, to);
    *reinterpret_cast<f16x8_t*>(values + ((v ^ v_swizzle) * 16)) = values_f16(x[0], x[1]);
    *reinterpret_cast<f16x8_t*>(values + (((v + 1) ^ v_swizzle) * 16)) = values_f16(x[2], x[3]);
    if (threadIdx.x < 4) {
      exponents[stage][piece] = v_page < 0 ? -__builtin_inff() : (float)(v_byte - 127);
      inverses[stage][piece] = v_page < 0 ? 0.f : inverse_of_byte(v_byte);
    }
  };

  f32x16_t o[DT];
  float m = kLowest, l = 0.f;
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;

  // a lane's operands: of the keys the token of row l32 (bits 2 and 3 of a row's number are exchanged), of the values dimension l32 of a tile
  const int key_token = (l32 & 0x13) | (l32 & 8) >> 1 | (l32 & 4) << 1;
  const int key_swizzle = key_token & 15, value_swizzle = (l32 ^ (l32 >> 3 & 1)) & 7;

  if (from < to) {
    find_pages(from);
    load(from);
    find_pages(from + kTile);
    store(from, 0);
    load(from + kTile);
    find_pages(from + 2 * kTile);
    __syncthreads();
  }
  int stage = 0;
  for (int t0 = from; t0 < to; t0 += kTile, stage ^= 1) {
    if (t0 + kTile < to) {
      store(t0 + kTile, stage ^ 1);
      load(t0 + 2 * kTile);   // (past the end: page 0, never stored)
      find_pages(t0 + 3 * kTile);
    }
    const uint8_t* keys = lds + stage * kStage;
    const uint8_t* values = keys + kKeys;
    if (t0 + kTile > wave_lo && t0 < wave_hi) {   // else none of the wavefront's rows sees the tile
      f32x16_t sc[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[tt][e] = 0.f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const bf16x8_t key = *reinterpret_cast<const bf16x8_t*>(keys + (tt * 32 + key_token) * kKeyRow + (((2 * i + h) ^ key_swizzle) * 16));
          sc[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, q[i], sc[tt], 0, 0, 0);
        }
      }
      if (t0 < all_lo || t0 + kTile > all_hi || t0 + kTile > to) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int t = t0 + 32 * tt + 16 * (e >> 3) + 8 * h + (e & 7);
            if (t < lo || t >= hi) sc[tt][e] = -__builtin_inff();
          }
      }
      float ev[4], top = kLowest;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ev[i] = exponents[stage][i];
        float most = sc[i >> 1][8 * (i & 1)];
#pragma unroll
        for (int e = 1; e < 8; ++e) most = fmaxf(most, sc[i >> 1][8 * (i & 1) + e]);
        top = fmaxf(top, fmaf(most, a.c, ev[i]));
      }
      top = fmaxf(top, xor32(top));
      if (__any(top > m + kRise)) {
        const float next = top > m + kRise ? top : m;
        const float f = __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] *= f;
      }
      f16x8_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float bias = ev[i] - m;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sc[i >> 1][8 * (i & 1) + e], a.c, bias));
          sum += p;
          w[i][e] = (_Float16)p;
        }
        l = fmaf(sum, inverses[stage][i], l);
      }
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f16x8_t value = *reinterpret_cast<const f16x8_t*>(values + (i * 32 + l32) * (2 * kTile) + (((2 * j + h) ^ value_swizzle) * 16));
          o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value, w[j], o[i], 0, 0, 0);
        }
    }
    __syncthreads();
  }

  // register e of a lane: dimension 8 (e / 4) + 4 h + e % 4 of its tile
  l += xor32(l);
  if (row0 + wave * 32 + l32 > last_row) return;
  if (a.splits > 1) {
    const int64_t at = ((int64_t)split * a.tokens + s.first + token) * a.q_heads + q_head;
    float* out = a.part_o + at * D + 4 * h;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<f32x4_t*>(out + 32 * i + 8 * e) = f32x4_t{o[i][4 * e], o[i][4 * e + 1], o[i][4 * e + 2], o[i][4 * e + 3]};
    if (h == 0) {
      a.part_ml[at * 2] = m;
      a.part_ml[at * 2 + 1] = l;
    }
  } else {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* out = a.out + (int64_t)(s.first + token) * a.o_token + (int64_t)q_head * a.o_head + 4 * h;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<u32x2_t*>(out + 32 * i + 8 * e) =
            u32x2_t{pack_bf16(o[i][4 * e] * inv, o[i][4 * e + 1] * inv), pack_bf16(o[i][4 * e + 2] * inv, o[i][4 * e + 3] * inv)};
  }
}

}  // namespace

int launch_attention_rows(const AttnArgs& a, void* stream) {
  const dim3 grid((unsigned)(a.kv_heads * a.row_tiles * a.splits), (unsigned)a.batch), block(2 * kManyRows);
  hipLaunchKernelGGL(ccq_attention_rows_kernel, grid, block, 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
