// Attention over the paged 8-bit cache for many rows: chunks of prompts.
//
// A first kernel converts the cached tokens that rows see, 64 at a time, to images of what the second has in LDS: keys in bf16 with their scale, values in fp16
// (converted by every workgroup for itself they cost a quarter of its time).  Then a wavefront holds 32 rows, a workgroup eight of them, and walks the images:
//   scores^T = K q^T   MFMA 32x32x16 bf16, cached tokens as rows
//   out^T    = V^T p^T MFMA 32x32x16 f16, dimensions as rows
// As in the kernel for few rows, tokens are dealt to the first product's rows so that a lane's scores lie in the order in which the second product wants
// its operand: the weights stay in registers.  Scales of values and pages that are not there enter as the exponent added to a score
// (-inf for the latter).  Only tiles that not all of a wavefront's rows see whole are masked.
// A tile costs a wavefront 32 MFMAs (1024 cycles) and 1070 cycles of vector instructions (32 scores a lane: largest, multiply-add, exp2, sum, fp16).  Left to
// themselves the two wavefronts of a SIMD do the same at the same time; so the second four are half a tile behind: while one multiplies (values of the last
// tile, keys of this one, operands read eight products ahead) the other has its softmax.  One barrier a tile holds them there (two, one a half: 4 % slower).  The
// weights are pinned to their half, or the compiler moves the exp2 behind the barrier.  Images go to LDS by buffer loads: with global ones to LDS under way the compiler
// waits for all LDS reads at once.
// A chunk of 2048 after 2048 tokens (56 / 8 heads): 178 - 186 us, 8 of them for the images, 1.0 PFLOP/s (an earlier form 222 with the conversion in the kernel itself and no halves).  Bound by
// issue and power (zeros for data: 15 % less time), and the chip is idle for a fifth of the time at the end, as 448 workgroups of unequal length meet 256 CUs.
// Slower: four wavefronts of 64 rows, whose accumulators leave the registers that vector instructions reach.
#include <type_traits>

#include "ccq_attention.h"

namespace ccq {

namespace {

constexpr int D = 128, kTile = 64, kThreads = 2 * kManyRows, kKeys = kTile * D * 2, kImage = 2 * kKeys, kLds = 3 * (kImage + 256);
static_assert(kImage == kImageBytes, "");
static_assert(kTile * D / 16 == kThreads, "a thread converts 16 keys' and 16 values' bytes");

// A tile's keys in bf16, with their scale, and values in fp16, in the order in which they lie in LDS (rows of a token's dimensions, and of a dimension's
// tokens; 16-byte pieces of a row exchanged by its number, so that the operand reads of neighbouring rows meet all banks), and four exponents of values and
// their 2^-e.  Nothing of pages that are not there (the exponent -inf), nothing of values that no row sees.
__global__ __launch_bounds__(kThreads) void ccq_attention_images_kernel(AttnArgs a) {
  const int head = blockIdx.x % a.kv_heads, n = blockIdx.x / a.kv_heads, b = blockIdx.y;
  const AttnSequence s = attn_sequence(a, b);
  const int t0 = image_begin(a, s) + n * kTile;
  if (s.n <= 0 || t0 >= s.len) return;
  const int32_t* pages = a.table + b * a.ld_table;
  const int in_page = (1 << a.page_shift) - 1, piece = threadIdx.x;
  // piece p of the keys is 16 dimensions of a token, of the values 16 tokens of a dimension
  const int t = piece / (D / 16), c = piece % (D / 16), d = piece >> 2, quarter = piece & 3;
  int k_page = pages[min(t0 + t, s.len - 1) >> a.page_shift], v_page = pages[min(t0 + 16 * quarter, s.len - 1) >> a.page_shift];
  k_page = k_page < a.pages ? k_page : -1, v_page = v_page < a.pages ? v_page : -1;
  const int64_t k_tile = (int64_t)max(k_page, 0) * a.kv_heads + head, v_tile = (int64_t)max(v_page, 0) * a.kv_heads + head;
  u32x4_t k = *reinterpret_cast<const u32x4_t*>(a.k + ((k_tile << a.page_shift) + ((t0 + t) & in_page)) * D + c * 16);
  u32x4_t v = *reinterpret_cast<const u32x4_t*>(a.v + ((v_tile * D + d) << a.page_shift) + ((t0 + 16 * quarter) & in_page));
  const float k_scale = pow2_of_byte(cache_byte(a.ks[k_tile]));
  const int v_byte = cache_byte(a.vs[v_tile]);
  if (k_page < 0) k = u32x4_t{0, 0, 0, 0};
  v = keep_tokens(v, t0 + 16 * quarter, v_page < 0 ? 0x7FFFFFFF : first_seen(a, s.old), s.len);
  const int64_t image = ((int64_t)b * a.kv_heads + head) * a.image_tiles + n;
  uint8_t* keys = a.images + image * kImage + t * (2 * D);
  uint8_t* values = a.images + image * kImage + kKeys + d * (2 * kTile);
  const int k_swizzle = t & 15, v_swizzle = (d ^ (d >> 3 & 1)) & 7;
  *reinterpret_cast<bf16x8_t*>(keys + (((2 * c) ^ k_swizzle) * 16)) = values_bf16(k[0], k[1], k_scale);
  *reinterpret_cast<bf16x8_t*>(keys + (((2 * c + 1) ^ k_swizzle) * 16)) = values_bf16(k[2], k[3], k_scale);
  *reinterpret_cast<f16x8_t*>(values + (((2 * quarter) ^ v_swizzle) * 16)) = values_f16(v[0], v[1]);
  *reinterpret_cast<f16x8_t*>(values + (((2 * quarter + 1) ^ v_swizzle) * 16)) = values_f16(v[2], v[3]);
  if (piece < 4) {
    a.image_scales[image * 8 + piece] = v_page < 0 ? -__builtin_inff() : (float)(v_byte - 127);
    a.image_scales[image * 8 + 4 + piece] = v_page < 0 ? 0.f : inverse_of_byte(v_byte);
  }
}

// LDS reads may be under way across it.
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void ccq_attention_rows_kernel(AttnArgs a) {
  constexpr int DT = D / 32, STEPS = D / 16;
  extern __shared__ __align__(256) uint8_t lds[];   // three images, and 256 bytes for the exponents of each
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
  const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, tile = a.row_tiles - 1 - rest % a.row_tiles, split = rest / a.row_tiles, b = blockIdx.y;
  const AttnSequence s = attn_sequence(a, b);
  const int rows = s.n * a.group, row0 = tile * kManyRows;
  if (row0 >= rows) return;
  const AttnTile all = attn_tile(a, s, row0, kManyRows);   // of the workgroup
  if (split >= all.splits) return;
  const int from = all.begin + split * all.chunk, to = from + min(all.chunk, all.any_hi - from);
  const AttnTile own = attn_tile(a, s, min(row0 + wave * 32, all.last_row), 32);   // of the wavefront
  const int all_lo = own.all_lo, all_hi = own.all_hi, last_row = all.last_row;

  const int row = min(row0 + wave * 32 + l32, last_row), token = row / a.group, q_head = head * a.group + row % a.group;
  const int lo = first_seen(a, s.old + token), hi = min(to, seen_end(a, s, s.old + token));
  bf16x8_t q[STEPS];
  {
    const uint16_t* at = a.q + (int64_t)(s.first + token) * a.q_token + (int64_t)q_head * a.q_head + 8 * h;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(at + 16 * i));
  }

  const int first_tile = (from - image_begin(a, s)) / kTile, tiles = from < to ? (to - from + kTile - 1) / kTile : 0;
  const int64_t image0 = ((int64_t)b * a.kv_heads + head) * a.image_tiles + first_tile;
  const uint8_t* images = a.images + image0 * kImage;
  auto copy = [&](int n, int slot) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(images) + (int64_t)n * kImage, 0, kImage, 4 << 15);   // (data format 32 bits)
#pragma unroll
    for (int i = 0; i < kImage / 1024 / 8; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(lds + slot * kImage + i * 8192 + wave * 1024), 16, lane * 16, i * 8192 + wave * 1024, 0, 0);
    if (wave == 0) {
      const auto scales = __builtin_amdgcn_make_buffer_rsrc(a.image_scales + (image0 + n) * 8, 0, 32, 4 << 15);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(scales, (__attribute__((address_space(3))) void*)(lds + 3 * kImage + slot * 256), 4, lane * 4, 0, 0, 0);
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

  f32x16_t sc[2];
  f16x8_t w[4];
  // operand p of a step: the values of the tile before (the first kValueOperands), then the keys of the tile
  constexpr int kValueOperands = 4 * DT, kOperands = kValueOperands + 2 * STEPS, kAhead = 8;
  u32x4_t operand[kAhead];
  auto read_operand = [&](int p, int before, int slot) {
    const uint8_t* at = p < kValueOperands ? lds + before * kImage + kKeys + (p % DT * 32 + l32) * (2 * kTile) + (((2 * (p / DT) + h) ^ value_swizzle) * 16)
                                           : lds + slot * kImage + ((p & 1) * 32 + key_token) * (2 * D) + (((p - kValueOperands) / 2 * 2 + h) ^ key_swizzle) * 16;
    operand[p % kAhead] = *reinterpret_cast<const u32x4_t*>(at);
  };
  auto read_ahead = [&](int first, int before, int slot) {
#pragma unroll
    for (int p = 0; p < kAhead; ++p) read_operand(first + p, before, slot);
  };
  auto multiply = [&](auto FIRST, auto LAST, int before, int slot) {
    constexpr int first = decltype(FIRST)::value, last = decltype(LAST)::value;
    if constexpr (last == kOperands) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[tt][e] = 0.f;
    }
#pragma unroll
    for (int p = first; p < last; ++p) {
      const u32x4_t x = operand[p % kAhead];
      if (p < kValueOperands) o[p % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, x), w[p / DT], o[p % DT], 0, 0, 0);
      else sc[p & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x), q[(p - kValueOperands) / 2], sc[p & 1], 0, 0, 0);
      if (p + kAhead < last) read_operand(p + kAhead, before, slot);
    }
#pragma unroll
    for (int p = first; p < last; ++p) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      if (p + kAhead < last) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
  };
  bool gone = false;   // whether a page is missing: its scores are masked then, for the sake of queries that hold NaN or infinities
  float least = 0.f;   // exponent of values, or less
  auto softmax = [&](int n, int slot) {
    const int t0 = from + n * kTile;
    const f32x4_t ev = *reinterpret_cast<const f32x4_t*>(lds + 3 * kImage + slot * 256), inv = *reinterpret_cast<const f32x4_t*>(lds + 3 * kImage + slot * 256 + 16);
    __builtin_amdgcn_sched_barrier(0);
    bool masked = t0 < all_lo || t0 + kTile > all_hi || t0 + kTile > to;
    if (gone) masked |= __any(fminf(fminf(ev[0], ev[1]), fminf(ev[2], ev[3])) == -__builtin_inff());
    if (masked) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = t0 + 32 * tt + 16 * (e >> 3) + 8 * h + (e & 7);
          if (t < lo || t >= hi || ev[2 * tt + (e >> 3)] == -__builtin_inff()) sc[tt][e] = -__builtin_inff();
        }
    }
    float most[4], top = kLowest;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      most[i] = -__builtin_inff();   // (from here on pairs: three-operand instructions)
#pragma unroll
      for (int e = 0; e < 8; e += 2) most[i] = fmaxf(fmaxf(most[i], sc[i >> 1][8 * (i & 1) + e]), sc[i >> 1][8 * (i & 1) + e + 1]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaf(most[i], a.c, ev[i]));
    least = fminf(fminf(fminf(least, ev[0]), ev[1]), fminf(ev[2], ev[3]));
    top = fmaxf(top, xor32(top));
    if (__any(top > m + kRise)) {
      const float next = top > m + kRise ? top : m;
      const float f = __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float bias = ev[i] - m;
      float sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sc[i >> 1][8 * (i & 1) + e], a.c, bias));
        sum = e == 0 ? p : sum + p;
        w[i][e] = (_Float16)p;
      }
      l = fmaf(sum, inv[i], l);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(w[i]));   // the weights are made here, not where they are used
    asm volatile("" : "+v"(l));
  };
  // Between two barriers the first four wavefronts multiply and then have the softmax of tile n, the others have the softmax of tile n - 1 and then multiply.  Where
  // tile n + 1 goes, tile n - 2 lay, last read before the barrier before.
  const std::integral_constant<int, 0> zero;
  const std::integral_constant<int, kValueOperands> values_end;
  const std::integral_constant<int, kOperands> end;
  const int behind = wave >> 2;
  if (tiles > 0) {
    copy(0, 0);
    if (1 < tiles) copy(1, 1);
    // (once, beside the first copies: looked for in each tile's exponents alone it cost 1.7 % of the whole)
    for (int i = (from >> a.page_shift) + lane; i <= (to - 1) >> a.page_shift; i += 64) {
      const int page = a.table[b * a.ld_table + i];
      gone |= page < 0 || page >= a.pages;
    }
    gone = __any(gone);
    wait_loads<0>();
    barrier();
    read_ahead(kValueOperands, 0, 0);
    multiply(values_end, end, 0, 0);
    if (behind) barrier();
    int slot = 1;   // of tile n
    for (int n = 1; n < tiles; ++n) {
      const int before = slot == 0 ? 2 : slot - 1, next = slot == 2 ? 0 : slot + 1;
      if (behind && n + 1 < tiles) copy(n + 1, next);
      __builtin_amdgcn_sched_barrier(0);
      softmax(n - 1, before);
      read_ahead(0, before, slot);
      __builtin_amdgcn_sched_barrier(0);
      if (!behind) {
        wait_loads<0>();
        barrier();
        if (n + 1 < tiles) copy(n + 1, next);
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      multiply(zero, end, before, slot);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      if (behind) {
        wait_loads<0>();
        barrier();
      }
      slot = next;
    }
    const int before = slot == 0 ? 2 : slot - 1;
    softmax(tiles - 1, before);
    if (!behind) barrier();
    read_ahead(0, before, slot);
    multiply(zero, values_end, before, slot);
  }
  if (__any(least < (float)kTiny) && tiny_pages(a, b, head, lane, from, to)) {   // the sums of weights once more, from the keys of the images as they lie in memory
    l = 0.f;
    for (int n = 0; n < tiles; ++n) {
      const uint8_t* keys = images + (int64_t)n * kImage + key_token * (2 * D);
      const f32x4_t ev = *reinterpret_cast<const f32x4_t*>(a.image_scales + (image0 + n) * 8);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        f32x16_t s2;
#pragma unroll
        for (int e = 0; e < 16; ++e) s2[e] = 0.f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const u32x4_t key = *reinterpret_cast<const u32x4_t*>(keys + tt * 32 * 2 * D + (((2 * i + h) ^ key_swizzle) * 16));
          s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, key), q[i], s2, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int t = from + n * kTile + 32 * tt + 16 * (e >> 3) + 8 * h + (e & 7);
          if (t >= lo && t < hi && ev[2 * tt + (e >> 3)] != -__builtin_inff()) l += __builtin_amdgcn_exp2f(fmaf(s2[e], a.c, -m));
        }
      }
    }
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
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(ccq_attention_rows_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return CCQ_ERR_HIP;
  hipLaunchKernelGGL(ccq_attention_images_kernel, dim3((unsigned)(a.kv_heads * a.image_tiles), (unsigned)a.batch), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(ccq_attention_rows_kernel, dim3((unsigned)(a.kv_heads * a.row_tiles * a.splits), (unsigned)a.batch), dim3(kThreads), kLds, s, a);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
