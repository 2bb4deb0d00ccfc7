// What the 8-bit product's kernels share.
//
//   y[m][n] = sum_b 2^ex[m][b] s[n / 128][b] sum_{k in b} x[m][k] w[n][k],   b: blocks of 128 of K
//
// One scaled MFMA, 16x16x128, covers a block of K: it starts from zero, takes the activations' power-of-two scale as its scale operand, and
// its result goes into the fp32 accumulators with one multiply-add by the weights' scale, which is one number for the whole
// tile.  The weights are the first operand: a lane then holds four neighbouring outputs of a row.
#pragma once
#include "ccq_layer.h"

namespace ccq {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

struct Gemm8Args {
  const uint8_t* w;
  const float* ws;
  const uint8_t* x;
  const uint8_t* xs;
  uint16_t* y;
  float* partial;       // fp32 [shares][M][ld_partial]
  int64_t ldw, ld_ws, ldx, ld_xs, ldy, ld_partial;   // ld_partial: N rounded up to a multiple of 4
  int32_t M, N, K, blocks;   // blocks: of K, the last one possibly shorter
  const uint16_t* x16;       // bf16 rows in place of x and xs, quantized by the kernels for few rows (null: none)
  int64_t ldx16;
};

__device__ __forceinline__ i32x8_t operand8(u32x4_t a, u32x4_t b) {
  return i32x8_t{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}
// 16 bf16 values of a row, on their way to codes; a row may start at any of them.
struct Wide16 {
  u32x4_t v[2];
};
__device__ __forceinline__ Wide16 load_wide16(const uint16_t* p, bool there) {
  Wide16 x = {};
  if (there) __builtin_memcpy(&x, p, 32);
  return x;
}
// The largest magnitude among them, as an fp32 number's bits.
__device__ __forceinline__ uint32_t magnitude16(const Wide16& x) {
  typedef __attribute__((ext_vector_type(2))) unsigned short pair;
  pair most = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(pair, x.v[i >> 2][i & 3] & 0x7FFF7FFFu));
  return (uint32_t)(most.x > most.y ? most.x : most.y) << 16;
}
// Their codes by the largest magnitude of their block: what ccq_quantize8 writes.
__device__ __forceinline__ u32x4_t codes16(const Wide16& x, uint32_t top) {
  const float inv = inverse_of_byte(scale_byte(top, kRowsByteLo, kRowsByteHi));
  u32x4_t q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = x.v[i >> 1][2 * (i & 1)], b = x.v[i >> 1][2 * (i & 1) + 1];
    q[i] = top >= kInfBits ? 0x7F7F7F7Fu : pack_e4m3(bf16_lo(a) * inv, bf16_hi(a) * inv, bf16_lo(b) * inv, bf16_hi(b) * inv);
  }
  return q;
}
__device__ __forceinline__ int scale_of(uint32_t top) { return top >= kInfBits ? 255 : scale_byte(top, kRowsByteLo, kRowsByteHi); }
// A block of K: weights times activations, scaled by the activations' scale byte (the low byte of `x_scale`).
__device__ __forceinline__ f32x4_t multiply8(i32x8_t w, i32x8_t x, int x_scale) {
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, 0, 0, 0x7F7F7F7F, 0, x_scale);
}

// All wavefronts' LDS reads and writes before it are done, their copies from memory not: those are waited for by wait_loads.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  asm volatile("s_barrier" ::: "memory");
}

// Blocks of 64 mi rows (mi 1, 2, 4) and 256 columns, K in `shares` (more than one: fp32 partial results in a.partial).
int launch_gemm8_block(const Gemm8Args& a, int mi, int shares, void* stream);

// Tiles of 16 mt rows (mt 1, 2, 3, 4, 6) and 128 columns.  A workgroup's LDS holds two steps of activations and the row scales of its whole share of K, then its sums.
constexpr int kMostLds = 160 * 1024;
constexpr int stream_blocks(int blocks, int shares) { return ((blocks + shares - 1) / shares + 1) & ~1; }   // of a share: even
constexpr int stream_pitch(int blocks_per_share) { return (blocks_per_share + 7) & ~3; }                    // bytes of a row's scales
constexpr int64_t stream_lds(int mt, int blocks_per_share) {
  const int64_t rows = 16 * mt, loop = 2 * rows * 2 * kScaleBlock + rows * stream_pitch(blocks_per_share), sums = 4 * rows * 36 * 4;
  return loop > sums ? loop : sums;
}
int launch_gemm8_stream(const Gemm8Args& a, int mt, int shares, void* stream);
int launch_gemm8_add(const Gemm8Args& a, int shares, void* stream);   // y = sum of the shares

}  // namespace ccq
