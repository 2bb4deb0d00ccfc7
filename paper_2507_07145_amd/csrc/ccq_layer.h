// What the kernels of the 8-bit layer operators share: values and scales in 8 bits, reductions over a wavefront, and the
// launchers that the host checks (ccq_layer.cpp) call.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "ccq.h"

namespace ccq {

constexpr int kScaleBlock = 128;   // columns per scale of 8-bit rows and weights
constexpr int kCacheExp = 60;      // exponents of the cache's scales lie in [-60, 60]

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

// The least e with amax <= 448 * 2^e, as e + 127: 448 = 1.75 * 2^8.  `bits`: amax's fp32 bits, finite.
__device__ __forceinline__ int scale_byte(uint32_t bits, int lo, int hi) {
  const int byte = (int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(byte, lo), hi);
}
constexpr int kRowsByteLo = 1, kRowsByteHi = 247;   // 2^-126 .. 2^120: 448 * 2^120 is past fp32's largest number
constexpr uint32_t kInfBits = 0x7F800000u;
__device__ __forceinline__ float pow2_of_byte(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }              // 2^(byte - 127), byte 1 .. 254
__device__ __forceinline__ float inverse_of_byte(int byte) { return __builtin_bit_cast(float, (uint32_t)(254 - byte) << 23); }   // its inverse, byte 1 .. 253

// Four floats (magnitudes up to 448, or NaN) as e4m3, the first in the low byte.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __builtin_bit_cast(float, v & 0xFFFF0000u); }
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) __bf16 pair;
  const pair p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// Lane l of every 16 takes the value of lane (l + N) % 16 of them.
template <int N>
__device__ __forceinline__ uint32_t ror16(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xF, 0xF, false);
}
// Largest of the 16 lanes, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, ror16<8>(v));
  v = max(v, ror16<4>(v));
  v = max(v, ror16<2>(v));
  return max(v, ror16<1>(v));
}
__device__ __forceinline__ float add16(float v) {
  v += __builtin_bit_cast(float, ror16<8>(__builtin_bit_cast(uint32_t, v)));
  v += __builtin_bit_cast(float, ror16<4>(__builtin_bit_cast(uint32_t, v)));
  v += __builtin_bit_cast(float, ror16<2>(__builtin_bit_cast(uint32_t, v)));
  return v + __builtin_bit_cast(float, ror16<1>(__builtin_bit_cast(uint32_t, v)));
}
// The value of lane l ^ 16 and of lane l ^ 32.
__device__ __forceinline__ uint32_t xor16(uint32_t v) {
  const u32x2_t r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return (threadIdx.x & 16) ? r.x : r.y;
}
__device__ __forceinline__ uint32_t xor32(uint32_t v) {
  const u32x2_t r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return (threadIdx.x & 32) ? r.x : r.y;
}
__device__ __forceinline__ float xor16(float v) { return __builtin_bit_cast(float, xor16(__builtin_bit_cast(uint32_t, v))); }
__device__ __forceinline__ float xor32(float v) { return __builtin_bit_cast(float, xor32(__builtin_bit_cast(uint32_t, v))); }

// At most n of the wavefront's loads (copies to LDS among them) are still under way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4 << 14) | 0x0F70);
}

// A launch has fewer than 2^32 threads: workgroups of `threads` of one launch; what has more is launched in parts.
constexpr int64_t most_groups(int threads) { return (int64_t(1) << 31) / threads; }

int launch_norm(const ccq_norm* n, bool norm, void* stream);
int launch_rope_table(const ccq_rope_scaling* s, int rows, int dims, float* table, void* stream);
int launch_cache_append(const ccq_cache* c, const ccq_batch* b, const ccq_rope* rope, const ccq_heads* k, const ccq_heads* v, const ccq_heads* q,
                        const ccq_heads* q_out, int q_heads, void* stream);
int64_t attention_workspace(const ccq_cache* c, const ccq_batch* b, const ccq_attn* a);
int launch_attention(const ccq_cache* c, const ccq_batch* b, const ccq_attn* a, const ccq_heads* q, const ccq_heads* out, void* workspace, void* stream);
int64_t gemm8_workspace(const ccq_weight8* w, int M);
int64_t gemm8_bf16_workspace(const ccq_weight8* w, int M);
int launch_gemm8_bf16(const ccq_weight8* w, const void* x, int64_t ldx, int M, void* y, int64_t ldy, void* workspace, void* stream);
int launch_gemm8_as(const ccq_weight8* w, const ccq_rows8* x, int M, void* y, int64_t ldy, void* workspace, const int32_t* plan, void* stream);
int launch_gemm8(const ccq_weight8* w, const ccq_rows8* x, int M, void* y, int64_t ldy, void* workspace, void* stream);

}  // namespace ccq
