// The weighted sum of the experts' rows of a token:  y[t] = base[t] + sum over j of weights[t][j] rows[places[t][j]].
//
// Bound by memory: k rows are read and one written for each token.  A wavefront has 512 columns of one token, eight neighbouring ones a lane, so that
// its places are the same for all lanes; the rows of up to eight places are asked for before the first is added.
// 2048 tokens of 7168, eight places, a bf16 base: 57 us, 5.1 TB/s, what a large copy reaches on the card; one token 4.8 us with its call.
#include "ccq_routing.h"

namespace ccq {

namespace {

struct CombineArgs {
  const uint16_t* rows;
  const int32_t* places;
  const float* weights;
  const void* base;
  void* y;
  int64_t ld_rows, ld_places, ld_weights, ld_base, ldy;
  int64_t units;       // pieces of 512 columns of all tokens of the launch
  int32_t N, k, P, pieces;
  uint8_t base_fp32, y_fp32;
};

constexpr int kTogether = 8;   // rows asked for at once

// Eight values of a row from column c on, zeros past N.  16-byte pieces may start at any value.
__device__ __forceinline__ u32x4_t load8(const uint16_t* row, int c, int N) {
  u32x4_t v = {0, 0, 0, 0};
  if (c + 8 <= N) {
    __builtin_memcpy(&v, row + c, 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < N) v[i >> 1] |= (uint32_t)row[c + i] << (16 * (i & 1));
  }
  return v;
}

__global__ __launch_bounds__(256) void ccq_combine_kernel(CombineArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= a.units) return;
  const int64_t t = unit / a.pieces;
  const int c = (int)(unit - t * a.pieces) * 512 + 8 * (threadIdx.x & 63);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = 0.f;
  if (a.base) {
    if (a.base_fp32) {
      const float* row = static_cast<const float*>(a.base) + t * a.ld_base;
      if (c + 8 <= a.N) {
        __builtin_memcpy(y, row + c, 32);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < a.N) y[i] = row[c + i];
      }
    } else {
      const u32x4_t v = load8(static_cast<const uint16_t*>(a.base) + t * a.ld_base, c, a.N);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[2 * i] = bf16_lo(v[i]), y[2 * i + 1] = bf16_hi(v[i]);
    }
  }
  const int32_t* places = a.places + t * a.ld_places;
  const float* weights = a.weights + t * a.ld_weights;
  for (int j0 = 0; j0 < a.k; j0 += kTogether) {
    u32x4_t v[kTogether];
    float w[kTogether];
    bool there[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const bool in = j0 + j < a.k;
      const int p = in ? places[j0 + j] : -1;
      w[j] = in ? weights[j0 + j] : 0.f;
      there[j] = (uint32_t)p < (uint32_t)a.P;
      if (there[j]) v[j] = load8(a.rows + (int64_t)p * a.ld_rows, c, a.N);
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      if (!there[j]) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[2 * i] = __builtin_fmaf(w[j], bf16_lo(v[j][i]), y[2 * i]);
        y[2 * i + 1] = __builtin_fmaf(w[j], bf16_hi(v[j][i]), y[2 * i + 1]);
      }
    }
  }
  if (a.y_fp32) {
    float* row = static_cast<float*>(a.y) + t * a.ldy;
    if (c + 8 <= a.N) {
      __builtin_memcpy(row + c, y, 32);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.N) row[c + i] = y[i];
    }
  } else {
    uint16_t* row = static_cast<uint16_t*>(a.y) + t * a.ldy;
    if (c + 8 <= a.N) {
      u32x4_t v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
      __builtin_memcpy(row + c, &v, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.N) row[c + i] = to_bf16(y[i]);
    }
  }
}

}  // namespace

int launch_combine(const ccq_combination* c, void* stream) {
  CombineArgs a;
  a.ld_rows = c->ld_rows, a.ld_places = c->ld_places, a.ld_weights = c->ld_weights, a.ld_base = c->ld_base, a.ldy = c->ldy;
  a.N = c->N, a.k = c->k, a.P = c->P, a.pieces = (int32_t)(((int64_t)c->N + 511) / 512);
  a.base_fp32 = c->base_type == CCQ_FP32, a.y_fp32 = c->y_type == CCQ_FP32;
  const int64_t most = most_groups(256) * 4 / a.pieces;   // tokens of a launch
  for (int64_t t = 0; t < c->T; t += most) {
    const int64_t n = c->T - t < most ? c->T - t : most;
    a.rows = static_cast<const uint16_t*>(c->rows);
    a.places = c->places + t * c->ld_places, a.weights = c->weights + t * c->ld_weights;
    a.base = c->base ? static_cast<const char*>(c->base) + t * c->ld_base * (a.base_fp32 ? 4 : 2) : nullptr;
    a.y = static_cast<char*>(c->y) + t * c->ldy * (a.y_fp32 ? 4 : 2);
    a.units = n * a.pieces;
    hipLaunchKernelGGL(ccq_combine_kernel, dim3((unsigned)((a.units + 3) / 4)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
  }
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
