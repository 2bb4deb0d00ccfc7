// Root-mean-square norm with the residual's addition, and rows of 8-bit values with a power-of-two scale per block of 128
// columns.
//
//   h = x + residual,  y = h / sqrt(mean(h^2) + eps) * weight
//
// Bound by memory: every value is read once and written once, the row lies in registers in between.  A row has a wavefront,
// four, or sixteen, so that a thread holds at most 32 values of it: eight neighbouring columns at a time (16 bytes of bf16),
// so that 16 neighbouring lanes hold a scale's block and find its largest magnitude among themselves.
// 2048 rows of 7168 with a bf16 residual, 8 bits out: 18 - 20 us, 5.2 - 5.7 TB/s; one row of 8192: 2.9 us, the latency of a launch and two loads.
#include <type_traits>

#include "ccq_layer.h"

namespace ccq {

namespace {

struct NormArgs {
  const uint16_t* x;
  const void* residual;
  void* sum;
  const void* weight;
  uint16_t* y;
  uint8_t* codes;
  uint8_t* scales;
  int64_t ldx, ld_residual, ld_sum, ldy, ld_codes, ld_scales;
  int32_t M, N;
  float eps, inv_n;
  uint8_t residual_fp32, weight_fp32;
};

// Eight values of a row from column c on; those at N and past it are `past`.  One or two 16-byte pieces, which may start at any value: the card's memory
// accesses need no alignment (4096 rows of 8191, one value at a time: 120 us instead of 60).
__device__ __forceinline__ void load8(const void* row, int c, int N, bool fp32, float past, float (&v)[8]) {
  if (c + 8 <= N) {
    if (fp32) {
      f32x4_t a, b;
      __builtin_memcpy(&a, static_cast<const float*>(row) + c, 16);
      __builtin_memcpy(&b, static_cast<const float*>(row) + c + 4, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
      }
    } else {
      u32x4_t a;
      __builtin_memcpy(&a, static_cast<const uint16_t*>(row) + c, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(a[i]);
        v[2 * i + 1] = bf16_hi(a[i]);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = past;
    if (c + i < N) v[i] = fp32 ? static_cast<const float*>(row)[c + i] : bf16_lo(static_cast<const uint16_t*>(row)[c + i]);
  }
}

__device__ __forceinline__ void store8(void* row, int c, int N, bool fp32, const float (&v)[8]) {
  if (c + 8 <= N) {
    if (fp32) {
      const f32x4_t a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
      __builtin_memcpy(static_cast<float*>(row) + c, &a, 16);
      __builtin_memcpy(static_cast<float*>(row) + c + 4, &b, 16);
    } else {
      u32x4_t a;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
      __builtin_memcpy(static_cast<uint16_t*>(row) + c, &a, 16);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (c + i < N) {
      if (fp32) static_cast<float*>(row)[c + i] = v[i];
      else static_cast<uint16_t*>(row)[c + i] = to_bf16(v[i]);
    }
  }
}

template <typename T>
__device__ __forceinline__ const char* row_of(const T* p, int64_t ld, int64_t m, int bytes) {
  return reinterpret_cast<const char*>(p) + m * ld * bytes;
}

// The 16 lanes of a block of 128 columns call this together, lane l with columns c = 8 l .. of it; y holds zeros past N.
__device__ __forceinline__ void store_rows8(const NormArgs& a, int64_t m, int c, const float (&y)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, y[i]) & 0x7FFFFFFFu);
  top = max16(top);   // (as integers NaN is the largest)
  const bool bad = top >= kInfBits;
  const int byte = scale_byte(top, kRowsByteLo, kRowsByteHi);
  const float inv = inverse_of_byte(byte);
  u32x2_t q = {pack_e4m3(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), pack_e4m3(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
  if (bad) q = u32x2_t{0x7F7F7F7Fu, 0x7F7F7F7Fu};
  if (c >= a.N) return;
  uint8_t* out = a.codes + m * a.ld_codes + c;
  if (c + 8 <= a.N) {
    *reinterpret_cast<u32x2_t*>(out) = q;
  } else {
    for (int i = 0; i < a.N - c; ++i) out[i] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
  }
  if ((threadIdx.x & 15) == 0) a.scales[m * a.ld_scales + c / kScaleBlock] = (uint8_t)(bad ? 255 : byte);
}

// T threads to a row.  C > 0: the row is at most 8 T C long and is held in registers; C = 0: any length, h is formed again
// in a second pass over the row (a thread reads and writes the same columns in both, so outputs may lie on inputs).
template <int T, int C, bool NORM>
__global__ __launch_bounds__(T < 256 ? 256 : T) void ccq_norm_kernel(NormArgs a) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  const int t = T < 256 ? threadIdx.x % T : threadIdx.x;
  const int64_t m = (int64_t)blockIdx.x * kRows + (T < 256 ? threadIdx.x / T : 0);
  if (kRows > 1 && m >= a.M) return;   // (no barrier below where a workgroup has several rows)
  const char* x = row_of(a.x, a.ldx, m, 2);
  const char* res = row_of(static_cast<const char*>(a.residual), a.ld_residual, m, a.residual_fp32 ? 4 : 2);
  char* sum = const_cast<char*>(row_of(static_cast<const char*>(a.sum), a.ld_sum, m, a.residual_fp32 ? 4 : 2));
  char* y_row = const_cast<char*>(row_of(a.y, a.ldy, m, 2));

  auto load_h = [&](int c, float (&h)[8]) {
    load8(x, c, a.N, false, 0.f, h);
    if (NORM && a.residual) {
      float r[8];
      load8(res, c, a.N, a.residual_fp32, 0.f, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] += r[i];
    }
  };
  auto finish = [&](int c, const float (&h)[8], float inv) {
    float y[8];
    if (NORM) {
      if (a.sum && c < a.N) store8(sum, c, a.N, a.residual_fp32, h);
      float w[8];
      if (a.weight) {
        load8(a.weight, c, a.N, a.weight_fp32, 0.f, w);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = c + i < a.N ? 1.f : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = c + i < a.N ? h[i] * inv * w[i] : 0.f;
      if (a.y && c < a.N) store8(y_row, c, a.N, false, y);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = h[i];
    }
    if (a.codes) store_rows8(a, m, c, y);
  };
  auto inverse_rms = [&](float square) -> float {
    square = add16(square);
    square += xor16(square);
    square += xor32(square);
    if constexpr (T > 64) {
      __shared__ float parts[T / 64];
      if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = square;
      __syncthreads();
      square = 0.f;
#pragma unroll
      for (int i = 0; i < T / 64; ++i) square += parts[i];
    }
    return 1.f / sqrtf(square * a.inv_n + a.eps);
  };

  if constexpr (C > 0) {
    float h[C][8], square = 0.f;
#pragma unroll
    for (int j = 0; j < C; ++j) load_h(8 * (j * T + t), h[j]);
    float inv = 1.f;
    if constexpr (NORM) {
#pragma unroll
      for (int j = 0; j < C; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) square += h[j][i] * h[j][i];
      inv = inverse_rms(square);
    }
#pragma unroll
    for (int j = 0; j < C; ++j) finish(8 * (j * T + t), h[j], inv);
  } else {
    const int end = (a.N + 127) & ~127;   // whole blocks: the 16 lanes of one go together
    float inv = 1.f;
    if constexpr (NORM) {
      float square = 0.f;
      for (int c = 8 * t; c < end; c += 8 * T) {
        float h[8];
        load_h(c, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) square += h[i] * h[i];
      }
      inv = inverse_rms(square);
    }
    for (int c = 8 * t; c < end; c += 8 * T) {
      float h[8];
      load_h(c, h);
      finish(c, h, inv);
    }
  }
}

// The same from row `rows` on.
NormArgs past(NormArgs a, int rows) {
  auto skip = [&](auto*& p, int64_t ld, int bytes) {
    if (p) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>((uintptr_t)p + (uintptr_t)(rows * ld * bytes));
  };
  const int wide = a.residual_fp32 ? 4 : 2;
  skip(a.x, a.ldx, 2), skip(a.residual, a.ld_residual, wide), skip(a.sum, a.ld_sum, wide), skip(a.y, a.ldy, 2);
  skip(a.codes, a.ld_codes, 1), skip(a.scales, a.ld_scales, 1);
  a.M -= rows;
  return a;
}

template <int T, int C>
void launch(const NormArgs& all, bool norm, hipStream_t s) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  constexpr int kMost = (int)most_groups(T < 256 ? 256 : T) * kRows;   // rows of a launch
  NormArgs a = all;
  a.M = all.M < kMost ? all.M : kMost;
  const dim3 grid((unsigned)((a.M + kRows - 1) / kRows)), block(T < 256 ? 256 : T);
  if (norm) hipLaunchKernelGGL((ccq_norm_kernel<T, C, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((ccq_norm_kernel<T, (T * C > 2048 ? 0 : C), false>), grid, block, 0, s, a);   // (long rows: their pieces do not need each other, and with four held at once the compiler spills)
  if (all.M > kMost) launch<T, C>(past(all, kMost), norm, s);
}

}  // namespace

int launch_norm(const ccq_norm* n, bool norm, void* stream) {
  NormArgs a;
  a.x = static_cast<const uint16_t*>(n->x);
  a.residual = n->residual;
  a.sum = n->sum;
  a.weight = n->weight;
  a.y = static_cast<uint16_t*>(n->y);
  a.codes = static_cast<uint8_t*>(n->y8.codes);
  a.scales = n->y8.scales;
  a.ldx = n->ldx, a.ld_residual = n->ld_residual, a.ld_sum = n->ld_sum, a.ldy = n->ldy;
  a.ld_codes = n->y8.ld, a.ld_scales = n->y8.ld_scales;
  a.M = n->M, a.N = n->N;
  a.eps = n->eps, a.inv_n = (float)(1.0 / n->N);
  a.residual_fp32 = n->residual_type == CCQ_FP32, a.weight_fp32 = n->weight_type == CCQ_FP32;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int N = n->N;
  // Few rows leave the chip empty: as many threads to a row as it has pieces of eight columns.  Many: fewer threads, which hold more of it.  On the GPU, with a residual, us:
  //   rows x columns      1 x 512    1 x 1024   4096 x 1024   1 x 2048   512 x 2048   4096 x 2048 | 1 x 4096   1 x 8192   256 x 8192   1024 x 8192   4096 x 4096
  //   64 threads          2.3        3.0        6.2           4.2        5.2          11.0        |
  //   256                 2.4        2.5        7.6           2.5        3.4          12.0        | 2.9        4.3        5.6          10.6          21.2
  //   1024                2.7        2.8        20.6          2.8        4.5          21.3        | 2.8        3.0        4.4          13.0          23.7
  // (The lines lie where most sizes change sides; 512 to 1024 rows of 1024 to 2048 would be faster with 256 threads still.)
  const bool few = n->M < 512;
  if (N <= 512) launch<64, 1>(a, norm, s);
  else if (N <= 2048 && !few) N <= 1024 ? launch<64, 2>(a, norm, s) : launch<64, 4>(a, norm, s);
  else if (N <= 2048) launch<256, 1>(a, norm, s);
  else if (N <= 8192 && !few) N <= 4096 ? launch<256, 2>(a, norm, s) : launch<256, 4>(a, norm, s);
  else if (N <= 8192) launch<1024, 1>(a, norm, s);
  else if (N <= 16384) launch<1024, 2>(a, norm, s);
  else if (N <= 32768) launch<1024, 4>(a, norm, s);
  else launch<1024, 0>(a, norm, s);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
