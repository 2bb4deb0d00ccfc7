// 8-bit product for few rows: weights go from memory to registers once, activations come from the caches.
//
// A workgroup owns 16 outputs (of all rows of a tile of 16 MT rows); its wavefronts take the blocks of K in turn and their
// accumulators are added through LDS at the end, in a fixed order.  Bound by memory: the weights' bytes.
#include "ccq_gemm8.h"

namespace ccq {

namespace {

template <int MT, int W>
__global__ __launch_bounds__(64 * W) void ccq_gemm8_few_kernel(Gemm8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MT);
  __shared__ __align__(16) float parts[W * MT * 16 * 20];
  const uint8_t* w = a.w + (int64_t)min(n0 + r16, a.N - 1) * a.ldw;
  const float* ws = a.ws + (int64_t)(n0 / kScaleBlock) * a.ld_ws;
  const uint8_t* x[MT];
  const uint8_t* xs[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = min(m0 + 16 * i + r16, a.M - 1);
    x[i] = a.x + m * a.ldx;
    xs[i] = a.xs + m * a.ld_xs;
  }
  f32x4_t acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // 16 bytes from column k on, zeros past K
  auto piece = [&](const uint8_t* row, int k) {
    u32x4_t v = *reinterpret_cast<const u32x4_t*>(row + min(k, a.K - 16));
    if (k >= a.K) v = u32x4_t{0, 0, 0, 0};
    return v;
  };
#pragma unroll 4
  for (int kb = wave; kb < a.blocks; kb += W) {
    const int k = kb * kScaleBlock + 16 * g;
    const i32x8_t wv = operand8(piece(w, k), piece(w, k + 64));
    const float s = ws[kb];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const f32x4_t p = multiply8(wv, operand8(piece(x[i], k), piece(x[i], k + 64)), xs[i][kb]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][e] = fmaf(p[e], s, acc[i][e]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) *reinterpret_cast<f32x4_t*>(parts + ((wave * MT + i) * 16 + r16) * 20 + 4 * g) = acc[i];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * 16 * 16; i += 64 * W) {
    const int row = i >> 4, n = i & 15;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) sum += parts[(j * MT * 16 + row) * 20 + n];
    if (m0 + row < a.M && n0 + n < a.N) a.y[(int64_t)(m0 + row) * a.ldy + n0 + n] = to_bf16(sum);
  }
}

}  // namespace

int64_t gemm8_workspace(const ccq_weight8*, int) { return 0; }

int launch_gemm8(const ccq_weight8* w, const ccq_rows8* x, int M, void* y, int64_t ldy, void* workspace, void* stream) {
  Gemm8Args a;
  a.w = static_cast<const uint8_t*>(w->codes), a.ws = w->scales, a.ldw = w->ldw, a.ld_ws = w->ld_scales;
  a.x = static_cast<const uint8_t*>(x->codes), a.xs = x->scales, a.ldx = x->ld, a.ld_xs = x->ld_scales;
  a.y = static_cast<uint16_t*>(y), a.ldy = ldy, a.partial = static_cast<float*>(workspace);
  a.M = M, a.N = w->N, a.K = w->K, a.blocks = (w->K + kScaleBlock - 1) / kScaleBlock;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned nt = (unsigned)((a.N + 15) / 16);
  if (M <= 16) hipLaunchKernelGGL((ccq_gemm8_few_kernel<1, 4>), dim3(nt, 1), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((ccq_gemm8_few_kernel<4, 4>), dim3(nt, (unsigned)((M + 63) / 64)), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
