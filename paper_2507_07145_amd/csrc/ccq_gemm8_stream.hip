// 8-bit product for a few dozen rows: weights stream from memory to registers, activations pass LDS once for all the columns of a workgroup.
//
// A workgroup of eight wavefronts owns 16 MT rows x 128 outputs and a share of K: four wavefronts along the columns (32 each), two that take
// the even and the odd blocks of K of the share.  Two blocks are a step: the activations of a step (16 MT rows, 256 bytes each) are copied to
// LDS, asked for as far ahead as the weights (mixed with copies that pass by the registers the compiler's waits would be for all loads); every
// wavefront asks for its 4 KB of weights two or three steps ahead, straight into registers: no
// other wavefront of the workgroup needs them.  Bound by memory: the weights' bytes.  64 rows, 28672 x 8192: 57 us, 4.1 TB/s; 37 rows, 5001 x 7184, six
// shares: 12.4 - 13.8 us and 3 - 4 for the join (40 blocks of columns alone would leave most of the chip idle).
#include <type_traits>

#include "ccq_gemm8.h"

namespace ccq {

namespace {

constexpr int kCols = 128, kWaves = 8, kStepK = 2 * kScaleBlock;
constexpr int depth(int mt) { return mt <= 4 ? 4 : 3; }               // steps that are under way: what registers hold
constexpr int pieces(int mt) { return (mt * 16 * 16 + 511) / 512; }   // 16-byte pieces of a step's activations to a thread

struct Gemm8Stream {
  Gemm8Args a;
  int32_t n_tiles, shares, blocks_per_share;   // blocks_per_share even
};

// The largest over eight neighbouring lanes.
__device__ __forceinline__ uint32_t max8(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));    // quad_perm 1 0 3 2
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));    // quad_perm 2 3 0 1
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));   // the other way round in each half row
}

// WIDE: bf16 rows, quantized on their way to LDS.
template <int MT, bool WIDE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 4))) void ccq_gemm8_stream_kernel(Gemm8Stream p) {
  constexpr int kRows = 16 * MT, kDepth = depth(MT), kPieces = pieces(MT), kStage = kRows * kStepK;
  extern __shared__ __align__(256) uint8_t lds[];             // two steps of activations, row scales; at the end the sums of the odd blocks
  const Gemm8Args& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int wn = wave & 3, odd = wave >> 2;
  const int share = blockIdx.x / p.n_tiles, n0 = blockIdx.x % p.n_tiles * kCols + wn * 32, m0 = blockIdx.y * kRows;
  const int first = share * p.blocks_per_share, blocks = min(p.blocks_per_share, a.blocks - first), steps = (blocks + 1) / 2;
  const int rows = min(kRows, a.M - m0);

  // row scales of the share
  uint8_t* scales = lds + 2 * kStage;
  const int pitch = stream_pitch(p.blocks_per_share);
  for (int i = threadIdx.x; !WIDE && i < rows * blocks; i += 64 * kWaves) {
    const int r = i / blocks, c = i % blocks;
    scales[r * pitch + c] = a.xs[(int64_t)(m0 + r) * a.ld_xs + first + c];
  }

  // Piece q of the step's activations: row q / 16, chunk q % 16, at the chunk's place ^ row % 16 (the reads of 16 rows meet all banks).
  const uint8_t* x = WIDE ? nullptr : a.x + (int64_t)m0 * a.ldx;
  const uint16_t* x16 = WIDE ? a.x16 + (int64_t)m0 * a.ldx16 : nullptr;
  std::conditional_t<WIDE, Wide16, u32x4_t> xr[kDepth][kPieces];
  auto load_x = [&](int step, int at) {
    const int k0 = (first + 2 * step) * kScaleBlock;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int q = threadIdx.x + 512 * i, row = min(q >> 4, rows - 1), k = min(k0 + (q & 15) * 16, a.K - 16);
      if constexpr (WIDE) xr[at][i] = load_wide16(x16 + (int64_t)row * a.ldx16 + k, true);
      else xr[at][i] = *reinterpret_cast<const u32x4_t*>(x + (int64_t)row * a.ldx + k);
    }
  };
  auto store_x = [&](int step, int at) {
    const int k0 = (first + 2 * step) * kScaleBlock;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int q = threadIdx.x + 512 * i, row = q >> 4;
      const bool there = k0 + (q & 15) * 16 < a.K;
      u32x4_t v;
      if constexpr (WIDE) {
        const uint32_t top = max8(there ? magnitude16(xr[at][i]) : 0);   // of the block: eight threads side by side
        v = codes16(xr[at][i], top);
        if ((q & 7) == 0 && row < kRows) scales[row * pitch + 2 * step + (q >> 3 & 1)] = (uint8_t)scale_of(top);
      } else {
        v = xr[at][i];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = there ? v[e] : 0;   // zeros past K
      if (row < kRows) *reinterpret_cast<u32x4_t*>(lds + (step & 1) * kStage + row * kStepK + (((q & 15) ^ (row & 15)) * 16)) = v;
    }
  };
  const uint8_t* w_row[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) w_row[j] = a.w + (int64_t)min(n0 + 16 * j + r16, a.N - 1) * a.ldw;
  // (constant memory: scalar loads)
  const auto* ws = reinterpret_cast<const __attribute__((address_space(4))) float*>(reinterpret_cast<uintptr_t>(a.ws + (int64_t)(min(n0, a.N - 1) / kScaleBlock) * a.ld_ws));
  u32x4_t w[kDepth][2][2];
  float s[kDepth];
  auto load_w = [&](int step, int at) {
    const int b = first + 2 * step + odd, k = b * kScaleBlock + 16 * g;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) w[at][j][e] = *reinterpret_cast<const u32x4_t*>(w_row[j] + min(k + 64 * e, a.K - 16));
    s[at] = ws[min(b, a.blocks - 1)];
  };

  f32x4_t acc[MT][2];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int i = 0; i < kDepth - 1; ++i) {
    load_x(i, i);
    load_w(i, i);
  }
  store_x(0, 0);
  // One straight line of instructions, left in the middle: the compiler then knows how many loads are under way at each wait.
  for (int step0 = 0;; step0 += kDepth) {
#pragma unroll
    for (int at = 0; at < kDepth; ++at) {
      const int step = step0 + at;
      if (step >= steps) goto done;
      lds_barrier();
      load_x(step + kDepth - 1, (at + kDepth - 1) % kDepth);
      load_w(step + kDepth - 1, (at + kDepth - 1) % kDepth);
      const int b = 2 * step + odd, k = (first + b) * kScaleBlock + 16 * g;
      i32x8_t weights[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        u32x4_t lo = w[at][j][0], hi = w[at][j][1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // zeros past K and past the share
          lo[e] = k < a.K && b < blocks ? lo[e] : 0;
          hi[e] = k + 64 < a.K && b < blocks ? hi[e] : 0;
        }
        weights[j] = operand8(lo, hi);
      }
      const uint8_t* stage = lds + (step & 1) * kStage;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const uint8_t* row = stage + (16 * i + r16) * kStepK;
        const int c = 8 * odd + g;
        const i32x8_t act = operand8(*reinterpret_cast<const u32x4_t*>(row + ((c ^ r16) * 16)), *reinterpret_cast<const u32x4_t*>(row + (((c + 4) ^ r16) * 16)));
        const int scale = scales[min(16 * i + r16, rows - 1) * pitch + min(b, blocks - 1)];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x4_t r = multiply8(weights[j], act, scale);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(r[e], s[at], acc[i][j][e]);
        }
      }
      store_x(step + 1, (at + 1) % kDepth);
    }
  }
done:

  // the odd blocks' sums join the even blocks'
  lds_barrier();
  float* sums = reinterpret_cast<float*>(lds);
  constexpr int kPitch = 36;   // floats between rows of 32 columns
  if (odd) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) *reinterpret_cast<f32x4_t*>(sums + (wn * kRows + 16 * i + r16) * kPitch + 16 * j + 4 * g) = acc[i][j];
  }
  __syncthreads();
  if (odd) return;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + 16 * i + r16;
    if (m >= a.M) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x4_t v = acc[i][j] + *reinterpret_cast<const f32x4_t*>(sums + (wn * kRows + 16 * i + r16) * kPitch + 16 * j + 4 * g);
      const int n = n0 + 16 * j + 4 * g;
      if (p.shares > 1) {
        float* out = a.partial + ((int64_t)share * a.M + m) * a.ld_partial + n;
        if (n < a.ld_partial) *reinterpret_cast<f32x4_t*>(out) = v;
      } else if (n + 4 <= a.N) {
        *reinterpret_cast<u32x2_t*>(a.y + (int64_t)m * a.ldy + n) = u32x2_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
      } else {
        for (int e = 0; e < a.N - n; ++e) a.y[(int64_t)m * a.ldy + n + e] = to_bf16(v[e]);
      }
    }
  }
}

// y = sum of the shares, in their order
__global__ __launch_bounds__(256) void ccq_gemm8_add_kernel(Gemm8Args a, int shares) {
  const int64_t quads = a.ld_partial / 4, at = (int64_t)blockIdx.x * 256 + threadIdx.x, m = at / quads;
  if (m >= a.M) return;
  const int n = (int)(at % quads) * 4;
  const float* from = a.partial + m * a.ld_partial + n;
  f32x4_t sum = *reinterpret_cast<const f32x4_t*>(from);
  for (int s = 1; s < shares; ++s) sum += *reinterpret_cast<const f32x4_t*>(from + s * a.M * a.ld_partial);
  uint16_t* out = a.y + m * a.ldy + n;
  if (n + 4 <= a.N) {
    *reinterpret_cast<u32x2_t*>(out) = u32x2_t{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
  } else {
    for (int e = 0; e < a.N - n; ++e) out[e] = to_bf16(sum[e]);
  }
}

template <int MT>
int launch(const Gemm8Stream& p, hipStream_t s) {
  constexpr int kRows = 16 * MT;
  const int64_t bytes = stream_lds(MT, p.blocks_per_share);
  if (bytes > kMostLds) return CCQ_ERR_UNSUPPORTED;
  constexpr bool kWide = MT <= 4;   // (of 96 bf16 rows the registers do not hold three steps)
  if (p.a.x16 && !kWide) return CCQ_ERR_UNSUPPORTED;
  const void* kernel = p.a.x16 ? reinterpret_cast<const void*>(ccq_gemm8_stream_kernel<MT, kWide>) : reinterpret_cast<const void*>(ccq_gemm8_stream_kernel<MT, false>);
  if (bytes > 64 * 1024 && hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) return CCQ_ERR_HIP;
  const dim3 grid((unsigned)(p.n_tiles * p.shares), (unsigned)((p.a.M + kRows - 1) / kRows));
  if (p.a.x16) hipLaunchKernelGGL((ccq_gemm8_stream_kernel<MT, kWide>), grid, dim3(64 * kWaves), (unsigned)bytes, s, p);
  else hipLaunchKernelGGL((ccq_gemm8_stream_kernel<MT, false>), grid, dim3(64 * kWaves), (unsigned)bytes, s, p);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace

int launch_gemm8_add(const Gemm8Args& a, int shares, void* stream) {
  const int64_t threads = a.M * (a.ld_partial / 4);
  hipLaunchKernelGGL(ccq_gemm8_add_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, static_cast<hipStream_t>(stream), a, shares);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

int launch_gemm8_stream(const Gemm8Args& a, int mt, int shares, void* stream) {
  Gemm8Stream p;
  p.a = a;
  p.n_tiles = (a.N + kCols - 1) / kCols;
  p.blocks_per_share = stream_blocks(a.blocks, shares);
  p.shares = (a.blocks + p.blocks_per_share - 1) / p.blocks_per_share;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rc = mt == 1 ? launch<1>(p, s) : mt == 2 ? launch<2>(p, s) : mt == 3 ? launch<3>(p, s) : mt == 4 ? launch<4>(p, s) : launch<6>(p, s);
  return rc != CCQ_OK || p.shares == 1 ? rc : launch_gemm8_add(a, p.shares, stream);
}

}  // namespace ccq
