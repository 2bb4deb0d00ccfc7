// Low-rank adapters of a batch's requests:  out[t] = y[t] + scale (x[t] A^T) B^T, A [rank][K] and B [N][rank] those of t's adapter.
//
// Two kernels of MFMA 16x16x32 bf16.  Rows come sorted by adapter; a workgroup takes a block of 16 TT of them and the runs of one adapter in it, one
// after the other or, where many are to be expected, one each.  The first forms v = x A^T: its wavefronts and, where there are few blocks, several workgroups share K; the wavefronts'
// sums are added through LDS, the workgroups' are left to the second kernel.  The second adds them up, multiplies by the scale and forms y + v B^T.
// v is a sum of thousands of products and would lose in bf16 what the result's own rounding keeps: it enters the second product as
// two bf16 numbers (within 2^-15 of it), which costs a second matrix instruction on operands that are there.
// Bound by memory: A and B of the adapters in use where rows are few, x, y and out where they are many.
#include "ccq_routing.h"

namespace ccq {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

struct AdapterArgs {
  const uint16_t *a, *b, *x, *y;
  uint16_t* out;
  const float* scales;
  const int32_t *ranks, *rows, *experts;
  float* v;               // [splits][T][padded rank]
  int64_t ldx, ldy, ld_out, block0;
  int32_t T, K, N, rank, count, padded;
  int32_t together;       // runs of a block that have a workgroup of their own at the same time
  int32_t splits, steps;  // workgroups along K, steps of 32 columns of each
  int32_t chunks;         // of ranks (first kernel), of columns (second)
  int32_t columns;        // of a workgroup of the second kernel
  uint8_t copies;         // out is not y
};

__device__ __forceinline__ f32x4_t mfma(const u32x4_t& a, const u32x4_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// The runs of one adapter in a block of sorted rows.
struct Runs {
  uint64_t starts;
  int adapter;   // lane i: of row i of the block, -1: none
  int rows;      // rows of the block that there are
  __device__ __forceinline__ Runs(const AdapterArgs& a, int64_t p0, int most) {
    const int lane = threadIdx.x & 63;
    rows = (int)min((int64_t)most, (int64_t)a.T - p0);
    adapter = lane < rows ? a.experts[p0 + lane] : -1;
    if ((uint32_t)adapter >= (uint32_t)a.count) adapter = -1;
    const int before = __shfl_up(adapter, 1);
    starts = __ballot(lane < rows && (lane == 0 || adapter != before));
  }
  __device__ __forceinline__ void skip(int n) {
    for (; n > 0 && starts; --n) starts &= starts - 1;
  }
  __device__ __forceinline__ int first() const { return __builtin_ctzll(starts); }
  __device__ __forceinline__ int end() const {
    const uint64_t later = starts & (starts - 1);
    return later ? __builtin_ctzll(later) : rows;
  }
};

__device__ __forceinline__ int rank_of(const AdapterArgs& a, int i) { return a.ranks ? min(max(a.ranks[i], 0), a.rank) : a.rank; }

constexpr int kDownWaves = 8, kAhead = 4;

template <int RT, int TT>
__global__ __launch_bounds__(64 * kDownWaves) void ccq_adapter_down_kernel(AdapterArgs a) {
  __shared__ __align__(16) f32x4_t sums[kDownWaves][RT * TT][64];
  uint32_t g = blockIdx.x;
  const int split = g % a.splits;
  g /= a.splits;
  const int r0 = (int)(g % a.chunks) * 16 * RT;
  g /= a.chunks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, quarter = lane >> 4;
  const int64_t p0 = (a.block0 + g / a.together) * 16 * TT;
  Runs runs(a, p0, 16 * TT);
  runs.skip((int)(g % a.together));
  if (!runs.starts) return;
  const uint16_t* xr[TT];
#pragma unroll
  for (int u = 0; u < TT; ++u) {
    const int64_t p = p0 + 16 * u + i16;
    const int t = p < a.T ? a.rows[p] : 0;
    xr[u] = a.x + ((uint32_t)t < (uint32_t)a.T ? t : 0) * a.ldx + 8 * quarter;   // (rows that are none: their columns of the product are not stored)
  }
  const int all = (a.K + 31) / 32;
  const int step0 = min(split * a.steps, all), step1 = min(step0 + a.steps, all);
  const int per = (step1 - step0 + kDownWaves - 1) / kDownWaves;
  const int from = min(step0 + wave * per, step1), to = min(from + per, step1);
  for (; runs.starts; runs.skip(a.together)) {
    const int first = runs.first(), end = runs.end();
    const int i = __builtin_amdgcn_readfirstlane(__shfl(runs.adapter, first));
    if (i < 0) continue;
    const int rank = rank_of(a, i);
    if (r0 >= rank) continue;
    const uint16_t* ar[RT];
#pragma unroll
    for (int u = 0; u < RT; ++u) ar[u] = a.a + ((int64_t)i * a.rank + min(r0 + 16 * u + i16, rank - 1)) * a.K + 8 * quarter;   // (past the rank its last row again)
    f32x4_t acc[RT][TT];
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int w = 0; w < TT; ++w) acc[u][w] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int whole = min(to, a.K / 32);
    int step = from;
    auto steps = [&](auto n) {
      constexpr int kSteps = decltype(n)::value;
      u32x4_t xa[kSteps][TT], aa[kSteps][RT];
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
#pragma unroll
        for (int w = 0; w < TT; ++w) __builtin_memcpy(&xa[s][w], xr[w] + (int64_t)(step + s) * 32, 16);
#pragma unroll
        for (int u = 0; u < RT; ++u) aa[s][u] = *reinterpret_cast<const u32x4_t*>(ar[u] + (int64_t)(step + s) * 32);
      }
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int u = 0; u < RT; ++u)
#pragma unroll
          for (int w = 0; w < TT; ++w) acc[u][w] = mfma(aa[s][u], xa[s][w], acc[u][w]);
      step += kSteps;
    };
    while (step + kAhead <= whole) steps(std::integral_constant<int, kAhead>());
    while (step < whole) steps(std::integral_constant<int, 1>());
    if (step < to) {   // the last columns: K is a multiple of 8
      const bool in = step * 32 + 8 * quarter < a.K;
      u32x4_t xa[TT];
#pragma unroll
      for (int w = 0; w < TT; ++w) {
        xa[w] = u32x4_t{0, 0, 0, 0};
        if (in) __builtin_memcpy(&xa[w], xr[w] + (int64_t)step * 32, 16);
      }
#pragma unroll
      for (int u = 0; u < RT; ++u) {
        u32x4_t aa = {0, 0, 0, 0};
        if (in) aa = *reinterpret_cast<const u32x4_t*>(ar[u] + (int64_t)step * 32);
#pragma unroll
        for (int w = 0; w < TT; ++w) acc[u][w] = mfma(aa, xa[w], acc[u][w]);
      }
    }
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int w = 0; w < TT; ++w) sums[wave][u * TT + w][lane] = acc[u][w];
    __syncthreads();
    for (int c = wave; c < RT * TT; c += kDownWaves) {
      f32x4_t sum = sums[0][c][lane];
#pragma unroll
      for (int w = 1; w < kDownWaves; ++w) sum += sums[w][c][lane];
      const int u = c / TT, row = 16 * (c % TT) + i16, r = r0 + 16 * u + 4 * quarter;
      if (row >= first && row < end && r < a.padded) *reinterpret_cast<f32x4_t*>(a.v + ((int64_t)split * a.T + p0 + row) * a.padded + r) = sum;
    }
    __syncthreads();
  }
}

// KK: steps of 32 ranks.
template <int KK, int TT>
__global__ __launch_bounds__(256) void ccq_adapter_up_kernel(AdapterArgs a) {
  __shared__ __align__(16) u32x4_t parts[2][TT * KK][64];   // v as matrix operands: its upper and its lower bits
  uint32_t g = blockIdx.x;
  const int64_t n_first = (int64_t)(g % a.chunks) * a.columns;
  g /= a.chunks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, quarter = lane >> 4;
  const int64_t p0 = (a.block0 + g / a.together) * 16 * TT;
  Runs runs(a, p0, 16 * TT);
  runs.skip((int)(g % a.together));
  if (!runs.starts) return;
  int64_t t[TT];
#pragma unroll
  for (int w = 0; w < TT; ++w) {
    const int64_t p = p0 + 16 * w + i16;
    const int row = p < a.T ? a.rows[p] : -1;
    t[w] = (uint32_t)row < (uint32_t)a.T ? row : -1;
  }
  const int n_end = (int)min(n_first + a.columns, (int64_t)a.N);
  for (; runs.starts; runs.skip(a.together)) {
    const int first = runs.first(), end = runs.end();
    const int i = __builtin_amdgcn_readfirstlane(__shfl(runs.adapter, first));
    const int rank = i < 0 ? 0 : rank_of(a, i);
    if (rank == 0 && !a.copies) continue;
    const int last = (rank - 1) >> 5;   // (arithmetic: -1 without ranks)
    if (rank > 0) {
      const float scale = a.scales ? a.scales[i] : 1.f;
      for (int c = wave; c < TT * KK; c += 4) {
        const int row = 16 * (c / KK) + i16, r = 32 * (c % KK) + 8 * quarter;
        f32x4_t v0 = {0.f, 0.f, 0.f, 0.f}, v1 = v0;
        if (row >= first && row < end && r < rank) {
          const float* from = a.v + (p0 + row) * a.padded + r;
          for (int s = 0; s < a.splits; ++s, from += (int64_t)a.T * a.padded) {
            v0 += *reinterpret_cast<const f32x4_t*>(from);
            v1 += *reinterpret_cast<const f32x4_t*>(from + 4);
          }
        }
        u32x4_t hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t h = 0, l = 0;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int at = 2 * j + half;
            float v = (at < 4 ? v0[at & 3] : v1[at & 3]) * scale;
            if (r + at >= rank) v = 0.f;
            const uint32_t top = __builtin_bit_cast(uint32_t, v) & 0xFFFF0000u;
            const float top_v = __builtin_bit_cast(float, top), rest = top_v == v ? 0.f : v - top_v;   // (infinity less infinity would be NaN)
            h |= half ? top : top >> 16;
            l |= (uint32_t)to_bf16(rest) << (16 * half);
          }
          hi[j] = h, lo[j] = l;
        }
        parts[0][c][lane] = hi;
        parts[1][c][lane] = lo;
      }
    }
    __syncthreads();
    u32x4_t v[2][TT][KK];
#pragma unroll
    for (int w = 0; w < TT; ++w)
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        v[0][w][k] = parts[0][w * KK + k][lane];
        v[1][w][k] = parts[1][w * KK + k][lane];
      }
    u32x4_t mask;   // of the last step: ranks in use
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 32 * last + 8 * quarter + 2 * j;
      mask[j] = (r < rank ? 0xFFFFu : 0u) | (r + 1 < rank ? 0xFFFF0000u : 0u);
    }
    for (int n0 = (int)n_first + 64 * wave; n0 < n_end; n0 += 256) {
      f32x4_t acc[TT][4];
#pragma unroll
      for (int w = 0; w < TT; ++w)
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[w][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      const uint16_t* br[4];   // lane's rows of B: 16 (i / 4) + 4 u + i % 4, so that a lane has 16 neighbouring columns of the result
#pragma unroll
      for (int u = 0; u < 4; ++u) br[u] = a.b + ((int64_t)max(i, 0) * a.N + min(n0 + 16 * (i16 >> 2) + 4 * u + (i16 & 3), a.N - 1)) * a.rank + 8 * quarter;
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        if (k > last) break;
        u32x4_t bb[4];
        const bool in = 32 * k + 8 * quarter < a.rank;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          bb[u] = u32x4_t{0, 0, 0, 0};
          if (in) bb[u] = *reinterpret_cast<const u32x4_t*>(br[u] + 32 * k);
          if (k == last) bb[u] &= mask;
        }
#pragma unroll
        for (int w = 0; w < TT; ++w)
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            acc[w][u] = mfma(bb[u], v[1][w][k], acc[w][u]);
            acc[w][u] = mfma(bb[u], v[0][w][k], acc[w][u]);
          }
      }
      const int n = n0 + 16 * quarter;
#pragma unroll
      for (int w = 0; w < TT; ++w) {
        const int row = 16 * w + i16;
        if (row < first || row >= end || t[w] < 0 || n >= a.N) continue;
        const uint16_t* yr = a.y + t[w] * a.ldy + n;
        uint16_t* o = a.out + t[w] * a.ld_out + n;
        if (n + 16 <= a.N) {
          u32x4_t y[2];
          __builtin_memcpy(y, yr, 32);
          if (rank > 0) {
#pragma unroll
            for (int h = 0; h < 8; ++h)
              y[h >> 2][h & 3] = pack_bf16(bf16_lo(y[h >> 2][h & 3]) + acc[w][h >> 1][2 * (h & 1)], bf16_hi(y[h >> 2][h & 3]) + acc[w][h >> 1][2 * (h & 1) + 1]);
          }
          __builtin_memcpy(o, y, 32);
        } else {
#pragma unroll
          for (int h = 0; h < 16; ++h)
            if (n + h < a.N) o[h] = rank > 0 ? to_bf16(bf16_lo(yr[h]) + acc[w][h >> 2][h & 3]) : yr[h];
        }
      }
    }
    __syncthreads();
  }
}

// How the rows and K of a call are cut.
struct Plan {
  int tiles;       // of 16 rows in a block
  int64_t blocks;
  int together, splits, steps, rank_tiles, chunks, padded;
  int columns, column_chunks;
};

Plan plan_of(const ccq_adapter_set* s, int T) {
  Plan p;
  p.tiles = T > 256 && s->rank <= 64 ? 2 : 1;
  const int rows = 16 * p.tiles;
  p.blocks = ((int64_t)T + rows - 1) / rows;
  // every adapter that begins inside a block makes one more run
  const int64_t begins = s->count < T ? s->count : T;
  const int64_t runs = 1 + (begins + p.blocks - 1) / p.blocks;
  p.together = (int)(runs < rows ? runs : rows);
  if (p.together > T) p.together = T;
  p.padded = (s->rank + 15) / 16 * 16;
  p.rank_tiles = p.padded >= 64 ? 4 : p.padded >= 32 ? 2 : 1;
  p.chunks = (p.padded + 16 * p.rank_tiles - 1) / (16 * p.rank_tiles);
  const int steps = (s->K + 31) / 32;
  const int64_t busy = p.blocks + begins < p.blocks * p.together ? p.blocks + begins : p.blocks * p.together;   // workgroups with work
  int64_t splits = 512 / (busy * p.chunks);
  const int most = steps / (2 * kDownWaves);   // two steps a wavefront at least
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  if (splits > 32) splits = 32;
  p.steps = (int)((steps + splits - 1) / splits);
  p.splits = (steps + p.steps - 1) / p.steps;
  int64_t column_chunks = (2048 + busy - 1) / busy;
  const int64_t pieces = ((int64_t)s->N + 255) / 256;
  if (column_chunks > pieces) column_chunks = pieces;
  p.columns = (int)((pieces + column_chunks - 1) / column_chunks * 256);
  p.column_chunks = (int)(((int64_t)s->N + p.columns - 1) / p.columns);
  return p;
}

template <int RT, int TT>
void down(const AdapterArgs& a, unsigned groups, hipStream_t s) {
  hipLaunchKernelGGL((ccq_adapter_down_kernel<RT, TT>), dim3(groups), dim3(64 * kDownWaves), 0, s, a);
}
template <int KK, int TT>
void up(const AdapterArgs& a, unsigned groups, hipStream_t s) {
  hipLaunchKernelGGL((ccq_adapter_up_kernel<KK, TT>), dim3(groups), dim3(256), 0, s, a);
}

}  // namespace

int64_t adapters_workspace(const ccq_adapter_set* set, int T) {
  if (T == 0) return 0;
  const Plan p = plan_of(set, T);
  return (int64_t)p.splits * T * p.padded * 4;
}

int launch_adapters(const ccq_adapter_set* set, int T, const int32_t* rows, const int32_t* experts, const void* x, int64_t ldx, const void* y, int64_t ldy, void* out,
                    int64_t ld_out, void* workspace, void* stream) {
  const Plan p = plan_of(set, T);
  AdapterArgs a;
  a.a = static_cast<const uint16_t*>(set->a), a.b = static_cast<const uint16_t*>(set->b);
  a.x = static_cast<const uint16_t*>(x), a.y = static_cast<const uint16_t*>(y), a.out = static_cast<uint16_t*>(out);
  a.scales = set->scales, a.ranks = set->ranks, a.rows = rows, a.experts = experts;
  a.v = static_cast<float*>(workspace);
  a.ldx = ldx, a.ldy = ldy, a.ld_out = ld_out;
  a.T = T, a.K = set->K, a.N = set->N, a.rank = set->rank, a.count = set->count, a.padded = p.padded;
  a.together = p.together, a.splits = p.splits, a.steps = p.steps, a.columns = p.columns;
  a.copies = out != y;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool two = p.tiles == 2;
  auto parts = [&](int64_t per_block, int threads, auto launch) {   // blocks at a time that a launch has room for
    const int64_t most = most_groups(threads) / per_block;
    for (int64_t b = 0; b < p.blocks; b += most) {
      a.block0 = b;
      launch((unsigned)((p.blocks - b < most ? p.blocks - b : most) * per_block));
    }
  };
  a.chunks = p.chunks;
  parts((int64_t)p.together * p.chunks * p.splits, 64 * kDownWaves, [&](unsigned n) {
    if (p.rank_tiles == 1) two ? down<1, 2>(a, n, s) : down<1, 1>(a, n, s);
    else if (p.rank_tiles == 2) two ? down<2, 2>(a, n, s) : down<2, 1>(a, n, s);
    else two ? down<4, 2>(a, n, s) : down<4, 1>(a, n, s);
  });
  a.chunks = p.column_chunks;
  parts((int64_t)p.together * p.column_chunks, 256, [&](unsigned n) {
    if (p.padded <= 32) two ? up<1, 2>(a, n, s) : up<1, 1>(a, n, s);
    else if (p.padded <= 64) two ? up<2, 2>(a, n, s) : up<2, 1>(a, n, s);
    else if (p.padded <= 128) up<4, 1>(a, n, s);
    else up<8, 1>(a, n, s);
  });
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
