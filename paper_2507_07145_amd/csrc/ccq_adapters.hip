// Low-rank adapters of a batch's requests:  out[t] = y[t] + scale (x[t] A^T) B^T, A [rank][K] and B [N][rank] those of t's adapter.
//
// The first product, v = x A^T, is one kernel (MFMA 16x16x32 bf16): rows come sorted by adapter, and a workgroup takes a block of 16 or 32 of them with one run of one adapter in it and a
// share of K; the shares' sums are left to the second product.  That has three forms:
//   runs of few rows (rank x rows up to 8192, no more than four rows an adapter): B is read along its memory and multiplied by v in fp32, no matrix instruction.
//     One row of 8192 to 8192, rank 16: 3.8 + 4.6 us; 37 rows, 7184 to 5001, rank 24, 12 adapters: 5.0 + 6.0; 128 rows of 96 adapters, 4096 to 11008, rank 32: 7.5 + 15.8, of
//     which B's 51 MB alone take 10.
//   up to 511 rows, or rows x N up to 2^22: MFMA, B and the products through LDS (256 rows, 4096 to 4096, rank 16, four adapters: 4.3 + 7.2 us; to 18432 4.3 + 12.4).
//   more: v is joined by a kernel of its own, B stays in registers (2048 rows, 7168 to 18432, rank 64, four adapters: 13 + 5 + 35 us; 4.3 TB/s of y and out).
// v is a sum of thousands of products and would lose in bf16 what the result's own rounding keeps: it enters matrix instructions as two bf16 numbers (within 2^-15 of it), which costs a
// second one on operands that are there.
// Bound by memory: A and B of the adapters in use where rows are few, x, y and out where they are many; short calls by a chain of four or five dependent loads in each kernel.
#include "ccq_routing.h"

namespace ccq {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef u32x4_t __attribute__((aligned(2))) u32x4_any_t;   // rows may start at any element

struct AdapterArgs {
  const uint16_t *a, *b, *x, *y;
  uint16_t* out;
  const float* scales;
  const int32_t *ranks, *rows, *experts;
  float* v;               // [splits][T][padded rank]
  int64_t ldx, ldy, ld_out, block0;
  uint32_t blocks;        // of the launch
  u32x4_t* parts;         // v as matrix operands, where there are many rows
  int64_t blocks_each;    // pieces of 32 rows and 128 columns of a workgroup then
  int32_t T, K, N, rank, count, padded;
  int32_t together;       // runs of a block that have a workgroup of their own at the same time
  int32_t splits, steps;  // workgroups along K, stages of 128 columns of each
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
  // the adapter of this lane's row, which the constructor is given
  static __device__ __forceinline__ int of_lane(const AdapterArgs& a, int64_t p0, int most) {
    const int lane = threadIdx.x & 63;
    return lane < most && p0 + lane < a.T ? a.experts[p0 + lane] : -1;
  }
  __device__ __forceinline__ Runs(const AdapterArgs& a, int64_t p0, int most) : Runs(a, p0, most, of_lane(a, p0, most)) {}
  __device__ __forceinline__ Runs(const AdapterArgs& a, int64_t p0, int most, int of_this_lane) : adapter(of_this_lane) {
    const int lane = threadIdx.x & 63;
    rows = (int)min((int64_t)most, (int64_t)a.T - p0);
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

// Rows of 128 columns in LDS: 16 pieces of 16 bytes, piece c of row r in place c ^ (r & 15), so that eight rows' reads of one piece meet all banks.
constexpr int kStageColumns = 128, kStageRow = 256;
__device__ __forceinline__ uint32_t staged(int row, int piece) { return (uint32_t)(row * kStageRow + ((piece ^ (row & 15)) * 16)); }

// Both operands go through LDS in stages of 128 columns: a matrix operand read from memory directly has its lanes 16 rows apart, a cache line each, which
// the card's address units take at a quarter of their rate.  Threads hold two stages more, or four, in registers; wavefront w multiplies columns 32 w .. of each
// stage, the wavefronts' sums are added at the end.
template <int RT, int TT>
__global__ __launch_bounds__(256, RT == 8 ? 2 : 3) void ccq_adapter_down_kernel(AdapterArgs a) {
  extern __shared__ __align__(256) uint8_t lds[];
  constexpr int kStage = (RT + TT) * 16 * kStageRow;
  uint32_t g = blockIdx.x;
  const int split = g % a.splits;
  g /= a.splits;
  const int r0 = (int)(g % a.chunks) * 16 * RT;
  g /= a.chunks;
  const uint32_t later = g / a.blocks, turn = a.together - 1 - later;   // (the runs that few blocks have first: begun last, they would run alone)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, quarter = lane >> 4;
  const int64_t p0 = (a.block0 + (g - later * a.blocks)) * 16 * TT;
  Runs runs(a, p0, 16 * TT);
  runs.skip((int)turn);
  if (!runs.starts) return;
  const int my_row = threadIdx.x >> 4, piece = threadIdx.x & 15;   // rows my_row + 16 j of the stage
  const uint16_t* xr[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) {
    const int64_t p = p0 + 16 * j + my_row;
    const int t = p < a.T ? a.rows[p] : -1;
    xr[j] = (uint32_t)t < (uint32_t)a.T ? a.x + t * a.ldx + 8 * piece : nullptr;
  }
  const int all = (a.K + kStageColumns - 1) / kStageColumns;
  const int from = min(split * a.steps, all), to = min(from + a.steps, all);
  const uint32_t write_at = staged(my_row, piece), read_at = staged(i16, 4 * wave + quarter);
  for (; runs.starts; runs.skip(a.together)) {
    const int first = runs.first(), end = runs.end();
    const int i = __builtin_amdgcn_readfirstlane(__shfl(runs.adapter, first));
    if (i < 0) continue;
    const int rank = rank_of(a, i);
    if (r0 >= rank) continue;
    const uint16_t* const ar = a.a + ((int64_t)i * a.rank + r0 + my_row) * a.K + 8 * piece;
    // (rows of other runs and ranks not in use are not read: what LDS holds for them reaches no sum that is kept)
    auto load = [&](int step, u32x4_t (&x)[TT], u32x4_t (&w)[RT]) {
      const int k = step * kStageColumns;
      const bool in = k + 8 * piece < a.K;
#pragma unroll
      for (int j = 0; j < TT; ++j) {
        x[j] = u32x4_t{0, 0, 0, 0};
        const int row = 16 * j + my_row;
        if (in && row >= first && row < end && xr[j]) __builtin_memcpy(&x[j], xr[j] + k, 16);
      }
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        w[j] = u32x4_t{0, 0, 0, 0};
        if (in && r0 + 16 * j + my_row < rank) w[j] = *reinterpret_cast<const u32x4_t*>(ar + (int64_t)16 * j * a.K + k);
      }
    };
    f32x4_t acc[RT][TT];
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int w = 0; w < TT; ++w) acc[u][w] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    constexpr int kDepth = RT * TT <= 2 ? 4 : 2;   // stages asked for ahead: three workgroups on a CU are worth more (2048 x 7168, rank 64: 12.6 us, with four stages and two of them 16.6)
    u32x4_t x[kDepth][TT], w[kDepth][RT];
    auto stage = [&](int s, int d) {
      uint8_t* const to_lds = lds + ((s - from) & 1) * kStage;
#pragma unroll
      for (int j = 0; j < TT; ++j) *reinterpret_cast<u32x4_t*>(to_lds + write_at + j * 16 * kStageRow) = x[d][j];
#pragma unroll
      for (int j = 0; j < RT; ++j) *reinterpret_cast<u32x4_t*>(to_lds + write_at + (TT + j) * 16 * kStageRow) = w[d][j];
      if (s + kDepth < to) load(s + kDepth, x[d], w[d]);
      __syncthreads();
      u32x4_t xa[TT];
#pragma unroll
      for (int j = 0; j < TT; ++j) xa[j] = *reinterpret_cast<const u32x4_t*>(to_lds + read_at + j * 16 * kStageRow);
#pragma unroll
      for (int u = 0; u < RT; ++u) {
        const u32x4_t wa = *reinterpret_cast<const u32x4_t*>(to_lds + read_at + (TT + u) * 16 * kStageRow);
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[u][j] = mfma(wa, xa[j], acc[u][j]);
      }
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
      if (from + d < to) load(from + d, x[d], w[d]);
    for (int s = from; s < to; s += kDepth) {
#pragma unroll
      for (int d = 0; d < kDepth; ++d)
        if (s + d < to) stage(s + d, d);
    }
    __syncthreads();
    f32x4_t* const sums = reinterpret_cast<f32x4_t*>(lds);   // [4][RT TT][64]
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int w = 0; w < TT; ++w) sums[(wave * RT * TT + u * TT + w) * 64 + lane] = acc[u][w];
    __syncthreads();
    for (int c = wave; c < RT * TT; c += 4) {
      f32x4_t sum = sums[c * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) sum += sums[(w * RT * TT + c) * 64 + lane];
      const int u = c / TT, row = 16 * (c % TT) + i16, r = r0 + 16 * u + 4 * quarter;
      if (row >= first && row < end && r < a.padded) *reinterpret_cast<f32x4_t*>(a.v + ((int64_t)split * a.T + p0 + row) * a.padded + r) = sum;
    }
    __syncthreads();
  }
}

template <int RT, int TT>
constexpr int down_lds() {
  const int stages = 2 * (RT + TT) * 16 * kStageRow, sums = 4 * RT * TT * 1024;
  return stages > sums ? stages : sums;
}

constexpr int kTogether = 8;   // partial sums asked for at once: their latency is what a short call waits for

// Two neighbouring ranks of a row of v, summed over the workgroups first, first + step, ... of those that shared K.
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
__device__ __forceinline__ f32x2_t sum_parts(const AdapterArgs& a, const float* from, int first, int step) {
  f32x2_t v = {0.f, 0.f};
  for (int s0 = first; s0 < a.splits; s0 += kTogether * step) {
    f32x2_t part[kTogether];
#pragma unroll
    for (int s = 0; s < kTogether; ++s) {
      part[s] = f32x2_t{0.f, 0.f};
      if (s0 + s * step < a.splits) part[s] = *reinterpret_cast<const f32x2_t*>(from + (int64_t)(s0 + s * step) * a.T * a.padded);
    }
#pragma unroll
    for (int s = 0; s < kTogether; ++s) v.x += part[s].x, v.y += part[s].y;
  }
  return v;
}
// As two bf16 numbers each: their upper bits and what is left.
__device__ __forceinline__ u32x2_t in_two(f32x2_t v) {
  const float v0 = v.x, v1 = v.y;
  const uint32_t top0 = __builtin_bit_cast(uint32_t, v0) & 0xFFFF0000u, top1 = __builtin_bit_cast(uint32_t, v1) & 0xFFFF0000u;
  const float up0 = __builtin_bit_cast(float, top0), up1 = __builtin_bit_cast(float, top1);
  const float rest0 = up0 == v0 ? 0.f : v0 - up0, rest1 = up1 == v1 ? 0.f : v1 - up1;   // (infinity less infinity would be NaN)
  return u32x2_t{top1 | top0 >> 16, pack_bf16(rest0, rest1)};
}

// The rows [first, end) of a block, which have no adapter or one without ranks: out is y, in the columns n_first .. n_end - 1.  A thread copies eight columns of one row at a time.
__device__ __forceinline__ void copy_rows(const AdapterArgs& a, int64_t p0, int first, int end, int n_first, int n_end, int thread, int threads) {
  const int pieces = (n_end - n_first + 7) / 8;
#pragma unroll 1
  for (int at = thread; at < (end - first) * pieces; at += threads) {
    const int row = at / pieces, n = n_first + (at - row * pieces) * 8, t = a.rows[p0 + first + row];
    if ((uint32_t)t >= (uint32_t)a.T) continue;
    const uint16_t* from = a.y + t * a.ldy;
    uint16_t* to = a.out + t * a.ld_out;
    if (n + 8 <= a.N) {
      u32x4_t v;
      __builtin_memcpy(&v, from + n, 16);
      __builtin_memcpy(to + n, &v, 16);
    } else {
#pragma unroll 1
      for (int h = n; h < a.N; ++h) to[h] = from[h];
    }
  }
}

// Sum of v over the G lanes of a row of B, in all of them.
template <int G>
__device__ __forceinline__ float over_row(float v) {
  auto moved = [](float x, auto ctrl) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false)); };
  if constexpr (G > 1) v += moved(v, std::integral_constant<int, 0xB1>());    // lane l ^ 1
  if constexpr (G > 2) v += moved(v, std::integral_constant<int, 0x4E>());    // l ^ 2
  if constexpr (G > 4) v += moved(v, std::integral_constant<int, 0x141>());   // the other four of eight
  if constexpr (G > 8) v += moved(v, std::integral_constant<int, 0x140>());   // the other eight of 16
  if constexpr (G > 16) v += xor16(v);
  return v;
}

// The second kernel for runs of few rows: B is read along its memory, 16 bytes a lane, G lanes to a row (8 G >= rank), and each lane multiplies its eight ranks by
// those of up to four rows of v, which it holds in registers.  No matrix operand is put together and nothing goes through LDS but v, once.
constexpr int kFewRows = 16;   // of a block
template <int G>
__global__ __launch_bounds__(256) void ccq_adapter_few_kernel(AdapterArgs a) {
  constexpr int kLoads = G < 8 ? G : 8, kRowsOfB = 64 / G, kColumns = kLoads * kRowsOfB, kWide = 8 * G;   // of a step of a wavefront
  __shared__ __align__(16) float v[kFewRows * kWide];
  __shared__ f32x2_t shares[256];
  uint32_t g = blockIdx.x;
  const int n_first = (int)((g % a.chunks) * (int64_t)a.columns);
  g /= a.chunks;
  const uint32_t later = g / a.blocks, turn = a.together - 1 - later;
  const int64_t p0 = (a.block0 + (g - later * a.blocks)) * kFewRows;
  const int row_of_lane = (threadIdx.x & 63) < kFewRows && p0 + (threadIdx.x & 63) < a.T ? a.rows[p0 + (threadIdx.x & 63)] : -1;   // (asked for together with the adapters)
  Runs runs(a, p0, kFewRows);
  runs.skip((int)turn);
  if (!runs.starts) return;
  const int n_end = (int)min(n_first + (int64_t)a.columns, (int64_t)a.N), tid = threadIdx.x, pieces = a.rank / 8;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), piece = lane % G, sub = lane / G;
  for (; runs.starts; runs.skip(a.together)) {
    const int first = runs.first(), end = runs.end();
    const int i = __builtin_amdgcn_readfirstlane(__shfl(runs.adapter, first));
    const int rank = i < 0 ? 0 : rank_of(a, i);
    if (i < 0 || rank == 0) {
      if (a.copies) copy_rows(a, p0, first, end, n_first, n_end, tid, 256);
      continue;
    }
    // Of four rows from row0 on: a step's B and y.  (Past N the last column is read again, and not stored; pieces past the rank are masked.)
    int t[4];
    auto take_rows = [&](int row0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        t[j] = row0 + j < end ? __builtin_amdgcn_readlane(row_of_lane, row0 + j) : -1;
        if ((uint32_t)t[j] >= (uint32_t)a.T) t[j] = -1;
      }
    };
    const uint16_t* const b_all = a.b + (int64_t)i * a.N * a.rank + 8 * min(piece, pieces - 1);
    auto load = [&](int n, u32x4_t (&b)[kLoads], uint16_t (&y)[4]) {
#pragma unroll
      for (int c = 0; c < kLoads; ++c) b[c] = *reinterpret_cast<const u32x4_t*>(b_all + (int64_t)min(n + c * kRowsOfB + sub, a.N - 1) * a.rank);
      const int column = min(n + piece * kRowsOfB + sub, a.N - 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = t[j] >= 0 ? a.y[t[j] * a.ldy + column] : 0;
    };
    const int n_mine = n_first + wave * kColumns;
    u32x4_t b[kLoads], next[kLoads];
    uint16_t y[4], y_next[4];
    take_rows(first);
    load(n_mine, next, y_next);   // (asked for before v is there)
    u32x4_t mask;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const int r = 8 * piece + 2 * h;
      mask[h] = (r < rank ? 0xFFFFu : 0u) | (r + 1 < rank ? 0xFFFF0000u : 0u);
    }
    // v: pairs of ranks of each row, the workgroups that shared K among as many threads as there are for each pair
    const float scale = a.scales ? a.scales[i] : 1.f;
    const int rows = end - first, pairs = rows * (kWide / 2), sharing = max(1, min(256 / pairs, (a.splits + kTogether - 1) / kTogether));
#pragma unroll 1
    for (int c0 = 0; c0 < pairs; c0 += 256) {
      const int c = c0 + tid % min(pairs, 256), share = tid / min(pairs, 256), row = c / (kWide / 2), r = c % (kWide / 2) * 2;
      f32x2_t two = {0.f, 0.f};
      if (c < pairs && share < sharing && r < rank) two = sum_parts(a, a.v + (p0 + first + row) * a.padded + r, share, sharing);
      if (sharing > 1) {
        shares[tid] = two;
        __syncthreads();
        if (tid < pairs)
          for (int s = 1; s < sharing; ++s) two.x += shares[s * pairs + tid].x, two.y += shares[s * pairs + tid].y;
      }
      if (c < pairs && share == 0) *reinterpret_cast<f32x2_t*>(v + row * kWide + r) = f32x2_t{r < rank ? two.x * scale : 0.f, r + 1 < rank ? two.y * scale : 0.f};
    }
    __syncthreads();
#pragma unroll 1
    for (int row0 = first; row0 < end; row0 += 4) {
      f32x4_t w[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = min(row0 + j, end - 1) - first;
        w[j][0] = *reinterpret_cast<const f32x4_t*>(v + row * kWide + 8 * piece);
        w[j][1] = *reinterpret_cast<const f32x4_t*>(v + row * kWide + 8 * piece + 4);
      }
      if (row0 > first) {
        take_rows(row0);
        load(n_mine, next, y_next);
      }
#pragma unroll 1
      for (int n = n_mine; n < n_end; n += 4 * kColumns) {
#pragma unroll
        for (int c = 0; c < kLoads; ++c) b[c] = next[c];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = y_next[j];
        if (n + 4 * kColumns < n_end) load(n + 4 * kColumns, next, y_next);
        const int column = n + piece * kRowsOfB + sub;   // whose sum this lane keeps
        const bool keeps = piece < kLoads && column < n_end;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kLoads; ++c) {
          float x[8];
          const u32x4_t bits = b[c] & mask;
#pragma unroll
          for (int h = 0; h < 4; ++h) x[2 * h] = bf16_lo(bits[h]), x[2 * h + 1] = bf16_hi(bits[h]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (row0 + j >= end) continue;
            float d = 0.f;
#pragma unroll
            for (int h = 0; h < 8; ++h) d = __builtin_fmaf(x[h], w[j][h >> 2][h & 3], d);
            d = over_row<G>(d);
            sum[j] = piece == c ? d : sum[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (keeps && t[j] >= 0) a.out[t[j] * a.ld_out + column] = to_bf16(bf16_lo(y[j]) + sum[j]);
      }
    }
    __syncthreads();
  }
}

// Columns of a piece of the second kernel, and pieces of 16 bytes between its rows of B in LDS: an odd number, so that eight rows' reads meet all banks.
constexpr int kRowFloats = 4;   // between a row's results in LDS and the next one's, for the same reason
constexpr int kUpWaves = 8;
constexpr int piece_columns(int kk) { return kk <= 2 ? 256 : 128; }
__host__ __device__ constexpr int b_pitch(int rank) { return (rank / 8 | 1) * 16; }
template <int KK>
constexpr int up_lds(int rank) {
  return 2 * KK * 1024 + 16 * (piece_columns(KK) + kRowFloats) * 4 + piece_columns(KK) * b_pitch(rank);
}

// KK: steps of 32 ranks.  A workgroup takes its columns in pieces; B and y of the next piece are asked for while one is worked on.  B goes through LDS for the
// reason given above, the products go through LDS to meet y, and y and out are read and written along their rows.
template <int KK>
__global__ __launch_bounds__(64 * kUpWaves, 4) void ccq_adapter_up_kernel(AdapterArgs a) {
  extern __shared__ __align__(256) uint8_t lds[];
  constexpr int kThreads = 64 * kUpWaves, kColumns = piece_columns(KK), kTiles = kColumns / (16 * kUpWaves);   // of 16 columns for each wavefront
  constexpr int kPitch = kColumns + kRowFloats;
  constexpr int kRowPieces = kColumns / 8, kRowsAtOnce = kThreads / kRowPieces, kMyRows = 16 < kRowsAtOnce ? 1 : 16 / kRowsAtOnce;
  constexpr int kMyB = kColumns * KK * 4 / kThreads;   // pieces of 16 bytes of B, at most
  u32x4_t* const parts = reinterpret_cast<u32x4_t*>(lds);                                   // [2][KK][64]: v as matrix operands, its upper and its lower bits
  float* const products = reinterpret_cast<float*>(lds + 2 * KK * 1024);              // [16][kPitch]
  uint8_t* const b_lds = lds + 2 * KK * 1024 + 16 * kPitch * 4;
  uint32_t g = blockIdx.x;
  const int64_t n_first = (int64_t)(g % a.chunks) * a.columns;
  g /= a.chunks;
  const uint32_t later = g / a.blocks, turn = a.together - 1 - later;   // (the runs that few blocks have first: begun last, they would run alone)
  const int64_t p0 = (a.block0 + (g - later * a.blocks)) * 16;
  Runs runs(a, p0, 16);
  runs.skip((int)turn);
  if (!runs.starts) return;
  const int pitch = b_pitch(a.rank), row_pieces = a.rank / 8;
  const int n_end = (int)min(n_first + a.columns, (int64_t)a.N);
  for (; runs.starts; runs.skip(a.together)) {
    const int first = runs.first(), end = runs.end();
    const int i = __builtin_amdgcn_readfirstlane(__shfl(runs.adapter, first));
    const int rank = i < 0 ? 0 : rank_of(a, i);
    int thread = threadIdx.x;
    asm volatile("" : "+v"(thread));   // (what follows from it is formed in the run, not kept in registers over all of them)
    const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), i16 = lane & 15, quarter = lane >> 4;
    if (rank == 0) {   // out is y
      if (a.copies) copy_rows(a, p0, first, end, (int)n_first, n_end, thread, kThreads);
      continue;
    }
    const int last = (rank - 1) >> 5;
    const int column = thread % kRowPieces * 8, row0 = thread / kRowPieces;   // this thread's part of y and out: rows row0 + kRowsAtOnce j
    int t[kMyRows];
    bool mine[kMyRows];   // rows of this run
#pragma unroll
    for (int j = 0; j < kMyRows; ++j) {
      const int row = row0 + kRowsAtOnce * j;
      const int at = row >= first && row < end ? a.rows[p0 + row] : -1;
      mine[j] = (uint32_t)at < (uint32_t)a.T;
      t[j] = at;
    }

    u32x4_t b[kMyB], y[kMyRows], y_next[kMyRows];
    const uint16_t* const b_all = a.b + (int64_t)i * a.N * a.rank;
    const int b_row = thread / row_pieces, b_piece = thread - b_row * row_pieces, rows_on = kThreads / row_pieces, pieces_on = kThreads - rows_on * row_pieces;
    // f(j, row, piece) for this thread's pieces of B
    auto my_b = [&](auto f) {
      int row = b_row, c = b_piece;
#pragma unroll
      for (int j = 0; j < kMyB; ++j) {
        f(j, row, c);
        row += rows_on, c += pieces_on;
        if (c >= row_pieces) c -= row_pieces, ++row;
      }
    };
    // (past the piece, N and the ranks in use the last ones are read again: they are in the caches, and no sum that is kept meets them)
    const int top_piece = (rank - 1) >> 3;
    auto load_b = [&](int n0) {
      const int top_row = min(kColumns, a.N - n0) - 1;
      const uint16_t* const from = b_all + (int64_t)n0 * a.rank;
      my_b([&](int j, int row, int c) { b[j] = *reinterpret_cast<const u32x4_t*>(from + (uint32_t)(min(row, top_row) * a.rank + 8 * min(c, top_piece))); });
    };
    auto load_y = [&](int n0) {
      const int n = n0 + column;
#pragma unroll
      for (int j = 0; j < kMyRows; ++j)
        if (mine[j] && n + 8 <= a.N) y_next[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any_t*>(a.y + (int64_t)t[j] * a.ldy + n));
    };
    auto store = [&](int n0) {
      const int n = n0 + column;
#pragma unroll
      for (int j = 0; j < kMyRows; ++j) {
        if (!mine[j] || n >= a.N) continue;
        const float* d = products + (row0 + kRowsAtOnce * j) * kPitch + column;
        uint16_t* o = a.out + (int64_t)t[j] * a.ld_out + n;
        if (n + 8 <= a.N) {
          const f32x4_t d0 = *reinterpret_cast<const f32x4_t*>(d), d1 = *reinterpret_cast<const f32x4_t*>(d + 4);
#pragma unroll
          for (int h = 0; h < 4; ++h)
            y[j][h] = pack_bf16(bf16_lo(y[j][h]) + (h < 2 ? d0[2 * h] : d1[2 * h - 4]), bf16_hi(y[j][h]) + (h < 2 ? d0[2 * h + 1] : d1[2 * h - 3]));
          __builtin_nontemporal_store(y[j], reinterpret_cast<u32x4_any_t*>(o));
        } else {   // the last columns
          const uint16_t* from = a.y + (int64_t)t[j] * a.ldy + n;
#pragma unroll 1
          for (int h = 0; h < a.N - n; ++h) o[h] = to_bf16(bf16_lo(from[h]) + d[h]);
        }
      }
    };
    load_b((int)n_first);   // (asked for before v is there)
    load_y((int)n_first);

    const float scale = a.scales ? a.scales[i] : 1.f;
#pragma unroll 1
    for (int c = thread; c < KK * 256; c += kThreads) {   // rows, and 16 KK pairs of ranks of each
      const int row = c / (16 * KK), r = c % (16 * KK) * 2;
      f32x2_t two = {0.f, 0.f};
      if (row >= first && row < end && r < rank) two = sum_parts(a, a.v + (p0 + row) * a.padded + r, 0, 1);
      two.x = r < rank ? two.x * scale : 0.f, two.y = r + 1 < rank ? two.y * scale : 0.f;
      const u32x2_t halves = in_two(two);
      const int at = r / 32 * 256 + (r / 8 % 4 * 16 + row) * 4 + r / 2 % 4;
      reinterpret_cast<uint32_t*>(parts)[at] = halves.x;
      reinterpret_cast<uint32_t*>(parts)[KK * 256 + at] = halves.y;
    }
    u32x4_t mask;   // of the last step: ranks in use
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = 32 * last + 8 * quarter + 2 * j;
      mask[j] = (r < rank ? 0xFFFFu : 0u) | (r + 1 < rank ? 0xFFFF0000u : 0u);
    }
    for (int n0 = (int)n_first; n0 < n_end; n0 += kColumns) {
      my_b([&](int j, int row, int c) {
        if (row < kColumns) *reinterpret_cast<u32x4_t*>(b_lds + row * pitch + c * 16) = b[j];
      });
      __syncthreads();   // (before the first piece v is in LDS too)
#pragma unroll
      for (int j = 0; j < kMyRows; ++j) y[j] = y_next[j];
      if (n0 + kColumns < n_end) {
        load_b(n0 + kColumns);
        load_y(n0 + kColumns);
      }
      f32x4_t acc[kTiles];
#pragma unroll
      for (int u = 0; u < kTiles; ++u) acc[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int k = 0; k <= last; ++k) {
        const u32x4_t hi = parts[k * 64 + lane], lo = parts[(KK + k) * 64 + lane];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
          u32x4_t bb = *reinterpret_cast<const u32x4_t*>(b_lds + ((wave * kTiles + u) * 16 + i16) * pitch + min(4 * k + quarter, row_pieces - 1) * 16);
          if (k == last) bb &= mask;
          acc[u] = mfma(bb, lo, acc[u]);
          acc[u] = mfma(bb, hi, acc[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < kTiles; ++u) *reinterpret_cast<f32x4_t*>(products + i16 * kPitch + (wave * kTiles + u) * 16 + 4 * quarter) = acc[u];
      __syncthreads();
      store(n0);
    }
    __syncthreads();
  }
}

// The second product for many rows, in two kernels.  The first adds v up, multiplies it by the scales and leaves it as matrix operands, 32 rows at a time: its upper bits and
// its lower ones, [blocks of 32 rows][2][2 KK][64] pieces of 16 bytes.
template <int KK>
__global__ __launch_bounds__(256) void ccq_adapter_join_kernel(AdapterArgs a) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, p = at / (16 * KK);
  const int r = (int)(at % (16 * KK)) * 2;
  f32x2_t two = {0.f, 0.f};
  if (p < a.T) {
    const int i = a.experts[p];
    if ((uint32_t)i < (uint32_t)a.count) {
      const int rank = rank_of(a, i);
      const float scale = a.scales ? a.scales[i] : 1.f;
      if (r < rank) two = sum_parts(a, a.v + p * a.padded + r, 0, 1);
      two.x = r < rank ? two.x * scale : 0.f, two.y = r + 1 < rank ? two.y * scale : 0.f;
    }
  }
  const u32x2_t halves = in_two(two);
  uint32_t* const to = reinterpret_cast<uint32_t*>(a.parts + p / 32 * (4 * KK * 64)) + ((p % 32 / 16 * KK + r / 32) * 64 + r / 8 % 4 * 16 + p % 16) * 4 + r / 2 % 4;
  to[0] = halves.x;
  to[2 * KK * 64 * 4] = halves.y;
}

// The second: a workgroup keeps 128 columns of an adapter's B in registers, a wavefront 32 of them, and goes along the rows, 32 at a time; y and v of the next 32 rows are on
// their way, v to LDS since all wavefronts need all of it, while the products of these go through LDS to meet theirs.  The work of all columns and rows lies on one line, of
// which each workgroup has as much.  STREAMS: y is not to stay in the caches.
// 2048 x 18432, rank 64: 35 us, 4.3 TB/s of y and out (a large copy 5.1); with v read by every wavefront for itself 39, with y two or three blocks ahead 36 and 37, with 64 columns
// 43 and with 256 columns 42 where 128 took 40.  Stores that pass the caches by are worth 1 to 2 us of 17 where y is to stay, and cost 1 to 3 of 40 where not.
constexpr int kRowsColumns = 128, kRowsThreads = 2 * kRowsColumns;
template <int KK, bool STREAMS>
__global__ __launch_bounds__(kRowsThreads, KK <= 2 ? 4 : 2) void ccq_adapter_rows_kernel(AdapterArgs a) {
  constexpr int kColumns = kRowsColumns, kPitch = kColumns + kRowFloats, kMyRows = 2;   // rows row0 and row0 + 16 of a thread
  constexpr int kDeep = KK <= 2 ? 1 : 2;
  constexpr int kParts = 4 * KK * 64;   // pieces of v of 32 rows
  __shared__ __align__(16) float products[32 * kPitch];
  __shared__ u32x4_t v[kParts];
  const int blocks = (int)(((int64_t)a.T + 31) / 32);
  // (an XCD's workgroups, every eighth, lie side by side on the line: its L2 meets an eighth of B)
  const uint32_t turn = gridDim.x % 8 == 0 ? blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8 : blockIdx.x;
  const int64_t all = (int64_t)blocks * a.chunks, from = (int64_t)turn * a.blocks_each, to = min(from + a.blocks_each, all);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, quarter = lane >> 4;
  const int column = threadIdx.x % (kColumns / 8) * 8, row0 = threadIdx.x / (kColumns / 8);
  struct Place {
    int piece, block;
    __device__ __forceinline__ void step(int blocks) {
      if (++block == blocks) block = 0, ++piece;
    }
  };
  // this thread's rows of a block, and their y
  auto rows_of = [&](const Place& p, int (&t)[kMyRows]) {
#pragma unroll
    for (int j = 0; j < kMyRows; ++j) {
      const int64_t at = (int64_t)p.block * 32 + row0 + 16 * j;
      t[j] = at < a.T ? a.rows[at] : -1;
      if ((uint32_t)t[j] >= (uint32_t)a.T) t[j] = -1;
    }
  };
  auto load_y = [&](const Place& p, const int (&t)[kMyRows], u32x4_t (&y)[kMyRows]) {
    const int n = p.piece * kColumns + column;
#pragma unroll
    for (int j = 0; j < kMyRows; ++j)
      if (t[j] >= 0 && n + 8 <= a.N) {
        const u32x4_any_t* at = reinterpret_cast<const u32x4_any_t*>(a.y + (int64_t)t[j] * a.ldy + n);
        if constexpr (STREAMS) y[j] = __builtin_nontemporal_load(at);
        else y[j] = *at;
      }
  };
  auto load_v = [&](const Place& p, u32x4_t (&part)[KK]) {
    const u32x4_t* const parts = a.parts + (int64_t)p.block * kParts + threadIdx.x;
#pragma unroll
    for (int c = 0; c < KK; ++c) part[c] = parts[c * kRowsThreads];
  };
  // t[d], y[d]: of the block d further on; of one beyond them the rows only
  Place now = {(int)(from / blocks), (int)(from % blocks)}, ahead = now;
  int t[kDeep + 1][kMyRows];
  u32x4_t y[kDeep][kMyRows], b[KK][2], v_next[KK];
  load_v(now, v_next);
#pragma unroll
  for (int d = 0; d < kDeep; ++d) {
    rows_of(ahead, t[d]);
    if (from + d < to) load_y(ahead, t[d], y[d]);
    ahead.step(blocks);
  }
  rows_of(ahead, t[kDeep]);
  int adapters = Runs::of_lane(a, (int64_t)now.block * 32, 32);
  int held = -1, held_piece = -1, last = -1;   // whose B the registers hold, and its last step of 32 ranks
  for (int64_t at = from; at < to; ++at) {
    const int n_first = now.piece * kColumns, n = n_first + column;
    const bool whole = n + 8 <= a.N;
    Runs runs(a, (int64_t)now.block * 32, 32, adapters);
    Place next = now;
    next.step(blocks);
    // (the last block's is read no more: its products were met behind a barrier)
#pragma unroll
    for (int c = 0; c < KK; ++c) v[threadIdx.x + c * kRowsThreads] = v_next[c];
    load_v(next, v_next);
    adapters = Runs::of_lane(a, (int64_t)next.block * 32, 32);
    u32x4_t y_next[kMyRows];   // of the block kDeep further on
    if (at + kDeep < to) load_y(ahead, t[kDeep], y_next);
    __syncthreads();
    for (; runs.starts; runs.skip(1)) {
      const int first = runs.first(), end = runs.end();
      const int i = __builtin_amdgcn_readfirstlane(__shfl(runs.adapter, first));
      if (i < 0 && !a.copies) continue;
      if (i >= 0 && (i != held || now.piece != held_piece)) {
        held = i, held_piece = now.piece;
        const int rank = rank_of(a, i);
        last = (rank - 1) >> 5;
#pragma unroll
        for (int k = 0; k < KK; ++k)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int r = 32 * k + 8 * quarter;
            u32x4_t bits = *reinterpret_cast<const u32x4_t*>(a.b + ((int64_t)i * a.N + min(n_first + 32 * wave + 16 * u + i16, a.N - 1)) * a.rank + min(r, a.rank - 8));
#pragma unroll
            for (int h = 0; h < 4; ++h) bits[h] &= (r + 2 * h < rank ? 0xFFFFu : 0u) | (r + 2 * h + 1 < rank ? 0xFFFF0000u : 0u);
            b[k][u] = bits;
          }
      }
      const bool adds = i >= 0 && last >= 0;
      if (adds) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int k = 0; k < KK; ++k) {
            if (k > last) break;
            const u32x4_t hi = v[(w * KK + k) * 64 + lane], lo = v[(2 * KK + w * KK + k) * 64 + lane];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              acc[u] = mfma(b[k][u], lo, acc[u]);
              acc[u] = mfma(b[k][u], hi, acc[u]);
            }
          }
#pragma unroll
          for (int u = 0; u < 2; ++u) *reinterpret_cast<f32x4_t*>(products + (16 * w + i16) * kPitch + 32 * wave + 16 * u + 4 * quarter) = acc[u];
        }
        __syncthreads();
      }
#pragma unroll
      for (int j = 0; j < kMyRows; ++j) {
        const int row = row0 + 16 * j;
        if (row < first || row >= end || t[0][j] < 0 || n >= a.N || (!adds && !a.copies)) continue;
        const float* d = products + row * kPitch + column;
        uint16_t* o = a.out + (int64_t)t[0][j] * a.ld_out + n;
        if (whole) {
          u32x4_t sum = y[0][j];
          if (adds) {
            const f32x4_t d0 = *reinterpret_cast<const f32x4_t*>(d), d1 = *reinterpret_cast<const f32x4_t*>(d + 4);
#pragma unroll
            for (int h = 0; h < 4; ++h)
              sum[h] = pack_bf16(bf16_lo(sum[h]) + (h < 2 ? d0[2 * h] : d1[2 * h - 4]), bf16_hi(sum[h]) + (h < 2 ? d0[2 * h + 1] : d1[2 * h - 3]));
          }
          if constexpr (STREAMS) *reinterpret_cast<u32x4_any_t*>(o) = sum;
          else __builtin_nontemporal_store(sum, reinterpret_cast<u32x4_any_t*>(o));
        } else {   // the last columns
          const uint16_t* from_y = a.y + (int64_t)t[0][j] * a.ldy + n;
#pragma unroll 1
          for (int h = 0; h < a.N - n; ++h) o[h] = adds ? to_bf16(bf16_lo(from_y[h]) + d[h]) : from_y[h];
        }
      }
      if (adds) __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kMyRows; ++j) {
#pragma unroll
      for (int d = 0; d + 1 < kDeep; ++d) y[d][j] = y[d + 1][j];
      y[kDeep - 1][j] = y_next[j];
#pragma unroll
      for (int d = 0; d < kDeep; ++d) t[d][j] = t[d + 1][j];
    }
    now = next;
    ahead.step(blocks);
    rows_of(ahead, t[kDeep]);
  }
}

constexpr int at_once(int kk) { return (kk <= 2 ? 512 : 256) * (256 / kRowsColumns); }   // workgroups of the last kernel that the chip holds

// How the rows and K of a call are cut.
struct Plan {
  int tiles;       // of 16 rows in a block
  int64_t blocks;
  int together, splits, steps, rank_tiles, chunks, padded;
  bool few, many;  // the second kernel for runs of few rows, the kernels for many rows
  int columns, column_chunks;
  int steps32;     // of 32 ranks: 1, 2, 4 or 8
};

Plan plan_of(const ccq_adapter_set* s, int T) {
  Plan p;
  // Runs of four rows or so, as far as one can tell here: the second product of 512 rows with 128 adapters of rank 16 (4096 to 4096) takes 13.6 us and by MFMA 15.7, of 128 rows
  // with 32 adapters 8.1 and 7.8; of 512 rows with 64 adapters 12.5 and 12.6, of 128 with 32 adapters of rank 64 14.3 and 9.5, and of 512 with 128 adapters of rank 64 36 and 25.5.
  p.few = (int64_t)T * s->rank <= 8192 && T <= 4 * (int64_t)s->count;
  // The launch that joins v costs 3 to 4 us: second products without and with it take, of rank 64, 8.5 and 10.7 us at 512 rows to 4096, 12.4 and 12.5 at 1024 rows to 4096, 13.5 and 12.6 at
  // 512 rows to 8192, 7.5 and 11.3 at 2048 rows to 1024; of rank 16 7.3 and 9.1 at 512 rows to 4096, 9.8 and 10.5 at 1024.  (T: its workgroups are one launch's.)
  p.many = !p.few && T >= 512 && (int64_t)T * s->N >= 4 << 20 && T <= 1 << 22;
  // Blocks of 32 rows read A half as often but are half as many: with 16 rows and with 32, all launches, four adapters,
  // 512 rows of 8192 to 8192, rank 64, take 22.4 and 24.6 us, 1024 24.6 and 25.0, 1536 30.9 and 32.1, 2048 35.8 and 35.2; rank 32, 4096 to 4096, 1024 rows 16.8 and 17.5, 2048 21.2 and 21.1, 4096 31.5 and 30.9.
  p.tiles = p.many && T >= 2048 ? 2 : 1;
  const int rows = 16 * p.tiles;
  p.blocks = ((int64_t)T + rows - 1) / rows;
  // Every adapter that begins inside a block makes one more run.  Few blocks have room for as many as there are rows (a workgroup that finds none ends at once, one
  // that finds two takes twice as long: 37 rows of 12 adapters 14.6 us with the mean number, 11.1 us so); more have it for the mean number.
  const int64_t begins = s->count < T ? s->count : T;
  const int64_t runs = p.blocks <= 16 ? 1 + begins : 1 + (begins + p.blocks - 1) / p.blocks;
  p.together = (int)(runs < rows ? runs : rows);
  if (p.together > T) p.together = T;
  p.padded = (s->rank + 15) / 16 * 16;
  p.rank_tiles = p.padded > 64 ? 8 : p.padded > 32 ? 4 : p.padded > 16 ? 2 : 1;
  p.chunks = (p.padded + 16 * p.rank_tiles - 1) / (16 * p.rank_tiles);
  const int steps = (s->K + kStageColumns - 1) / kStageColumns;
  const int64_t busy = p.blocks + begins < p.blocks * p.together ? p.blocks + begins : p.blocks * p.together;   // workgroups with work
  // K is shared by a power of two of workgroups, neighbours in the grid: with eight and more of them an XCD's L2 meets the same columns of all A.
  // Up to as many workgroups as the chip holds.  Where every workgroup of the second product adds the shares up again fewer are worth more: 300 rows of 8192 to 8192, rank 64, 18.3 us
  // with 256, 21.7 with 512.  (Where many adapters make x A^T the larger part it is the other way: 512 rows of 4096 to 4096 with 128 adapters 54 and 47.5.)  Of ranks above 64 a CU holds two: 2048
  // rows of 8192, rank 128, 22.0 us in x A^T with half as many, 23.8 otherwise; 256 rows 26.1 in all and 26.5.
  const int wanted = (p.many ? 512 : 256) / (p.padded > 64 ? 2 : 1);
  int splits = 1;
  while (splits < 32 && busy * p.chunks * splits < wanted && steps >= splits * 4) splits *= 2;
  p.steps = (steps + splits - 1) / splits;
  p.splits = (steps + p.steps - 1) / p.steps;
  p.steps32 = p.padded <= 32 ? 1 : p.padded <= 64 ? 2 : p.padded <= 128 ? 4 : 8;
  const int width = p.few || p.many || p.padded <= 64 ? 256 : 128;
  const int64_t pieces = ((int64_t)s->N + width - 1) / width;
  // Parts of the columns: runs of few rows in a multiple of eight, for the same reason.  The MFMA kernel's workgroups all at once (two on a CU, or one by the LDS that ranks near 256 need), since a second
  // turn waits for the first one's end: 256 rows of 8192 to 8192, rank 64, in runs of any length 11.0 us with 480 workgroups, 14.5 with 640; 3000 rows to 1000 8.4 and 11.2.
  const int64_t places = p.padded > 128 && 2 * up_lds<8>(s->rank) > 160 * 1024 ? 256 : 512;
  int64_t parts = p.few ? ((512 + busy - 1) / busy + 7) / 8 * 8 : busy < places ? places / busy : 1;
  p.columns = (int)((pieces + parts - 1) / parts * width);
  p.column_chunks = (int)(((int64_t)s->N + p.columns - 1) / p.columns);
  if (p.many) p.columns = kRowsColumns, p.column_chunks = (s->N + kRowsColumns - 1) / kRowsColumns;
  return p;
}

template <typename K>
bool launch(K kernel, const AdapterArgs& a, unsigned groups, int threads, int lds, hipStream_t s) {
  if (lds > 48 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return false;
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(threads), (size_t)lds, s, a);
  return true;
}
template <int RT, int TT>
bool down(const AdapterArgs& a, unsigned groups, hipStream_t s) {
  return launch(ccq_adapter_down_kernel<RT, TT>, a, groups, 256, down_lds<RT, TT>(), s);
}
template <int KK>
bool up(const AdapterArgs& a, unsigned groups, hipStream_t s) {
  return launch(ccq_adapter_up_kernel<KK>, a, groups, 64 * kUpWaves, up_lds<KK>(a.rank), s);
}

int64_t v_bytes(const Plan& p, int T) { return ((int64_t)p.splits * T * p.padded * 4 + 15) / 16 * 16; }

}  // namespace

int64_t adapters_workspace(const ccq_adapter_set* set, int T) {
  if (T == 0) return 0;
  const Plan p = plan_of(set, T);
  return v_bytes(p, T) + (p.many ? ((int64_t)T + 31) / 32 * (p.steps32 * 4 * 1024) : 0);
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
  bool ok = true;
  auto in_parts = [&](int64_t per_block, int threads, auto part) {   // as many blocks at a time as a launch has room for
    const int64_t most = most_groups(threads) / per_block;
    for (int64_t b = 0; b < p.blocks && ok; b += most) {
      a.block0 = b;
      a.blocks = (uint32_t)(p.blocks - b < most ? p.blocks - b : most);
      ok = part((unsigned)(a.blocks * per_block));
    }
  };
  a.chunks = p.chunks;
  in_parts((int64_t)p.together * p.chunks * p.splits, 256, [&](unsigned n) {
    if (p.rank_tiles == 1) return two ? down<1, 2>(a, n, s) : down<1, 1>(a, n, s);
    if (p.rank_tiles == 2) return two ? down<2, 2>(a, n, s) : down<2, 1>(a, n, s);
    if (p.rank_tiles == 4) return two ? down<4, 2>(a, n, s) : down<4, 1>(a, n, s);
    return two ? down<8, 2>(a, n, s) : down<8, 1>(a, n, s);
  });
  a.chunks = p.column_chunks;
  if (p.many) {
    a.parts = reinterpret_cast<u32x4_t*>(static_cast<char*>(workspace) + v_bytes(p, T));
    // What the caches hold of y, x and v is worth keeping while y and out fit the last of them (256 MB) beside other things: with loads that leave them alone 2048 rows of 8192
    // take 20.0 us in this kernel and 16.7 with plain ones, 2048 rows of 18432 with x from memory 59.5 us in all and 63.3.
    const bool streams = (int64_t)T * set->N * 4 > (int64_t)128 << 20;
    const int64_t blocks = ((int64_t)T + 31) / 32, all = blocks * p.column_chunks, most = at_once(p.steps32), groups = all < most ? all : most;
    a.blocks_each = (all + groups - 1) / groups;
    auto join_rows = [&](auto kk) {
      constexpr int KK = decltype(kk)::value;
      return ok && launch(ccq_adapter_join_kernel<KK>, a, (unsigned)(blocks * 2 * KK), 256, 0, s) &&
             (streams ? launch(ccq_adapter_rows_kernel<KK, true>, a, (unsigned)groups, kRowsThreads, 0, s) : launch(ccq_adapter_rows_kernel<KK, false>, a, (unsigned)groups, kRowsThreads, 0, s));
    };
    ok = p.steps32 == 1   ? join_rows(std::integral_constant<int, 1>())
         : p.steps32 == 2 ? join_rows(std::integral_constant<int, 2>())
         : p.steps32 == 4 ? join_rows(std::integral_constant<int, 4>())
                          : join_rows(std::integral_constant<int, 8>());
    return ok && hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
  }
  in_parts((int64_t)p.together * p.column_chunks, p.few ? 256 : 64 * kUpWaves, [&](unsigned n) {
    if (p.few) {
      if (a.rank <= 8) return launch(ccq_adapter_few_kernel<1>, a, n, 256, 0, s);
      if (a.rank <= 16) return launch(ccq_adapter_few_kernel<2>, a, n, 256, 0, s);
      if (a.rank <= 32) return launch(ccq_adapter_few_kernel<4>, a, n, 256, 0, s);
      if (a.rank <= 64) return launch(ccq_adapter_few_kernel<8>, a, n, 256, 0, s);
      return a.rank <= 128 ? launch(ccq_adapter_few_kernel<16>, a, n, 256, 0, s) : launch(ccq_adapter_few_kernel<32>, a, n, 256, 0, s);
    }
    return p.steps32 == 1 ? up<1>(a, n, s) : p.steps32 == 2 ? up<2>(a, n, s) : p.steps32 == 4 ? up<4>(a, n, s) : up<8>(a, n, s);
  });
  return ok && hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
