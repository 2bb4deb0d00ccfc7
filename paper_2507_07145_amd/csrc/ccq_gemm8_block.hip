// 8-bit product for many rows.
//
// A workgroup of eight wavefronts, two per SIMD, owns a block of 64 MI x 256 outputs (two wavefronts along the rows, four along the columns,
// 32 MI x 64 each) and a share of K.  A block of K (128) is a step.  Activations and weights go from memory to LDS without passing
// registers (16 bytes a lane), in the order of memory; a row's eight 16-byte chunks are permuted by its number, so that the operand reads
// of neighbouring rows meet all banks.  Two steps lie in LDS, or three: before its last tile of rows a step's operands are all in registers, and its place
// is filled again, so that a copy has a step's time to arrive, or two.
// Products are scaled MFMAs 32x32x64, two for a block of K, into a fresh result that one multiply-add per register adds to the
// accumulators with the weights' scale.  The vector unit does not reach accumulation registers: 512 registers a wavefront would not help.
// 2048 rows, 8192 x 8192 (a block to each CU): 133 us, 2.1 PFLOP/s; 18432 x 7168: 276 - 290 us, 1.9.  Bound by the way into and out of LDS (64 KB in, 192 KB out a step) and by
// power; on 2048 x 16384 x 7168 an earlier form with 262 us took 190 without the copies, 231 with copies that all read one address, no less without
// waiting for them.
#include <algorithm>
#include <type_traits>

#include "ccq_gemm8.h"

namespace ccq {

namespace {

constexpr int kCols = 256, kWaves = 8;
constexpr int kWBytes = kCols * kScaleBlock;
constexpr int kScaleSteps = 64, kScalePitch = kScaleSteps + 4;   // steps whose row scales lie in LDS; bytes between rows

struct Gemm8Block {
  Gemm8Args a;
  int32_t m_tiles, n_tiles, shares, steps_per_share;
};

__device__ const uint4 kZeros = {0, 0, 0, 0};

// Which 16-byte chunk of a block of K a lane copies in an eighth of rows.  Eighths past the one in which the array ends are read as that one, its chunks with them: what
// lies past K goes by the chunk that is read.
__host__ __device__ __forceinline__ int block_chunk(int lane, int eighth) { return (lane & 7) ^ (lane >> 3) ^ (eighth & 1); }
__host__ __device__ __forceinline__ bool block_past_k(int lane, int eighth, int end, int k, int K) { return k + block_chunk(lane, eighth < end ? eighth : end) * 16 >= K; }

__device__ __forceinline__ f32x16_t zeros16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// Steps that lie in LDS.  A copy that waits for memory takes longer than a step of the smallest blocks: of 64 rows, 256 x 8192 x 8192, with three 49 us, with two 67.  In blocks of 128
// rows three gain 8 % where weights come from memory (73 us, 67) and lose 7 % where neighbours have read them (2048 x 2048 x 7168: 55 us, 59).
constexpr int slots(int mi) { return mi == 1 ? 3 : 2; }

template <int MI>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void ccq_gemm8_block_kernel(Gemm8Block p) {
  constexpr int kRows = 64 * MI, kXBytes = kRows * kScaleBlock;
  constexpr int kSlots = slots(MI);
  extern __shared__ __align__(256) uint8_t lds[];   // kSlots steps of activations, as many of weights, row scales, the weights' scales
  const Gemm8Args& a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
  const int wm = wave & 1, wn = wave >> 1;
  // workgroups of a chiplet (every eighth) take neighbouring tiles: up to eight blocks of rows of one block of columns, then the next columns
  const int tiles = p.m_tiles * p.n_tiles, per = (tiles + 7) / 8;
  const int share = blockIdx.x / (8 * per), at = blockIdx.x % (8 * per), t = at % 8 * per + at / 8;
  if (t >= tiles) return;
  const int panel = t / (8 * p.n_tiles), in_panel = t - panel * 8 * p.n_tiles, high = min(8, p.m_tiles - 8 * panel);
  const int m0 = (8 * panel + in_panel % high) * kRows, n0 = in_panel / high * kCols;
  const int first = share * p.steps_per_share, last = min(first + p.steps_per_share, a.blocks);

  // A copy moves eight rows; lane l fills position l % 8 of row l / 8 with the chunk that belongs there.  Uniform bases and 32-bit lane offsets:
  // one for even and odd eighths of rows, one for the eighth in which the array ends (rows past it are read in its place, and never stored).
  struct Rows {
    const uint8_t* base;
    int64_t ld;
    int end;          // the last eighth
    uint32_t at[3];
  };
  const int sub = lane >> 3;
  auto rows_from = [&](const uint8_t* base, int64_t ld, int last_row) {
    Rows r = {base, ld, last_row >> 3, {}};
#pragma unroll
    for (int e = 0; e < 3; ++e) r.at[e] = (uint32_t)(e < 2 ? sub : min(sub, last_row & 7)) * (uint32_t)ld + block_chunk(lane, e < 2 ? e : r.end) * 16;
    return r;
  };
  Rows xr = rows_from(a.x + (int64_t)m0 * a.ldx, a.ldx, a.M - 1 - m0), wr = rows_from(a.w + (int64_t)n0 * a.ldw, a.ldw, a.N - 1 - n0);
  auto copy = [&](Rows& r, int eighth, int step, uint8_t* to, auto RAGGED) {
    const int k = step * kScaleBlock;
    const uint8_t* base = r.base + (int64_t)min(eighth, r.end) * (8 * r.ld) + k;
    uint32_t from = eighth >= r.end ? r.at[2] : (eighth & 1) ? r.at[1] : r.at[0];
    asm volatile("" : "+v"(from));   // (the zero extension stays next to the load)
    if constexpr (decltype(RAGGED)::value) {   // zeros past K
      const uint8_t* src = base + from;
      if (block_past_k(lane, eighth, r.end, k, a.K)) src = reinterpret_cast<const uint8_t*>(&kZeros);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    } else {   // (with global loads to LDS under way the compiler waits for all LDS reads at once)
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, -1, 4 << 15);   // (data format 32 bits)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)to, 16, from, 0, 0, 0);
    }
  };
  auto x_slot = [&](int s) { return lds + s * kXBytes; };
  auto w_slot = [&](int s) { return lds + kSlots * kXBytes + s * kWBytes; };
  // Copy c of a wavefront's kCopies of a step: weights, then activations.
  constexpr int kCopiers = MI < 4 ? 4 : 8, kMyW = kCols / 8 / kCopiers, kMyX = kRows / 8 / kCopiers, kCopies = kMyW + kMyX;
  const int copier = wave & (kCopiers - 1);
  auto copy_one = [&](int c, int step, int slot, auto RAGGED) {
    if (c < kMyW) copy(wr, copier * kMyW + c, step, w_slot(slot) + (copier * kMyW + c) * 1024, RAGGED);
    else copy(xr, copier * kMyX + c - kMyW, step, x_slot(slot) + (copier * kMyX + c - kMyW) * 1024, RAGGED);
  };

  // scales: of the rows a byte each, 64 steps at a time in LDS (from memory they are a cache line each in every step); of the weights one
  // number (64 columns lie in one block)
  uint8_t* scales = lds + kSlots * (kXBytes + kWBytes);
  auto stage_scales = [&](int step) {
    for (int i = threadIdx.x; i < kRows * (kScaleSteps / 4); i += 64 * kWaves) {
      const int row = i / (kScaleSteps / 4), c = i % (kScaleSteps / 4) * 4;
      const uint8_t* from = a.xs + (int64_t)min(m0 + row, a.M - 1) * a.ld_xs + step + c;
      uint32_t v = 0;
      if (step + c + 4 <= a.blocks) {
        __builtin_memcpy(&v, from, 4);   // (rows may start at any byte)
      } else {
        for (int e = 0; e < a.blocks - step - c; ++e) v |= (uint32_t)from[e] << (8 * e);
      }
      *reinterpret_cast<uint32_t*>(scales + row * kScalePitch + c) = v;
    }
    for (int i = threadIdx.x; i < 2 * kScaleSteps; i += 64 * kWaves)   // of the weights: 128 columns each
      reinterpret_cast<float*>(scales + kRows * kScalePitch)[i] =
          a.ws[(int64_t)(min(n0 + i / kScaleSteps * kScaleBlock, a.N - 1) / kScaleBlock) * a.ld_ws + min(step + i % kScaleSteps, a.blocks - 1)];
  };
  const uint8_t* my_scales = scales + (wm * 32 * MI + l32) * kScalePitch;
  const float* my_ws = reinterpret_cast<const float*>(scales + kRows * kScalePitch) + (wn >> 1) * kScaleSteps;

  // operand reads: lane (row l32, half h) takes chunks 4 kk + 2 h and 4 kk + 2 h + 1 for MFMA kk of the block
  uint32_t operand_at = l32 * kScaleBlock + (((2 * h) ^ ((l32 ^ (l32 >> 3 & 1)) & 7)) * 16);   // of kk = 0; the others differ in bits 4 and 6
  auto operand = [&](const uint8_t* rows, int kk) {
    const uint32_t at = operand_at ^ (kk * 64);
    return operand8(*reinterpret_cast<const u32x4_t*>(rows + at), *reinterpret_cast<const u32x4_t*>(rows + (at ^ 16)));
  };

  f32x16_t acc[MI][2];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = zeros16();

  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  constexpr int kLastTile = MI - 1;
  int xs_now[MI];
  int third = 0;   // of step k, of three
  i32x8_t w[2][2], x[2][2];
  auto load_x = [&](int slot, int i) {
    const uint8_t* rows = x_slot(slot) + (wm * 32 * MI + i * 32) * kScaleBlock;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) x[i & 1][kk] = operand(rows, kk);
  };
  auto load_w = [&](int slot, int j) {
    const uint8_t* rows = w_slot(slot) + (wn * 64 + j * 32) * kScaleBlock;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) w[j][kk] = operand(rows, kk);
  };
  // Two MFMAs of a tile, and the result of the two before them goes into its accumulators: the matrix unit has work while the vector unit adds.
  float s = 0.f, s_before = 0.f, s_read = 0.f;   // of this step, the one before, the next (s_read: the same in all lanes, the others in scalar registers)
  f32x16_t before = zeros16();
  auto multiply = [&](int i, int j) {
    f32x16_t r = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[j][0], x[i & 1][0], zeros16(), 0, 0, 0, 0x7F7F7F7F, 0, xs_now[i]);
    r = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[j][1], x[i & 1][1], r, 0, 0, 0, 0x7F7F7F7F, 0, xs_now[i]);
    const int pi = j > 0 ? i : i > 0 ? i - 1 : kLastTile, pj = j > 0 ? 0 : 1;
    const float f = i == 0 && j == 0 ? s_before : s;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[pi][pj][e] = fmaf(before[e], f, acc[pi][pj][e]);
    before = r;
  };
  auto uniform = [](float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); };
  // Step k: its first operands were asked for in step k - 1.  Before its last tile of rows all its operands are in registers: a barrier there
  // frees its place, and shows that step k + 1 is in LDS.
  // (after the last step of those that are staged: another's, and read again when the next are)
  auto next_scale = [&](int k, int i) { xs_now[i] = my_scales[i * 32 * kScalePitch + (k + 1 - first) % kScaleSteps]; };
  auto one_step = [&](int k, auto AHEAD, auto RAGGED) {
    const int slot = kSlots == 2 ? (k - first) & 1 : third, next = kSlots == 2 ? slot ^ 1 : third == 2 ? 0 : third + 1;
    const bool turn = MI == 4 || ((k - first) & 1) == wave >> 2;   // to copy
    // (which of the three an eighth takes, and where operands lie, is formed in each step, not kept)
    asm volatile("" : "+v"(xr.at[0]), "+v"(xr.at[1]), "+v"(xr.at[2]), "+v"(wr.at[0]), "+v"(wr.at[1]), "+v"(wr.at[2]), "+v"(operand_at));
    __builtin_amdgcn_sched_barrier(0);
    load_w(slot, 1);
#pragma unroll
    for (int i = 1; i < MI; ++i) next_scale(k - 1, i);
    s = uniform(s_read);
#pragma unroll
    for (int i = 0; i < kLastTile; ++i) {
      load_x(slot, i + 1);
      multiply(i, 0);
      __builtin_amdgcn_sched_barrier(0);
      multiply(i, 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    // (products are not moved past the branch)
#pragma unroll
    for (int i = 0; i < kLastTile; ++i) asm volatile("" : "+v"(acc[i][0]), "+v"(acc[i][1]));
    if (kSlots == 2 || turn) wait_loads<0>();   // step k + 1 (of three steps the others' copies under way are of step k + 2)
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // A wavefront that issues copies waits for the path to LDS, which they keep busy for half a step.  In the largest blocks all eight copy, some before each of
    // the last two products, and the others' products go on meanwhile (2048 x 18432 x 7168, when it was tried, before other steps: 318 us, with one wavefront of a SIMD that copies in turn 340); in
    // smaller ones the barriers lie too close for that, and in turn is faster (256 x 8192 x 8192 in blocks of 128 rows: 74 us against 84).
    if constexpr (decltype(AHEAD)::value && MI < 4) {
      if (turn) {
#pragma unroll
        for (int c = 0; c < kCopies; ++c) copy_one(c, k + kSlots, slot, RAGGED);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    auto copy_some = [&](int from, int to) {
      if constexpr (decltype(AHEAD)::value && MI == 4) {
#pragma unroll
        for (int c = from; c < to; ++c) copy_one(c, k + kSlots, slot, RAGGED);
      }
    };
    if (kLastTile % 2 == 1) load_x(next, 0);
    copy_some(0, (kCopies + 1) / 2);
    multiply(kLastTile, 0);
    __builtin_amdgcn_sched_barrier(0);
    load_w(next, 0);
    copy_some((kCopies + 1) / 2, kCopies);
    multiply(kLastTile, 1);
    if (kLastTile % 2 == 0) load_x(next, 0);
    next_scale(k, 0);
    s_read = my_ws[(k + 1 - first) % kScaleSteps];
    s_before = s;
    third = next;
    __builtin_amdgcn_sched_barrier(0);
  };

  for (int step = first; step < min(first + kSlots, last); ++step) {
    if (MI < 4 && wave >> 2 != ((step - first) & 1)) continue;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) copy_one(c, step, step - first, yes);
  }
  int k = first;
  while (k < last) {
    const int until = min(k + kScaleSteps, last);   // the steps whose scales are staged next
    stage_scales(k);
    wait_loads<0>();
    lds_barrier();
    if (k == first) {
      load_x(0, 0);
      load_w(0, 0);
    }
    next_scale(k - 1, 0);
    s_read = my_ws[(k - first) % kScaleSteps];
    if (k == first) s_before = uniform(s_read);
    for (; k < until && k + kSlots + 1 < last; ++k) one_step(k, yes, no);
    for (; k < until && k + kSlots < last; ++k) one_step(k, yes, yes);
    for (; k < until; ++k) one_step(k, no, no);   // (in the last one the operands asked for are of no step: what lies in the place, unused)
    lds_barrier();   // the scales of these steps have been read
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[kLastTile][1][e] = fmaf(before[e], s_before, acc[kLastTile][1][e]);

  // register e of a lane: column 8 (e / 4) + 4 h + e % 4 of its tile, row l32
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int m = m0 + wm * 32 * MI + i * 32 + l32;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int n = n0 + wn * 64 + j * 32;
      if (p.shares > 1) {
        if (m < a.M) {
          float* out = a.partial + ((int64_t)share * a.M + m) * a.ld_partial;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int c = n + 8 * q + 4 * h;
            if (c < a.ld_partial) *reinterpret_cast<f32x4_t*>(out + c) = f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          }
        }
        continue;
      }
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        // halves exchange, so that a lane holds eight neighbouring columns
        u32x4_t v;
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const uint32_t even = pack_bf16(acc[i][j][4 * q + 2 * d], acc[i][j][4 * q + 2 * d + 1]), odd = pack_bf16(acc[i][j][4 * q + 4 + 2 * d], acc[i][j][4 * q + 5 + 2 * d]);
          const u32x2_t both = __builtin_amdgcn_permlane32_swap(even, odd, false, false);
          v[d] = both.x;
          v[2 + d] = both.y;
        }
        const int c = n + 8 * (q + h);
        if (m < a.M && c < a.N) {
          uint16_t* out = a.y + (int64_t)m * a.ldy + c;
          if (c + 8 <= a.N) {
            *reinterpret_cast<u32x4_t*>(out) = v;
          } else {
            for (int e = 0; e < a.N - c; ++e) out[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    }
  }
}

template <int MI>
int launch(const Gemm8Block& p, hipStream_t s) {
  constexpr int kLds = slots(MI) * (64 * MI * kScaleBlock + kWBytes) + 64 * MI * kScalePitch + 2 * kScaleSteps * 4;
  const void* kernel = reinterpret_cast<const void*>(ccq_gemm8_block_kernel<MI>);
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) return CCQ_ERR_HIP;
  const int per = (p.m_tiles * p.n_tiles + 7) / 8;
  hipLaunchKernelGGL((ccq_gemm8_block_kernel<MI>), dim3((unsigned)(8 * per * p.shares)), dim3(64 * kWaves), kLds, s, p);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace

// For tests, no part of the interface: what lane `lane` copies for eighth `eighth` of rows 0 .. last_row at column k: the offset of its 16 bytes, or -1 for zeros.
extern "C" int64_t ccq_gemm8_block_source(int32_t lane, int32_t eighth, int32_t last_row, int64_t ld, int32_t k, int32_t K) {
  const int end = last_row >> 3, sub = lane >> 3;
  if (block_past_k(lane, eighth, end, k, K)) return -1;
  const int64_t row = eighth >= end ? 8 * end + std::min(sub, last_row & 7) : 8 * eighth + sub;
  return row * ld + k + block_chunk(lane, std::min(eighth, end)) * 16;
}

int launch_gemm8_block(const Gemm8Args& a, int mi, int shares, void* stream) {
  Gemm8Block p;
  p.a = a;
  p.m_tiles = (a.M + 64 * mi - 1) / (64 * mi);
  p.n_tiles = (a.N + kCols - 1) / kCols;
  p.steps_per_share = (a.blocks + shares - 1) / shares;
  p.shares = (a.blocks + p.steps_per_share - 1) / p.steps_per_share;
  if ((int64_t)p.m_tiles * p.n_tiles * p.shares > most_groups(64 * kWaves)) return CCQ_ERR_UNSUPPORTED;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rc = mi == 4 ? launch<4>(p, s) : mi == 2 ? launch<2>(p, s) : launch<1>(p, s);
  if (rc != CCQ_OK) return rc;
  return p.shares > 1 ? launch_gemm8_add(a, p.shares, stream) : CCQ_OK;
}

}  // namespace ccq
