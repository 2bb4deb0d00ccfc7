// The order of entries by expert: a counting sort that keeps the entries of one expert in their order and uses no atomic whose order counts.
//
// A workgroup's entries are cut into one stretch for each wavefront, and wavefronts count in LDS, each for itself: 64 entries at a time, lanes with the same
// expert find each other by one ballot per bit of it, the lowest of them adds their number.  Sums over the wavefronts, then over the experts, make
// the first place of each wavefront's share of each expert; a second pass over the same entries hands the places out.  Bound by the latency of these
// steps, not by memory.
#pragma once
#include <type_traits>

#include "ccq_routing.h"

namespace ccq {

// Division of numbers below 2^31 by one that is known on the host: with s bits in by - 1, the upper half of n ceil(2^(31 + s) / by), shifted by s - 1.
struct Divisor {
  int32_t by = 1, shift = 0;
  uint32_t factor = 0;
  Divisor() = default;
  explicit Divisor(int by_) : by(by_) {
    int s = 0;
    while ((by - 1) >> s) ++s;
    if (s == 0) return;
    shift = s - 1;
    factor = (uint32_t)(((1ull << (31 + s)) + by - 1) / by);
  }
  __device__ __forceinline__ int divide(int n) const { return by == 1 ? n : (int)(__umulhi((uint32_t)n, factor) >> shift); }
};

struct SortArgs {
  const int32_t* ids;
  int64_t ld_ids;
  uint32_t* counts;    // [workgroups][E + 1] of the workspace: entries of each expert, where there are several workgroups
  int32_t *rows, *experts, *offsets, *places;
  Divisor k;
  int32_t P, first, E;
  int32_t chunk;       // entries of a workgroup
  int32_t stretch;     // of a wavefront, a multiple of 64
  int32_t bits;        // of an expert's number, E itself (none) among them
};

// Lanes of `active` whose expert is this lane's.
__device__ __forceinline__ uint64_t peers_of(uint32_t e, int bits, uint64_t active) {
  uint32_t lo = (uint32_t)active, hi = (uint32_t)(active >> 32);
  for (int b = 0; b < bits; ++b) {
    const uint32_t mine = (uint32_t)__builtin_amdgcn_sbfe((int)e, b, 1);   // all ones or none
    const uint64_t with = __ballot(mine != 0);
    lo &= ~((uint32_t)with ^ mine);
    hi &= ~((uint32_t)(with >> 32) ^ mine);
  }
  return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Adds 64 entries to the wavefront's counters, those of the lanes that are `in`.  What a lane's expert had before is had of lane `leader` and the returned lanes below this one.
__device__ __forceinline__ uint64_t add_64(uint32_t* mine, uint32_t e, bool in, int bits, uint32_t* had, uint32_t* leader) {
  const int lane = threadIdx.x & 63;
  const uint64_t same = peers_of(e, bits, __ballot(in));
  *leader = (uint32_t)__builtin_ctzll(same | (1ull << lane));   // (lanes past the end lead themselves, and add nothing)
  *had = 0;
  if (in && *leader == (uint32_t)lane) *had = atomicAdd(mine + e, (uint32_t)__builtin_popcountll(same));
  return same;
}
template <typename Expert>
__device__ __forceinline__ uint32_t count_64(uint32_t* mine, int i0, int end, int bits, const Expert& expert, uint32_t* e) {
  const int i = i0 + (threadIdx.x & 63);
  uint32_t had, leader;
  *e = i < end ? expert(i) : 0;
  const uint64_t same = add_64(mine, *e, i < end, bits, &had, &leader);
  return (uint32_t)__shfl((int)had, (int)leader) + (uint32_t)lanes_below(same);
}

// LDS words that sort_entries needs.
inline __host__ __device__ int sort_words(int waves, int E) { return (waves + 2) * (E + 1) + 66; }

// Sum of v over the lanes up to this one, by moves between lanes.
__device__ __forceinline__ uint32_t up_to_lane(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);   // from one lane, two, four and eight below, within 16
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);   // the last lane of 16 to the next 16, of 32 to the next 32
  return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);
}

// All threads of a workgroup of `waves` wavefronts: the entries [begin, end), expert(i) 0 .. E (E: none).  With several workgroups `all_counts` are their
// counts, `block` is this one's number; where there are none each counts all entries.  ROUNDS > 0: a stretch has at most 64 ROUNDS entries, which stay in registers between the passes.
template <int ROUNDS, typename Expert>
__device__ __forceinline__ void sort_entries(const SortArgs& a, uint32_t* lds, int waves, int begin, int end, const Expert& expert, const uint32_t* all_counts, int block,
                                             int blocks) {
  const bool counts_others = blocks > 1 && !all_counts;
  const int E1 = a.E + 1, tid = threadIdx.x, threads = waves * 64, wave = tid >> 6, lane = tid & 63;
  uint32_t* const mine = lds + wave * E1;
  uint32_t* const total = lds + waves * E1;
  uint32_t* const below = total + E1;
  uint32_t* const parts = below + E1;   // sums of 64 experts each
  const int64_t from64 = (int64_t)begin + (int64_t)wave * a.stretch, to64 = from64 + a.stretch;
  const int from = (int)min(from64, (int64_t)end), to = (int)min(to64, (int64_t)end);
  constexpr int kKept = ROUNDS > 0 ? ROUNDS : 1;
  uint32_t e[kKept];
  if constexpr (ROUNDS > 0) {   // all are on their way before the first is needed (past the end the last one again)
    if (a.P > 0) {
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) e[r] = expert(min(from + 64 * r + lane, a.P - 1));
    }
  }
  for (int i = tid; i < (waves + 2) * E1; i += threads) lds[i] = 0;
  __syncthreads();
  if (all_counts) {   // as many threads to an expert as there are, each with every n-th workgroup's counts
    const int n = max(1, threads / E1);
    for (int x = tid % min(E1, threads); x < E1; x += threads) {
      uint32_t sum = 0, before = 0;
      const int b0 = tid / min(E1, threads);
      if (b0 >= n) break;
      auto add = [&](int b1, auto most) {   // so many at once; past the last workgroup the last one's again, which do not count
        uint32_t c[most.value];
#pragma unroll
        for (int j = 0; j < most.value; ++j) c[j] = all_counts[(int64_t)min(b1 + j * n, blocks - 1) * E1 + x];
#pragma unroll
        for (int j = 0; j < most.value; ++j) {
          const int b = b1 + j * n;
          before += b < block ? c[j] : 0;
          sum += b < blocks ? c[j] : 0;
        }
      };
      int b = b0;
      for (; b + 4 * n < blocks; b += 16 * n) add(b, std::integral_constant<int, 16>());
      for (; b < blocks; b += 4 * n) add(b, std::integral_constant<int, 4>());
      atomicAdd(total + x, sum);
      atomicAdd(below + x, before);
    }
  }
  if (counts_others) {   // total: the entries from this workgroup's first on
    constexpr int kAtOnce = 8;
    for (int i0 = tid; i0 < a.P; i0 += kAtOnce * threads) {
      uint32_t of[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) of[j] = expert(min(i0 + j * threads, a.P - 1));
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int i = i0 + j * threads;
        if (i < a.P) atomicAdd((i < begin ? below : total) + of[j], 1u);
      }
    }
  }
  uint32_t kept[kKept];   // expert << 16 | entries of the stretch before this one with the same
  if constexpr (ROUNDS > 0) {
    uint32_t had[kKept], leaders[kKept];
    uint64_t same[kKept];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) same[r] = add_64(mine, e[r], from + 64 * r + lane < to, a.bits, &had[r], &leaders[r]);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) kept[r] = e[r] << 16 | ((uint32_t)__shfl((int)had[r], (int)leaders[r]) + (uint32_t)lanes_below(same[r]));
  } else {
    for (int i = from; i < to; i += 64) count_64(mine, i, to, a.bits, expert, &e[0]);
  }
  __syncthreads();
  // the entries of each expert before each wavefront's, and of the experts before: sums within 64 experts first
  for (int x0 = wave * 64; x0 < E1; x0 += threads) {
    const int x = x0 + lane;
    uint32_t all = 0;
    if (x < E1) {
      uint32_t sum = below[x];
      all = counts_others ? total[x] + sum : total[x];
      for (int w = 0; w < waves; ++w) {
        const uint32_t c = lds[w * E1 + x];
        lds[w * E1 + x] = sum;
        sum += c;
      }
      if (blocks == 1) all = sum;
    }
    const uint32_t upto = up_to_lane(all);
    if (x < E1) total[x] = upto - all;
    if (lane == 63) parts[x0 / 64] = upto;
  }
  __syncthreads();
  for (int x0 = wave * 64; x0 < E1; x0 += threads) {
    const int x = x0 + lane;
    const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)up_to_lane(lane < x0 / 64 ? parts[lane] : 0), 63);
    if (x < E1) {
      total[x] += before;
      if (block == 0) a.offsets[x] = (int32_t)total[x];
    }
  }
  __syncthreads();
  auto place = [&](int i, uint32_t e, uint32_t at) {
    const int32_t p = (int32_t)(total[e] + at);
    const bool has = e < (uint32_t)a.E;
    a.rows[p] = a.k.divide(i);
    if (a.experts) a.experts[p] = has ? (int32_t)e : -1;
    if (a.places) a.places[i] = has ? p : -1;
  };
  if constexpr (ROUNDS > 0) {
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const int i = from + 64 * r + lane;
      if (i < to) place(i, kept[r] >> 16, mine[kept[r] >> 16] + (kept[r] & 0xFFFF));
    }
  } else {   // the counters go on from where each stretch's entries begin
    for (int i0 = from; i0 < to; i0 += 64) {
      const uint32_t at = count_64(mine, i0, to, a.bits, expert, &e[0]);
      if (i0 + lane < to) place(i0 + lane, e[0], at);
    }
  }
}

inline int bits_of(int E) {
  int bits = 1;
  while (E >> bits) ++bits;
  return bits;
}

}  // namespace ccq
