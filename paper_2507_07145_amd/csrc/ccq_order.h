// The order of entries by expert: a counting sort that keeps the entries of one expert in their order and uses no atomic whose order counts.
//
// A workgroup's entries are cut into one stretch for each wavefront, and wavefronts count in LDS, each for itself: 64 entries at a time, lanes with the same
// expert find each other by one ballot per bit of it, the lowest of them adds their number.  Sums over the wavefronts, then over the experts, make
// the first place of each wavefront's share of each expert; a second pass over the same entries hands the places out.  Bound by the latency of these
// steps, not by memory.
#pragma once
#include "ccq_routing.h"

namespace ccq {

struct SortArgs {
  const int32_t* ids;
  int64_t ld_ids;
  uint32_t* counts;    // [workgroups][E + 1] of the workspace: entries of each expert, where there are several workgroups
  int32_t *rows, *experts, *offsets, *places;
  int32_t P, k, first, E;
  int32_t chunk;       // entries of a workgroup
  int32_t stretch;     // of a wavefront, a multiple of 64
  int32_t bits;        // of an expert's number, E itself (none) among them
};

// Lanes of `active` whose expert is this lane's.
__device__ __forceinline__ uint64_t peers_of(uint32_t e, int bits, uint64_t active) {
  uint64_t same = active;
  for (int b = 0; b < bits; ++b) {
    const uint64_t with = __ballot((e >> b) & 1);
    same &= (e >> b) & 1 ? with : ~with;
  }
  return same;
}

__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Adds the 64 entries from `i0` on to the wavefront's counters; returns what this lane's expert had before, entries of lower lanes included.
template <typename Expert>
__device__ __forceinline__ uint32_t count_64(uint32_t* mine, int i0, int end, int bits, const Expert& expert, uint32_t* e_out) {
  const int lane = threadIdx.x & 63, i = i0 + lane;
  const bool in = i < end;
  const uint32_t e = in ? expert(i) : 0;
  const uint64_t same = peers_of(e, bits, __ballot(in));
  const int leader = __builtin_ctzll(same | (1ull << lane));   // (lanes past the end lead themselves, and add nothing)
  uint32_t had = 0;
  if (in && leader == lane) had = atomicAdd(mine + e, (uint32_t)__builtin_popcountll(same));
  had = (uint32_t)__shfl((int)had, leader);
  *e_out = e;
  return had + (uint32_t)lanes_below(same);
}

// LDS words that sort_entries needs.
inline __host__ __device__ int sort_words(int waves, int E) { return (waves + 1) * (E + 1); }

// All threads of a workgroup of `waves` wavefronts: the entries [begin, end), expert(i) 0 .. E (E: none).  `mine_of_all`: with several
// workgroups their counts, this one's number and how many there are.
template <typename Expert>
__device__ __forceinline__ void sort_entries(const SortArgs& a, uint32_t* lds, int waves, int begin, int end, const Expert& expert, const uint32_t* all_counts, int block,
                                             int blocks) {
  const int E1 = a.E + 1, tid = threadIdx.x, threads = waves * 64, wave = tid >> 6;
  uint32_t* const mine = lds + wave * E1;
  uint32_t* const total = lds + waves * E1;
  const int64_t from64 = (int64_t)begin + (int64_t)wave * a.stretch, to64 = from64 + a.stretch;
  const int from = (int)min(from64, (int64_t)end), to = (int)min(to64, (int64_t)end);
  for (int i = tid; i < waves * E1; i += threads) lds[i] = 0;
  __syncthreads();
  uint32_t e;
  for (int i = from; i < to; i += 64) count_64(mine, i, to, a.bits, expert, &e);
  __syncthreads();
  for (int x = tid; x < E1; x += threads) {
    uint32_t below = 0, all = 0;
    for (int b = 0; b < blocks && all_counts; ++b) {
      const uint32_t c = all_counts[(int64_t)b * E1 + x];
      if (b < block) below += c;
      all += c;
    }
    uint32_t sum = below;
    for (int w = 0; w < waves; ++w) {
      const uint32_t c = lds[w * E1 + x];
      lds[w * E1 + x] = sum;
      sum += c;
    }
    total[x] = all_counts ? all : sum;
  }
  __syncthreads();
  if (wave == 0) {   // sums over the experts before each
    uint32_t before = 0;
    for (int x0 = 0; x0 < E1; x0 += 64) {
      const int x = x0 + tid;
      const uint32_t c = x < E1 ? total[x] : 0;
      uint32_t sum = c;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = (uint32_t)__shfl_up((int)sum, d);
        if (tid >= d) sum += other;
      }
      if (x < E1) {
        total[x] = before + sum - c;
        if (block == 0) a.offsets[x] = (int32_t)(before + sum - c);
      }
      before += (uint32_t)__shfl((int)sum, 63);
    }
  }
  __syncthreads();
  for (int i0 = from; i0 < to; i0 += 64) {
    const uint32_t at = count_64(mine, i0, to, a.bits, expert, &e);
    const int i = i0 + (tid & 63);
    if (i >= to) continue;
    const int32_t p = (int32_t)(total[e] + at);
    const bool has = e < (uint32_t)a.E;
    a.rows[p] = i / a.k;
    if (a.experts) a.experts[p] = has ? (int32_t)e : -1;
    if (a.places) a.places[i] = has ? p : -1;
  }
}

inline int bits_of(int E) {
  int bits = 1;
  while (E >> bits) ++bits;
  return bits;
}

}  // namespace ccq
