// The order of ids by expert (ccq_order.h has the sort): one workgroup for few entries; several, each of which counts all of them; for many one launch that counts each workgroup's
// share and one that places it.  Alone 200 entries of 128 experts take 2.5 us; in a graph's steps 3066 of 160 take 4.8, 131072 of 8 7.1, of 256 11.9 us.
#include "ccq_order.h"

namespace ccq {

namespace {

struct FromIds {
  const int32_t* ids;
  int64_t ld;
  Divisor k;
  int first, E;
  __device__ __forceinline__ uint32_t operator()(int i) const {
    int64_t at = i;
    if (ld != k.by) {
      const int t = k.divide(i);
      at = (int64_t)t * ld + (i - t * k.by);
    }
    const int32_t id = ids[at];
    return id >= first && id - first < E ? (uint32_t)(id - first) : (uint32_t)E;
  }
};

__global__ __launch_bounds__(1024) void ccq_sort_count_kernel(SortArgs a) {
  extern __shared__ uint32_t lds[];
  const int E1 = a.E + 1;
  for (int x = threadIdx.x; x < E1; x += blockDim.x) lds[x] = 0;
  __syncthreads();
  const int64_t begin = (int64_t)blockIdx.x * a.chunk;
  const int end = (int)min(begin + a.chunk, (int64_t)a.P);
  const FromIds expert{a.ids, a.ld_ids, a.k, a.first, a.E};
  for (int64_t i = begin + threadIdx.x; i < end; i += blockDim.x) atomicAdd(lds + expert((int)i), 1u);
  __syncthreads();
  for (int x = threadIdx.x; x < E1; x += blockDim.x) a.counts[(int64_t)blockIdx.x * E1 + x] = lds[x];
}

template <int ROUNDS>
__global__ __launch_bounds__(1024) void ccq_sort_kernel(SortArgs a) {
  extern __shared__ uint32_t lds[];
  const int64_t begin = (int64_t)blockIdx.x * a.chunk;
  const int end = (int)min(begin + a.chunk, (int64_t)a.P);
  sort_entries<ROUNDS>(a, lds, blockDim.x >> 6, (int)begin, end, FromIds{a.ids, a.ld_ids, a.k, a.first, a.E}, a.counts, blockIdx.x, gridDim.x);
}

// One workgroup up to 1024 entries (2048 of 8 and 256 experts take 4.3 and 5.5 us in one, 4.1 and 4.8 in four), then workgroups of 512 and more: 0.5 us less than 1024.  Each counts
// all entries up to 8192 (of 8 and 256 experts 5.2 and 5.5 us, with a launch that counts 5.9 and 7.1; 16384 6.9 and 6.6, and 5.9 and 7.8), and beyond adds up the counts of all,
// so that there may be as many as P entries and E experts make worth it: 131072 entries of 1024 experts take 20.6 us with 64 workgroups and 26.1 with 128, 2^21 of 256 94 us
// with 64, 57 with 128, 39 with 256.
constexpr int kOneBlock = 1024, kCounted = 8192, kChunk = 512, kMostBlocks = 256, kLeastBlocks = 32;

int blocks_of(int64_t P, int E) {
  if (P <= kOneBlock) return 1;
  int most = kMostBlocks;
  while (most > kLeastBlocks && (int64_t)most * most * E > 32 * P) most /= 2;
  const int64_t n = (P + kChunk - 1) / kChunk;
  return (int)(n > most ? most : n);
}

// As many wavefronts as have 64 entries or 64 experts each, and their counters in 56 KB of LDS.
int waves_of(int E, int chunk) {
  const int work = chunk > E + 1 ? chunk : E + 1;
  int waves = 16;
  while (waves > 1 && (sort_words(waves, E) * 4 > 56 * 1024 || (waves - 1) * 64 >= work)) waves /= 2;
  return waves;
}

}  // namespace

int64_t sort_workspace(int T, int k, int experts) {
  const int64_t P = (int64_t)T * k;
  return P > kCounted ? (int64_t)blocks_of(P, experts) * (experts + 1) * 4 : 0;
}

int launch_sort(const int32_t* ids, int64_t ld_ids, int T, int k, int first, int experts, const ccq_order* order, void* workspace, void* stream) {
  SortArgs a;
  a.ids = ids, a.ld_ids = ld_ids;
  a.rows = order->rows, a.experts = order->experts, a.offsets = order->offsets, a.places = order->places;
  a.P = T * k, a.k = Divisor(k), a.first = first, a.E = experts;
  const int blocks = blocks_of(a.P, experts);
  a.chunk = (int)(((int64_t)a.P + blocks - 1) / blocks);
  const bool counted = a.P > kCounted;
  a.counts = counted ? static_cast<uint32_t*>(workspace) : nullptr;
  const int waves = waves_of(experts, blocks > 1 && !counted ? a.P : a.chunk);
  a.stretch = (int)((((int64_t)a.chunk + waves - 1) / waves + 63) / 64 * 64);
  a.bits = bits_of(experts);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (counted) hipLaunchKernelGGL(ccq_sort_count_kernel, dim3(blocks), dim3(a.chunk < 1024 ? (a.chunk + 63) / 64 * 64 : 1024), (size_t)(experts + 1) * 4, s, a);
  const auto sort = a.stretch <= 64 ? ccq_sort_kernel<1> : a.stretch <= 128 ? ccq_sort_kernel<2> : a.stretch <= 256 ? ccq_sort_kernel<4> : a.stretch <= 512 ? ccq_sort_kernel<8> : ccq_sort_kernel<0>;
  hipLaunchKernelGGL(sort, dim3(blocks), dim3(waves * 64), (size_t)sort_words(waves, experts) * 4, s, a);
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

}  // namespace ccq
