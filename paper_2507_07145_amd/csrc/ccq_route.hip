// A router's choice of experts.
//
// L lanes hold a row's logits, V each: expert i L + lane in value i.  Scores are formed in 64 bits (the card's vector units take 64-bit
// operations at the 32-bit rate), so that sums of scores and biases next to each other are told apart as exact arithmetic has them; the choice itself is then
// top_k times the largest that is left: every lane keeps its own best, the lanes of a row compare theirs with DPP moves, and the lane that held the largest looks for its
// next.  Without a bias the logits are compared, in 32 bits.
#include <cmath>

#include "ccq_order.h"

namespace ccq {

namespace {

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* ids;
  float* weights;
  int64_t ld;
  int32_t T, E, k;
  int32_t groups, top_groups, group_size, inv_group;   // inv_group = ceil(2^20 / group_size): e / group_size = e * inv_group >> 20 for e < 1024
  float scale;
  uint8_t fp32, sigmoid, two_best, renormalize;
};

// The lanes' exchanges of ccq_layer.h for values of 32 and 64 bits.
template <typename T, typename Move>
__device__ __forceinline__ T moved(T v, Move move) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, move(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(T, (uint64_t)move((uint32_t)(b >> 32)) << 32 | move((uint32_t)b));
  }
}

// f over the L lanes of a row, in all of them.
template <int L, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f) {
  v = f(v, moved(v, [](uint32_t u) { return ror16<8>(u); }));
  v = f(v, moved(v, [](uint32_t u) { return ror16<4>(u); }));
  v = f(v, moved(v, [](uint32_t u) { return ror16<2>(u); }));
  v = f(v, moved(v, [](uint32_t u) { return ror16<1>(u); }));
  if constexpr (L > 16) {
    v = f(v, moved(v, [](uint32_t u) { return xor16(u); }));
    v = f(v, moved(v, [](uint32_t u) { return xor32(u); }));
  }
  return v;
}

constexpr float kNone = -INFINITY;

// Logits as fp32 (bf16's are exact); what is not open is -infinity.
__device__ __forceinline__ float logit(const RouteArgs& a, int64_t at) {
  const float l = a.fp32 ? static_cast<const float*>(a.logits)[at] : bf16_lo(static_cast<const uint16_t*>(a.logits)[at]);
  return l == l ? l : kNone;
}

// exp(l - top), or the sigmoid; 0 for -infinity.
__device__ __forceinline__ double part(const RouteArgs& a, float l, float top) {
  if (a.sigmoid) return 1.0 / (1.0 + exp(-(double)l));
  return l == top && top > kNone ? 1.0 : l == kNone ? 0.0 : exp((double)l - (double)top);   // (infinity minus infinity would be NaN)
}

// What a workgroup's rows need in LDS where there are groups: values of all experts, values of the groups, which are kept.
int group_bytes(int rows, int E, int groups) { return rows * (E * 8 + groups * 8 + (groups + 7) / 8 * 8); }

// Closes the experts of groups that are not kept (keys become -infinity).  by: the values that groups are compared by.
template <int L, int V, typename Key>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, char* lds, int rows, int row, int sub, const double (&by)[V], Key (&key)[V]) {
  double* const values = reinterpret_cast<double*>(lds) + row * a.E;
  double* const sums = reinterpret_cast<double*>(lds) + rows * a.E + row * a.groups;
  uint8_t* const kept = reinterpret_cast<uint8_t*>(reinterpret_cast<double*>(lds) + rows * (a.E + a.groups)) + row * ((a.groups + 7) / 8 * 8);
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i * L + sub < a.E) values[i * L + sub] = by[i];
  __syncthreads();
  for (int g = sub; g < a.groups; g += L) {
    double best = -INFINITY, next = -INFINITY;
    int at = g % a.group_size;   // (lanes begin at different places of their groups: their reads meet different banks)
    for (int i = 0; i < a.group_size; ++i) {
      const double v = values[g * a.group_size + at];
      next = fmax(next, fmin(best, v));
      best = fmax(best, v);
      if (++at == a.group_size) at = 0;
    }
    sums[g] = a.two_best && next > -INFINITY ? best + next : best;
  }
  __syncthreads();
  for (int g = sub; g < a.groups; g += L) {
    const double mine = sums[g];
    int ahead = 0;
    for (int o = 0; o < a.groups; ++o) ahead += sums[o] > mine || (sums[o] == mine && o < g);
    kept[g] = ahead < a.top_groups;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = i * L + sub;
    if (e < a.E && !kept[e * a.inv_group >> 20]) key[i] = -INFINITY;
  }
}

// A row's choice: L lanes, V values each; Key: double with a bias, float without.  Returns this lane's places j = sub and sub + L of the row in id[0], id[1].
template <int L, int V, typename Key>
__device__ __forceinline__ void choose(const RouteArgs& a, char* lds, int rows, int row, int64_t t, int sub, int (&id)[2]) {
  const bool live = t < a.T;
  float l[V], top = kNone;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = i * L + sub;
    l[i] = live && e < a.E ? logit(a, t * a.ld + e) : kNone;
    top = fmaxf(top, l[i]);
  }
  top = over_lanes<L>(top, [](float x, float y) { return fmaxf(x, y); });
  const bool summed = !a.sigmoid && (sizeof(Key) == 8 || !a.renormalize || (a.groups > 1 && a.two_best));
  constexpr bool kWide = sizeof(Key) == 8;
  Key key[V];
  double total = 1.0;
  if (kWide || summed || a.groups > 1) {
    double s[V], sum = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s[i] = part(a, l[i], top);
      sum += s[i];
    }
    if (summed) total = over_lanes<L>(sum, [](double x, double y) { return x + y; });
    const double inverse = 1.0 / total;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int e = i * L + sub;
      const float bias = kWide && e < a.E ? a.bias[e] : 0.f;
      s[i] *= inverse;
      s[i] = l[i] > kNone && bias > kNone ? s[i] + (double)bias : -INFINITY;   // (a comparison with NaN is false)
      key[i] = kWide ? (Key)s[i] : (Key)l[i];
    }
    if (a.groups > 1) keep_groups<L, V, Key>(a, lds, rows, row, sub, s, key);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = (Key)l[i];
  }

  Key best = -INFINITY;
  int at = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (key[i] > best) best = key[i], at = i * L + sub;
  }
  id[0] = id[1] = -1;
  for (int r = 0; r < a.k; ++r) {
    const Key most = over_lanes<L>(best, [](Key x, Key y) { return x > y ? x : y; });
    const int won = over_lanes<L>(best == most ? at : 0x7FFFFFFF, [](int x, int y) { return min(x, y); });
    const int chosen = most > (Key)-INFINITY ? won : -1;
    if (r == sub) id[0] = chosen;
    if (L < kMostChosen && r == sub + L) id[1] = chosen;
    best = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i * L + sub == won) key[i] = -INFINITY;
      if (key[i] > best) best = key[i], at = i * L + sub;
    }
  }

  double w[2] = {0.0, 0.0};
#pragma unroll
  for (int j = 0; j < (L < kMostChosen ? 2 : 1); ++j)
    if (id[j] >= 0) w[j] = part(a, logit(a, t * a.ld + id[j]), top);
  if (a.renormalize) total = over_lanes<L>(w[0] + w[1], [](double x, double y) { return x + y; });
  if (!live) return;
#pragma unroll
  for (int j = 0; j < (L < kMostChosen ? 2 : 1); ++j) {
    const int place = sub + j * L;
    if (place >= a.k) continue;
    a.ids[t * a.k + place] = id[j];
    a.weights[t * a.k + place] = total > 0.0 ? (float)(w[j] / total * (double)a.scale) : 0.f;
  }
}

template <int L, int V, typename Key>
__global__ __launch_bounds__(256) void ccq_route_kernel(RouteArgs a) {
  extern __shared__ char lds[];
  constexpr int kRows = 256 / L;
  const int row = threadIdx.x / L;
  int id[2];
  choose<L, V, Key>(a, lds, kRows, row, (int64_t)blockIdx.x * kRows + row, threadIdx.x % L, id);
}

template <int L, int V, typename Key>
int launch(const RouteArgs& all, hipStream_t s) {
  constexpr int kRows = 256 / L;
  constexpr int64_t kMost = most_groups(256) * kRows;
  const int lds = all.groups > 1 ? group_bytes(kRows, all.E, all.groups) : 0;
  if (lds > 48 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(ccq_route_kernel<L, V, Key>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return CCQ_ERR_HIP;
  RouteArgs a = all;
  for (int64_t t = 0; t < all.T; t += kMost) {
    a.T = (int32_t)(all.T - t < kMost ? all.T - t : kMost);
    a.logits = static_cast<const char*>(all.logits) + t * all.ld * (all.fp32 ? 4 : 2);
    a.ids = all.ids + t * all.k, a.weights = all.weights + t * all.k;
    hipLaunchKernelGGL((ccq_route_kernel<L, V, Key>), dim3((unsigned)((a.T + kRows - 1) / kRows)), dim3(256), (size_t)lds, s, a);
  }
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

template <typename Key>
int launch_by_size(const RouteArgs& a, hipStream_t s) {
  if (a.E <= 64) return launch<16, 4, Key>(a, s);
  if (a.E <= 128) return launch<16, 8, Key>(a, s);
  if (a.E <= 256) return launch<16, 16, Key>(a, s);
  if (a.E <= 512) return launch<64, 8, Key>(a, s);
  return launch<64, 16, Key>(a, s);
}

}  // namespace

int64_t route_workspace(const ccq_router* r) { return sort_workspace(r->T, r->top_k, r->experts); }

int launch_route(const ccq_router* r, const ccq_order* order, void* workspace, void* stream) {
  RouteArgs a;
  a.logits = r->logits, a.bias = r->bias, a.ids = r->ids, a.weights = r->weights, a.ld = r->ld;
  a.T = r->T, a.E = r->experts, a.k = r->top_k;
  a.groups = r->groups, a.top_groups = r->top_groups, a.group_size = r->experts / r->groups;
  a.inv_group = ((1 << 20) + a.group_size - 1) / a.group_size;
  a.scale = r->scale;
  a.fp32 = r->logits_type == CCQ_FP32, a.sigmoid = r->scoring == CCQ_SIGMOID, a.two_best = r->group_best == 2, a.renormalize = r->renormalize != 0;
  if (a.top_groups == a.groups) a.groups = a.top_groups = 1;   // (all of them stay)
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rc = a.T == 0 ? CCQ_OK : a.bias ? launch_by_size<double>(a, s) : launch_by_size<float>(a, s);
  if (rc != CCQ_OK || !order) return rc;
  return launch_sort(r->ids, r->top_k, r->T, r->top_k, 0, r->experts, order, workspace, stream);
}

}  // namespace ccq
