// A router's choice of experts.
//
// L lanes hold a row's logits, V each: expert i L + lane in value i.  The choice is top_k times the largest that is left: every lane keeps its own best, the lanes of a row
// compare theirs with DPP moves, and the lane that held the largest looks for its next.  Scores next to each other have to be told apart as exact arithmetic has
// them: the choice is made in 32 bits where these leave no doubt, and else in 64.
// One row of 64, with its order: 4.8 us; 64 rows of 256 with groups 7.0, 511 of 160 6.9: the latency of k rounds that wait for each other.  16384 rows of 256 with groups 19.4 us: vector
// instructions, 1680 a wavefront (3.8 for the bytes alone).
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

__device__ __forceinline__ float max_of(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ double max_of(double x, double y) { return fmax(x, y); }
__device__ __forceinline__ float abs_of(float x) { return fabsf(x); }
__device__ __forceinline__ double abs_of(double x) { return fabs(x); }
__device__ __forceinline__ float min_of(float x, float y) { return fminf(x, y); }
__device__ __forceinline__ double min_of(double x, double y) { return fmin(x, y); }

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

// The sum of a row's values, f(i) that of expert i L + sub: the same additions in the same order for 16 lanes and for 64, so that it does not depend on how many rows there are.
template <int L, int V, typename F>
__device__ __forceinline__ double row_sum(F f) {
  double sum[4] = {0.0, 0.0, 0.0, 0.0};   // of 64 experts, those of sub % 16 + 16 j
#pragma unroll
  for (int i = 0; i < V; ++i) sum[L == 16 ? i % 4 : 0] += f(i);
  if constexpr (L == 16) {
    sum[0] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  } else {
    sum[0] += moved(sum[0], [](uint32_t u) { return xor16(u); });
    sum[0] += moved(sum[0], [](uint32_t u) { return xor32(u); });
  }
  return over_lanes<16>(sum[0], [](double x, double y) { return x + y; });
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

// Orders a wavefront's LDS writes before its lanes' reads: a row's lanes are of one wavefront, whose LDS accesses are done in their order.
__device__ __forceinline__ void wave_lds() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What a row needs in LDS where there are groups: values of all experts, values of the groups, which are kept.
__host__ __device__ inline int padded(int e) { return e + (e >> 5); }   // (groups of 32 begin in different banks)
__host__ __device__ inline int group_bytes(int E, int groups) { return (padded(E) + groups) * 8 + (groups + 7) / 8 * 8; }

// Lanes of a row for each group: a power of two, so that they meet by the moves of over_lanes.
template <int L>
__device__ __forceinline__ int lanes_of_group(int groups) {
  int q = L;
  while (q > 1 && q * groups > L) q /= 2;
  return q;
}

// Logits whose scores may be the same in 64 bits though they are not: both above 20 or 600 below (1 + e^-l is rounded, or e^l or e^(l - top) lost), or nearer to each other than
// 2^-30, as logits of less than 2^-7 can be.  Of others the scores are some 2^-48 apart at least, of 1 or, below 0, of themselves.
struct Meeting {
  float lo, hi;
  __device__ __forceinline__ Meeting(const RouteArgs& a, float top) : lo(a.sigmoid ? -600.f : top - 600.f), hi(a.sigmoid ? 20.f : INFINITY) {}
  __device__ __forceinline__ bool may(float x) const { return x > -INFINITY && (x >= hi || x <= lo || fabsf(x) < 0x1p-6f); }   // (with one of which this holds too)
  __device__ __forceinline__ bool operator()(float x, float y) const { return !(fabsf(fminf(fmaxf(x, lo), hi) - fminf(fmaxf(y, lo), hi)) >= 0x1p-30f); }
};

// Closes the experts of groups that are not kept (keys become -infinity).  by: the values that groups are compared by.  Returns by how much the last group kept is
// ahead of the first that is not, less `off` and what 2^-21 of the largest numbers that were added comes to.  Of logits (LOGITS) it is -1 in a lane that finds two groups
// whose scores may be the same, else 1.
template <int L, int V, bool LOGITS, typename Key, typename Value>
__device__ __forceinline__ Value keep_groups(const RouteArgs& a, char* lds, int sub, const Value (&by)[V], Key (&key)[V], Value off, Meeting meet) {
  Value* const values = reinterpret_cast<Value*>(lds);
  Value* const sums = reinterpret_cast<Value*>(lds + padded(a.E) * 8);
  uint8_t* const kept = reinterpret_cast<uint8_t*>(lds + (padded(a.E) + a.groups) * 8);
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i * L + sub < a.E) values[padded(i * L + sub)] = by[i];
  wave_lds();
  const int q = lanes_of_group<L>(a.groups), mine = sub & (q - 1);
  Value size = 0;
  for (int g0 = 0; g0 < a.groups; g0 += L / q) {
    const int g = g0 + sub / q;
    Value best = -INFINITY, next = -INFINITY;
    if (g < a.groups) {
#pragma unroll 4
      for (int at = mine; at < a.group_size; at += q) {
        const Value v = values[padded(g * a.group_size + at)];
        next = max_of(next, min_of(best, v));
        best = max_of(best, v);
      }
    }
    auto join = [&](int lanes, auto move) {
      if (q <= lanes) return;
      const Value b = moved(best, move), n = moved(next, move);
      next = max_of(max_of(next, n), min_of(best, b));
      best = max_of(best, b);
    };
    join(1, [](uint32_t u) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0xB1, 0xF, 0xF, false); });    // lane l ^ 1
    join(2, [](uint32_t u) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x4E, 0xF, 0xF, false); });    // l ^ 2
    join(4, [](uint32_t u) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x141, 0xF, 0xF, false); });   // the other four of eight
    join(8, [](uint32_t u) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, 0x140, 0xF, 0xF, false); });   // the other eight of 16
    if constexpr (L > 16) {
      join(16, [](uint32_t u) { return xor16(u); });
      join(32, [](uint32_t u) { return xor32(u); });
    }
    size = max_of(size, max_of(best > (Value)-INFINITY ? abs_of(best) : 0, next > (Value)-INFINITY ? abs_of(next) : 0));
    if (g < a.groups && mine == 0) sums[g] = a.two_best && next > (Value)-INFINITY ? best + next : best;
  }
  wave_lds();
  Value least = INFINITY, most = -INFINITY;   // of the groups that are kept, of the others
  bool met = false;
  for (int g = sub; g < a.groups; g += L) {
    const Value own = sums[g];
    int ahead = 0;
    for (int o = 0; o < a.groups; ++o) ahead += sums[o] > own || (sums[o] == own && o < g);
    if constexpr (LOGITS) {
      if (meet.may(own))   // (as good as never: 0.2 us of 6.8 for 511 rows of eight groups, with all pairs looked at 0.8)
        for (int o = 0; o < a.groups; ++o) met |= sums[o] != own && meet(sums[o], own);
    }
    kept[g] = ahead < a.top_groups;
    if (ahead < a.top_groups) least = min_of(least, own);
    else most = max_of(most, own);
  }
  wave_lds();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = i * L + sub;
    if (e < a.E && !kept[e * a.inv_group >> 20]) key[i] = -INFINITY;
  }
  if constexpr (LOGITS) return met ? -1.f : 1.f;
  least = over_lanes<L>(least, [](Value x, Value y) { return min_of(x, y); });
  most = over_lanes<L>(most, [](Value x, Value y) { return max_of(x, y); });
  size = over_lanes<L>(size, [](Value x, Value y) { return max_of(x, y); });
  return most == (Value)-INFINITY ? (Value)INFINITY : least - most - (off + size * (Value)0x1p-21);   // (NaN with infinities on both sides)
}

// The k largest keys of a row, the largest first, equal ones by the lower index; winners go to `out` in LDS, -1 where there are no more.
template <int L, int V, typename Key>
__device__ __forceinline__ void largest(const RouteArgs& a, int sub, Key (&key)[V], int32_t* out) {
  Key best = -INFINITY;
  int at = 0;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (key[i] > best) best = key[i], at = i * L + sub;
  for (int r = 0; r < a.k; ++r) {
    const Key most = over_lanes<L>(best, [](Key x, Key y) { return max_of(x, y); });
    const int won = over_lanes<L>(best == most ? at : 0x7FFFFFFF, [](int x, int y) { return min(x, y); });
    if (sub == 0) out[r] = most > (Key)-INFINITY ? won : -1;
    best = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (i * L + sub == won) key[i] = -INFINITY;
      if (key[i] > best) best = key[i], at = i * L + sub;
    }
  }
}

// The same on keys of 28 bits, one winner after the other: a number's bits in an order that integers have too, its lowest four replaced by V - 1 - i, so that of a
// lane's equal ones the lowest index is the largest and no two are the same (-0 + 0 is 0).  A lane's next best is the largest below its last: one subtraction and half a minimum
// for each value.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return __builtin_bit_cast(float, k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u)); }

template <int L, int V>
struct Picker {
  static_assert(V <= 16, "four bits for a lane's values");
  uint32_t key[V], best = 0, limit = 0xFFFFFFFFu;
  uint64_t row;   // its lanes of the wavefront
  __device__ __forceinline__ explicit Picker(const float (&value)[V]) {
    row = L == 64 ? ~0ull : 0xFFFFull << (threadIdx.x & 48);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      key[i] = value[i] > kNone ? (ordered(value[i] + 0.f) & ~15u) | (uint32_t)(15 - i) : 0;
      best = max(best, key[i]);
    }
  }
  // The next winner's index to `out` (-1: there is none); returns its key.
  __device__ __forceinline__ uint32_t next(int sub, int32_t* out) {
    const uint32_t most = over_lanes<L>(best, [](uint32_t x, uint32_t y) { return max(x, y); });
    const bool mine = best == most && lanes_below(__ballot(best == most) & row) == 0;   // (of equal ones, which have the same i, the lowest lane)
    if (mine) *out = most ? (int)(15 - (most & 15)) * L + sub : -1;
    limit = mine ? most : limit;
    uint32_t least = 0xFFFFFFFFu;
#pragma unroll
    for (int i = 0; i < V; ++i) least = min(least, limit - 1 - key[i]);   // (those that are not below wrap)
    best = least < limit ? limit - 1 - least : 0;
    return most;
  }
};
__device__ __forceinline__ float number(uint32_t key) { return key ? unordered(key & ~15u) : kNone; }
// Whether a number is ahead of a later one by more than `off` and 2^-18 of both, which the four bits and roundings may have cost.  No number is behind all.
__device__ __forceinline__ bool ahead_by(float one, float later, float off) { return !(later > kNone) || one - later > off + (fabsf(one) + fabsf(later)) * 0x1p-18f; }

// Scores in 32 bits, and how far they may be off.  2^x and 1 / x are right to one step (2^-23 of themselves).  The exponent l log2 e is off by 2^-24 of itself and the constant's
// 2^-26, which makes e^-l off by 2^-23.6 |l|, and |l| s (1 - s) is at most 0.224; with 2^x's own step and the sum's and the reciprocal's roundings a sigmoid
// is off by less than 2.5e-7.  For the softmax the same holds of each part (x e^-x is at most 0.37), and its sum of up to 1024 terms (64 lanes' sums of 16) is off by 22 roundings of 2^-24 more.
constexpr float kSigmoidOff = 2.5e-7f, kSoftmaxOff = 2.5e-6f;
constexpr int kMore = 4;   // further candidates where the order of the first is not sure

__device__ __forceinline__ float part32(const RouteArgs& a, float l, float top) {
  constexpr float kLog2e = 1.44269504f;
  if (a.sigmoid) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-l * kLog2e));
  return l == top && top > kNone ? 1.f : l == kNone ? 0.f : __builtin_amdgcn_exp2f((l - top) * kLog2e);
}

// A row's winners in LDS, and the bytes it needs there otherwise: what groups need, or the numbers in 64 bits that decide an order.
constexpr int kPlaces = kMostChosen + kMore;
__host__ __device__ inline int row_bytes(int E, int groups) { return groups > 1 && group_bytes(E, groups) > 8 * kPlaces ? group_bytes(E, groups) : 8 * kPlaces; }

// A row's choice: L lanes, V values each, whose experts i L + sub are open where l[i] is more than -infinity; BIAS: with one.  `lds`: row_bytes for the row.
//
// The choice is the one that 64-bit scores make, or the logits themselves.  It is made on fewer bits first.  Where every winner is ahead of the next by more than
// these may be off, it is that already; where not, kMore candidates further on the last one mostly is behind all by that much, and their numbers in 64 bits, one to a
// lane, set them in order.  Equal numbers in a row (and groups that are as near, for their choice) have all values formed in 64 bits: a row in thousands, unless
// logits and biases are the same.  Groups that are compared by their best logits need no scores, but where two of these may be equal although the logits are not.
template <int L, int V, bool BIAS>
__device__ __forceinline__ void choose(const RouteArgs& a, char* lds, int32_t (&chosen)[kPlaces], int64_t t, int sub) {
  const bool live = t < a.T;
  float l[V], bias[V], top = kNone;
  if (a.fp32) {
    const float* from = static_cast<const float*>(a.logits) + t * a.ld + sub;
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = live && i * L + sub < a.E ? from[i * L] : kNone;
  } else {
    const uint16_t* from = static_cast<const uint16_t*>(a.logits) + t * a.ld + sub;
#pragma unroll
    for (int i = 0; i < V; ++i) l[i] = live && i * L + sub < a.E ? bf16_lo(from[i * L]) : kNone;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    bias[i] = 0.f;
    if (BIAS && i * L + sub < a.E) bias[i] = a.bias[i * L + sub];
    l[i] = l[i] == l[i] ? l[i] : kNone;
    top = fmaxf(top, l[i]);
  }
  top = over_lanes<L>(top, [](float x, float y) { return fmaxf(x, y); });

  double total = a.sigmoid ? 1.0 : 0.0;   // of the softmax, once it is asked for
  auto form_total = [&]() { total = row_sum<L, V>([&](int i) { return part(a, l[i], top); }); };
  auto score = [&](float of) { return a.sigmoid ? part(a, of, top) : part(a, of, top) / total; };   // (one form wherever it is asked for: sums may differ by their last bit alone)
  auto exact = [&](double (&s)[V]) {   // scores plus biases
    if (!a.sigmoid && total == 0.0) form_total();
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = l[i] > kNone && bias[i] > kNone ? score(l[i]) + (double)bias[i] : -INFINITY;   // (a comparison with NaN is false)
  };

  float key[V], off = 0.f;
  const Meeting meet(a, top);
  auto keep_groups_exactly = [&](const float (&k)[V]) {
    double s64[V];
    exact(s64);
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = k[i];
    keep_groups<L, V, false>(a, lds, sub, s64, key, 0.0, meet);
  };
  const bool by_sums = BIAS || (a.groups > 1 && a.two_best);
  if (by_sums) {
    float s[V], inverse = 1.f;
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = part32(a, l[i], top);
    if (!a.sigmoid) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) sum += s[i];
      inverse = __builtin_amdgcn_rcpf(over_lanes<L>(sum, [](float x, float y) { return x + y; }));
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      s[i] = l[i] > kNone && bias[i] > kNone ? s[i] * inverse + bias[i] : kNone;
      key[i] = BIAS ? s[i] : l[i];
    }
    off = 2.f * (a.sigmoid ? kSigmoidOff : kSoftmaxOff);   // two of them against each other
    if (a.groups > 1) {
      const bool groups_sure = keep_groups<L, V, false>(a, lds, sub, s, key, 2.f * off, meet) > 0.f;
      if (__ballot(live && !groups_sure)) keep_groups_exactly(BIAS ? s : l);
    }
    if (!BIAS) off = 0.f;
  } else {   // (a group's best logit has its best score, which another group may have too)
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = l[i];
    if (a.groups > 1) {
      const bool groups_sure = keep_groups<L, V, true>(a, lds, sub, l, key, 0.f, meet) > 0.f;
      if (__ballot(live && !groups_sure)) keep_groups_exactly(l);
    }
  }

  const bool check = BIAS || a.fp32;   // (bf16 has its lowest 16 bits zero: its keys are whole)
  Picker<L, V> pick(key);
  float before = INFINITY, last_in = 0.f;
  bool sure = true;
#pragma unroll 1
  for (int r = 0; r < a.k + (check ? 1 : 0); ++r) {
    const float now = number(pick.next(sub, &chosen[r]));
    if (r > 0) sure = sure && ahead_by(before, now, off);
    if (r < a.k) last_in = now;
    before = now;
  }
  if (check && __ballot(live && !sure)) {
    float now = before;
#pragma unroll 1
    for (int r = a.k + 1; r < a.k + kMore; ++r) now = number(pick.next(sub, &chosen[r]));
    const int candidates = a.k + kMore;
    const bool enough = candidates <= L && ahead_by(last_in, now, off);
    if (__ballot(live && !sure && !enough) == 0) {
      wave_lds();
      if (BIAS && !a.sigmoid && total == 0.0) form_total();
      int id = -1;
      double n = -INFINITY;
      if (sub < candidates) id = chosen[sub];
      if (live && id >= 0) n = BIAS ? score(logit(a, t * a.ld + id)) + (double)a.bias[id] : (double)logit(a, t * a.ld + id);
      double* const numbers = reinterpret_cast<double*>(lds);
      if (sub < candidates) numbers[sub] = n;
      wave_lds();
      const int order = id >= 0 ? id : kMostExperts + sub;
      int place = 0;
#pragma unroll 4
      for (int c = 0; c < candidates; ++c) {
        const double other = numbers[c];
        const int other_id = chosen[c], other_order = other_id >= 0 ? other_id : kMostExperts + c;
        place += other > n || (other == n && other_order < order);
      }
      wave_lds();
      if (sub < candidates) chosen[place] = id;
    } else if constexpr (BIAS) {
      double s64[V];
      exact(s64);
#pragma unroll
      for (int i = 0; i < V; ++i) s64[i] = key[i] > kNone ? s64[i] : -INFINITY;   // (groups that are not kept)
      largest<L, V>(a, sub, s64, chosen);
    } else {
      largest<L, V>(a, sub, key, chosen);
    }
  }

  wave_lds();
  if (!a.sigmoid && !a.renormalize && total == 0.0) form_total();
  int id[2] = {-1, -1};
  double w[2] = {0.0, 0.0};
#pragma unroll
  for (int j = 0; j < (L < kMostChosen ? 2 : 1); ++j) {
    if (L * j >= a.k) continue;
    if (sub + L * j < a.k) id[j] = chosen[sub + L * j];
    if (live && id[j] >= 0) w[j] = part(a, logit(a, t * a.ld + id[j]), top);
  }
  if (a.renormalize) total = row_sum<L, 1>([&](int) { return w[0] + w[1]; });   // (places sub and sub + 16; with 64 lanes, one place each, these meet first)
  if (!live) return;
#pragma unroll
  for (int j = 0; j < (L < kMostChosen ? 2 : 1); ++j) {
    const int place = sub + j * L;
    if (place >= a.k) continue;
    a.ids[t * a.k + place] = id[j];
    a.weights[t * a.k + place] = total > 0.0 ? (float)(w[j] / total * (double)a.scale) : 0.f;
  }
}

template <int L, int V, bool BIAS>
__global__ __launch_bounds__(256) void ccq_route_kernel(RouteArgs a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int kRows = 256 / L;
  __shared__ int32_t chosen[kRows][kPlaces];
  const int row = threadIdx.x / L;
  choose<L, V, BIAS>(a, lds + row * row_bytes(a.E, a.groups), chosen[row], (int64_t)blockIdx.x * kRows + row, threadIdx.x % L);
}

// A few rows and their order in one launch, a wavefront for each row and as many more as help the order.
struct FromLds {
  const int32_t (*rows)[kPlaces];
  Divisor k;
  int E;
  __device__ __forceinline__ uint32_t operator()(int i) const {
    const int t = k.divide(i), id = rows[t][i - t * k.by];
    return id >= 0 ? (uint32_t)id : (uint32_t)E;
  }
};
// Two launches and one, with the call's order in a graph: one row of 64 experts 6.7 and 5.6 us, eight of 64 7.3 and 6.3, of 256 8.6 and 7.0, of 512 9.0 and 8.1, eight with 32 of 1024 16.2
// and 16.7.  (A workgroup has room for 16 rows' wavefronts; more than eight have not been measured.)
constexpr int kFewRows = 8;
template <int V, bool BIAS>
__global__ __launch_bounds__(64 * kFewRows) void ccq_route_few_kernel(RouteArgs a, SortArgs sort) {
  extern __shared__ __align__(16) char lds[];
  __shared__ int32_t chosen[kFewRows][kPlaces];
  const int row = threadIdx.x / 64;
  if (row < a.T) choose<64, V, BIAS>(a, lds + row * row_bytes(a.E, a.groups), chosen[row], row, threadIdx.x & 63);
  __syncthreads();
  sort_entries<1>(sort, reinterpret_cast<uint32_t*>(lds), blockDim.x / 64, 0, sort.P, FromLds{chosen, sort.k, a.E}, nullptr, 0, 1);
}

template <typename Kernel>
bool fits(Kernel kernel, int lds) {
  return lds <= 48 * 1024 || hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) == hipSuccess;
}

template <int L, int V, bool BIAS>
bool launch(const RouteArgs& all, hipStream_t s) {
  constexpr int kRows = 256 / L;
  constexpr int64_t kMost = most_groups(256) * kRows;
  const int lds = kRows * row_bytes(all.E, all.groups);
  if (!fits(ccq_route_kernel<L, V, BIAS>, lds)) return false;
  RouteArgs a = all;
  for (int64_t t = 0; t < all.T; t += kMost) {
    a.T = (int32_t)(all.T - t < kMost ? all.T - t : kMost);
    a.logits = static_cast<const char*>(all.logits) + t * all.ld * (all.fp32 ? 4 : 2);
    a.ids = all.ids + t * all.k, a.weights = all.weights + t * all.k;
    hipLaunchKernelGGL((ccq_route_kernel<L, V, BIAS>), dim3((unsigned)((a.T + kRows - 1) / kRows)), dim3(256), (size_t)lds, s, a);
  }
  return true;
}

template <bool BIAS>
bool launch_by_size(const RouteArgs& a, hipStream_t s) {
  // Few rows: a wavefront each, so that its steps are short; many: 16 lanes each, which have less to exchange.  Eight of 256, 1024 / 4096 / 8192 rows: 5.5 / 7.9 / 12.3 us with 64
  // lanes, 8.1 / 8.6 / 9.9 with 16; of 64 experts 4.6 / 6.3 / 9.5 and 4.9 / 5.0 / 5.5.
  if (a.T > 2048) {
    if (a.E <= 64) return launch<16, 4, BIAS>(a, s);
    if (a.E <= 128) return launch<16, 8, BIAS>(a, s);
    if (a.E <= 256) return launch<16, 16, BIAS>(a, s);
  }
  if (a.E <= 64) return launch<64, 1, BIAS>(a, s);
  if (a.E <= 128) return launch<64, 2, BIAS>(a, s);
  if (a.E <= 256) return launch<64, 4, BIAS>(a, s);
  if (a.E <= 512) return launch<64, 8, BIAS>(a, s);
  return launch<64, 16, BIAS>(a, s);
}

template <int V, bool BIAS>
bool launch_few(const RouteArgs& a, const SortArgs& sort, hipStream_t s) {
  const int for_sort = (a.E + 1 + 63) / 64, waves = a.T > for_sort ? a.T : for_sort < kFewRows ? for_sort : kFewRows;   // (the sort's sums go over all experts)
  const int rows = a.T * row_bytes(a.E, a.groups), words = 4 * sort_words(waves, a.E), lds = rows > words ? rows : words;
  if (!fits(ccq_route_few_kernel<V, BIAS>, lds)) return false;
  hipLaunchKernelGGL((ccq_route_few_kernel<V, BIAS>), dim3(1), dim3(64 * waves), (size_t)lds, s, a, sort);
  return true;
}
template <bool BIAS>
bool launch_few_by_size(const RouteArgs& a, const SortArgs& sort, hipStream_t s) {
  if (a.E <= 64) return launch_few<1, BIAS>(a, sort, s);
  if (a.E <= 128) return launch_few<2, BIAS>(a, sort, s);
  if (a.E <= 256) return launch_few<4, BIAS>(a, sort, s);
  if (a.E <= 512) return launch_few<8, BIAS>(a, sort, s);
  return launch_few<16, BIAS>(a, sort, s);
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
  if (order && a.T > 0 && a.T <= kFewRows) {
    SortArgs sort;
    sort.ids = nullptr, sort.counts = nullptr, sort.ld_ids = 0;
    sort.rows = order->rows, sort.experts = order->experts, sort.offsets = order->offsets, sort.places = order->places;
    sort.P = a.T * a.k, sort.k = Divisor(a.k), sort.first = 0, sort.E = a.E, sort.chunk = sort.P;
    sort.stretch = 64;   // (top_k is 32 at most)
    sort.bits = bits_of(a.E);
    const bool ok = a.bias ? launch_few_by_size<true>(a, sort, s) : launch_few_by_size<false>(a, sort, s);
    return ok && hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
  }
  if (a.T > 0 && (!(a.bias ? launch_by_size<true>(a, s) : launch_by_size<false>(a, s)) || hipGetLastError() != hipSuccess)) return CCQ_ERR_HIP;
  return order ? launch_sort(r->ids, r->top_k, r->T, r->top_k, 0, r->experts, order, workspace, stream) : CCQ_OK;
}

}  // namespace ccq
