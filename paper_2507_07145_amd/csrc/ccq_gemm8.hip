// 8-bit product for few rows: weights go from memory to registers once, activations come from the caches.
//
// A workgroup owns 16 outputs (of all rows of a tile of 16 MT rows); its wavefronts take the blocks of K in turn and their
// accumulators are added through LDS at the end, in a fixed order.  Bound by memory: the weights' bytes.  One row, 8192 x 8192: 13.0 us, 5.2 TB/s.
// (For 17 to 64 rows its activations cost more than the weights: every 16 columns read them all.  37 rows, 5001 x 7184: 22 to 27 us in all shapes tried, the
// streaming kernel with its join 15.5.)
#include <algorithm>
#include <cmath>

#include "ccq_gemm8.h"

namespace ccq {

namespace {

// WIDE: bf16 rows, quantized on the way to the product: the lanes of a row hold a block between them.
template <int MT, int W, bool WIDE>
__global__ __launch_bounds__(64 * W) void ccq_gemm8_few_kernel(Gemm8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * (16 * MT);
  __shared__ __align__(16) float parts[W * MT * 16 * 20];
  const uint8_t* w = a.w + (int64_t)min(n0 + r16, a.N - 1) * a.ldw;
  const float* ws = a.ws + (int64_t)(n0 / kScaleBlock) * a.ld_ws;
  const uint8_t* x[MT];
  const uint8_t* xs[MT];
  const uint16_t* x16[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = min(m0 + 16 * i + r16, a.M - 1);
    if constexpr (WIDE) {
      x16[i] = a.x16 + m * a.ldx16;
    } else {
      x[i] = a.x + m * a.ldx;
      xs[i] = a.xs + m * a.ld_xs;
    }
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
  for (int kb = wave; kb < a.blocks; kb += W) {
    const int k = kb * kScaleBlock + 16 * g;
    const i32x8_t wv = operand8(piece(w, k), piece(w, k + 64));
    const float s = ws[kb];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      i32x8_t xv;
      int scale;
      if constexpr (WIDE) {
        const Wide16 lo = load_wide16(x16[i] + k, k < a.K), hi = load_wide16(x16[i] + k + 64, k + 64 < a.K);
        uint32_t top = max(magnitude16(lo), magnitude16(hi));
        top = max(top, xor16(top));
        top = max(top, xor32(top));
        xv = operand8(codes16(lo, top), codes16(hi, top));
        scale = scale_of(top);
      } else {
        xv = operand8(piece(x[i], k), piece(x[i], k + 64));
        scale = xs[i][kb];
      }
      const f32x4_t p = multiply8(wv, xv, scale);
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

namespace {

Gemm8Args args_of(const ccq_weight8* w, const ccq_rows8* x, int M, void* y, int64_t ldy, void* workspace) {
  Gemm8Args a = {};
  a.w = static_cast<const uint8_t*>(w->codes), a.ws = w->scales, a.ldw = w->ldw, a.ld_ws = w->ld_scales;
  if (x) a.x = static_cast<const uint8_t*>(x->codes), a.xs = x->scales, a.ldx = x->ld, a.ld_xs = x->ld_scales;
  a.y = static_cast<uint16_t*>(y), a.ldy = ldy, a.partial = static_cast<float*>(workspace);
  a.M = M, a.N = w->N, a.K = w->K, a.blocks = (w->K + kScaleBlock - 1) / kScaleBlock;
  a.ld_partial = ((int64_t)a.N + 3) / 4 * 4;
  return a;
}

// (rows far apart may be many: in parts, for a grid's second dimension ends at 65535)
template <int MT, int W>
int launch_few(Gemm8Args a, hipStream_t s) {
  constexpr int kMost = 65535 * 16 * MT;
  for (int rows = a.M; rows > 0; rows -= kMost) {
    a.M = std::min(rows, kMost);
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
    if (a.x16) hipLaunchKernelGGL((ccq_gemm8_few_kernel<MT, W, true>), grid, dim3(64 * W), 0, s, a);
    else hipLaunchKernelGGL((ccq_gemm8_few_kernel<MT, W, false>), grid, dim3(64 * W), 0, s, a);
    if (a.x16) a.x16 += (int64_t)kMost * a.ldx16;
    else a.x += (int64_t)kMost * a.ldx, a.xs += (int64_t)kMost * a.ld_xs;
    a.y += (int64_t)kMost * a.ldy;
  }
  return hipGetLastError() == hipSuccess ? CCQ_OK : CCQ_ERR_HIP;
}

// How a call is served: `kind` few rows (mt: 16-row tiles of a workgroup, waves), stream (mt, shares), block (mt: 64-row units, shares); a block plan
// may end at column n_rest, the columns from there on are a product of their own in blocks of mt_rest and shares_rest.
enum Kind8 { kFew = 0, kStream = 1, kBlock = 2 };
struct Plan8 {
  int kind = kFew, mt = 1, shares = 1, waves = 4, n_rest = 0, mt_rest = 0, shares_rest = 1;
  bool quantizes = false;   // bf16 rows become 8-bit rows in the kernel, not by a launch before it
  double time = 1e30;       // estimate, microseconds
};

int64_t columns_of_partial(int64_t n) { return (n + 3) / 4 * 4; }
int64_t workspace_of(const Plan8& p, int64_t M, int64_t N) {
  if (p.n_rest > 0) return p.shares_rest > 1 ? p.shares_rest * M * columns_of_partial(N - p.n_rest) * 4 : 0;
  return p.shares > 1 ? p.shares * M * columns_of_partial(N) * 4 : 0;
}

int run(const Gemm8Args& a, const Plan8& p, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.kind == kFew) return p.mt == 4 ? launch_few<4, 4>(a, s) : p.waves == 16 ? launch_few<1, 16>(a, s) : launch_few<1, 4>(a, s);
  if (p.kind == kStream) return launch_gemm8_stream(a, p.mt, p.shares, stream);
  if (p.n_rest == 0) return launch_gemm8_block(a, p.mt, p.shares, stream);
  Gemm8Args left = a, rest = a;
  left.N = p.n_rest;
  rest.N = a.N - p.n_rest;   // (n_rest is a multiple of 256: whole blocks of scales, aligned outputs)
  rest.w += (int64_t)p.n_rest * a.ldw, rest.ws += (int64_t)(p.n_rest / kScaleBlock) * a.ld_ws, rest.y += p.n_rest;
  rest.ld_partial = columns_of_partial(rest.N);
  const int rc = launch_gemm8_block(left, p.mt, 1, stream);
  return rc != CCQ_OK ? rc : launch_gemm8_block(rest, p.mt_rest, p.shares_rest, stream);
}

// The kernels' times as they were measured on K = 8192, N = 8192 and 28672, M = 1 .. 2048 (and short and narrow products), as lines in the steps of a
// workgroup and the share of the chip that is busy: within about 15 % of all of them, which are further apart than that where the choice matters.
constexpr double kCus = 256.0;
double rounds_of(double groups) { return std::ceil(groups / kCus); }
double busy(double groups) { return std::min(1.0, groups / (kCus * rounds_of(groups))); }
double add_time(double shares, double M, double N, bool block) { return shares > 1 ? (block ? 4.0 + shares * M * N * 4.0 / 3e6 : 2.0 + shares * M * N * 4.0 / 5e6) : 0.0; }
double few_time(int mt, int waves, int M, int N, int blocks) {
  const double tiles = (N + 15) / 16, its = (blocks + waves - 1) / waves;
  if (mt == 4) return 4.0 + its * std::ceil(M / 64.0) * (1.2 + 2.3 * std::min(4.0, tiles / 512.0));
  return std::max(2.5 + (double)N * blocks * kScaleBlock / 5.7e6 * (1.0 + 0.04 * (M - 1)), 4.0 + its * (waves == 16 ? 1.0 : 0.4));
}
double stream_time(int mt, int shares, int M, int N, int blocks) {
  const double groups = (double)((N + 127) / 128) * shares * ((M + 16 * mt - 1) / (16 * mt)), steps = std::ceil(std::ceil((double)blocks / shares) / 2.0);
  return 4.0 + rounds_of(groups) * (1.0 + steps * (0.75 + 0.1 * mt + 0.6 * busy(groups))) + add_time(shares, M, N, false);
}
// `alone`: one block of rows, whose weights come from memory and not from a neighbour's reading
double block_rounds_time(int mi, double groups, double steps, bool alone) {
  const double full = busy(groups);
  const double per = mi == 4 ? 1.45 + 0.5 * full : mi == 2 ? (alone ? 0.9 + 0.6 * full : 0.8 + 0.35 * full) : alone ? 0.7 + 0.4 * full : 0.55 + 0.22 * full;
  return rounds_of(groups) * ((alone ? 5.0 : mi == 4 ? 4.0 : 2.5) + steps * per);
}
double block_groups(int mi, int M, int n, int shares) { return (double)((M + 64 * mi - 1) / (64 * mi)) * ((n + 255) / 256) * shares; }

// Whether a kernel for few rows quantizes bf16 rows itself: that saves a launch of 3 us, and every workgroup does it for all rows.  Measured against the
// launch: few rows, 2048 x 7168, 1 / 4 / 16 rows: 7.6 / 8.4 / 12.8 us against 8.8 / 9.7 / 11.1; 5001 x 7184: alike; 28672 x 8192: 48 - 55 against 43 - 47.  Streaming
// kernel, 8192 x 8192, 32 / 37 rows: 20.3 / 23.5 against 22.5 / 23.1; 2048 x 7168, 37 rows: 16.3 against 17.5.  1024 x 1024, 1 to 64 rows: 4.2 - 8.2 against 9.
bool quantizes(const Plan8& p, int M, int N, int K) {
  const double size = (double)N * K;
  if (p.kind == kFew) return size <= (M <= 8 ? 40e6 : 4e6);
  return p.kind == kStream && (p.mt <= 2 || (p.mt <= 4 && size <= 16e6));
}

// wide: bf16 rows
Plan8 find_plan(int M, int N, int K, bool wide) {
  const int blocks = (K + kScaleBlock - 1) / kScaleBlock;
  const double quantizing = wide ? 3.0 + (double)M * K * 3.0 / 4.9e6 : 0.0;
  Plan8 best;
  auto offer = [&](Plan8 p) {
    p.quantizes = wide && quantizes(p, M, N, K);
    if (wide && !p.quantizes) p.time += quantizing;
    if (p.time < best.time) best = p;
  };
  auto few = [&](int mt, int waves) {
    Plan8 p;
    p.kind = kFew, p.mt = mt, p.waves = waves, p.time = few_time(mt, waves, M, N, blocks);
    offer(p);
  };
  if (M <= 16) {
    few(1, 16);
    if (M > 4) few(1, 4);
  }
  if (M <= 64) few(4, 4);
  static const int kShares[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 24, 32};
  if (M <= 192) {
    for (const int mt : {1, 2, 3, 4, 6}) {
      if (mt > 1 && 16 * (mt - 1) >= M) break;   // (rows of nothing)
      if (M > 16 * mt && mt < 4) continue;       // (a tile of all rows, or the larger ones)
      for (const int shares : kShares) {
        if (shares > 1 && shares * 2 > blocks) break;
        if (stream_lds(mt, stream_blocks(blocks, shares)) > kMostLds) continue;   // (the scales of a long share)
        Plan8 p;
        p.kind = kStream, p.mt = mt, p.shares = shares, p.time = stream_time(mt, shares, M, N, blocks);
        offer(p);
      }
    }
  }
  if (M > 32) {
    const double bytes = 4.0 + ((double)N * K + (double)M * K + 2.0 * M * N) / 4.9e6;
    for (const int mi : {1, 2, 4}) {
      if (mi > 1 && M <= 32 * mi) break;
      for (const int shares : kShares) {
        if (shares > 1 && (shares * 4 > blocks || (double)shares * M * N * 4 > 256e6)) break;
        Plan8 p;
        p.kind = kBlock, p.mt = mi, p.shares = shares;
        p.time = std::max(bytes, 4.0 + block_rounds_time(mi, block_groups(mi, M, N, shares), std::ceil((double)blocks / shares), M <= 64 * mi)) + add_time(shares, M, N, true);
        offer(p);
      }
      // whole rounds of the chip in these blocks, the columns that are left in smaller ones
      const int m_tiles = (M + 64 * mi - 1) / (64 * mi), n_tiles = (N + 255) / 256, full = (int)((int64_t)m_tiles * n_tiles / 256) * 256 / m_tiles;
      if (mi > 1 && full > 0 && full < n_tiles) {
        for (const int rest : {1, 2, 4}) {
          for (const int shares : kShares) {
            if (shares > 8 || (shares > 1 && shares * 4 > blocks)) break;
            Plan8 p;
            p.kind = kBlock, p.mt = mi, p.n_rest = full * 256, p.mt_rest = rest, p.shares_rest = shares;
            p.time = 6.0 + block_rounds_time(mi, block_groups(mi, M, p.n_rest, 1), blocks, M <= 64 * mi) +
                     block_rounds_time(rest, block_groups(rest, M, N - p.n_rest, shares), std::ceil((double)blocks / shares), false) + add_time(shares, M, N - p.n_rest, true);
            offer(p);
          }
        }
      }
    }
  }
  return best;
}

// The plans of the sizes that a thread asked for last: finding one takes up to 5 us of host time.
Plan8 plan_of(int M, int N, int K, bool wide) {
  struct Known {
    int M = 0, N = 0, K = 0;
    Plan8 plan;
  };
  static thread_local Known known[2][64];
  Known& k = known[wide][((unsigned)M * 31 + (unsigned)N * 7 + (unsigned)K / 16) % 64];
  if (k.M != M || k.N != N || k.K != K) {
    k.plan = find_plan(M, N, K, wide);
    k.M = M, k.N = N, k.K = K;
  }
  return k.plan;
}

}  // namespace

int64_t gemm8_workspace(const ccq_weight8* w, int M) {
  if (M <= 0) return 0;
  return workspace_of(plan_of(M, w->N, w->K, false), M, w->N);
}

namespace {

// Calls whose weights' or activations' rows are too far apart for 32-bit offsets within the block kernel's 256 rows.
constexpr int64_t kFarRows = 1 << 23;
const Plan8 kFar = {kFew, 4, 1, 4, 0, 0, 1, true, 0.0};

Plan8 wide_plan(const ccq_weight8* w, int M) { return w->ldw > kFarRows || w->K > kFarRows ? kFar : plan_of(M, w->N, w->K, true); }
// Workspace of a call with bf16 rows that are quantized first: partial results, codes, scales.
int64_t codes_at(const Plan8& p, int64_t M, int64_t N) { return (workspace_of(p, M, N) + 255) / 256 * 256; }

}  // namespace

int64_t gemm8_bf16_workspace(const ccq_weight8* w, int M) {
  if (M <= 0) return 0;
  const Plan8 p = wide_plan(w, M);
  return !p.quantizes ? codes_at(p, M, w->N) + (int64_t)M * w->K + (int64_t)M * ((w->K + kScaleBlock - 1) / kScaleBlock) : workspace_of(p, M, w->N);
}

int launch_gemm8_bf16(const ccq_weight8* w, const void* x, int64_t ldx, int M, void* y, int64_t ldy, void* workspace, void* stream) {
  const Plan8 p = wide_plan(w, M);
  if (p.quantizes) {
    Gemm8Args a = args_of(w, nullptr, M, y, ldy, workspace);
    a.x16 = static_cast<const uint16_t*>(x), a.ldx16 = ldx;
    return run(a, p, stream);
  }
  ccq_norm n = {};
  n.M = M, n.N = w->K, n.x = x, n.ldx = ldx;
  n.y8.codes = static_cast<uint8_t*>(workspace) + codes_at(p, M, w->N), n.y8.ld = w->K;
  n.y8.scales = static_cast<uint8_t*>(n.y8.codes) + (int64_t)M * w->K, n.y8.ld_scales = (w->K + kScaleBlock - 1) / kScaleBlock;
  const int rc = launch_norm(&n, false, stream);
  return rc != CCQ_OK ? rc : run(args_of(w, &n.y8, M, y, ldy, workspace), p, stream);
}

int launch_gemm8(const ccq_weight8* w, const ccq_rows8* x, int M, void* y, int64_t ldy, void* workspace, void* stream) {
  const Gemm8Args a = args_of(w, x, M, y, ldy, workspace);
  return run(a, a.ldw > kFarRows || a.ldx > kFarRows ? kFar : plan_of(M, a.N, a.K, false), stream);
}

// For tests, no part of the interface: how a call of these sizes is served (the numbers of the plan, and the estimate).
extern "C" void ccq_gemm8_plan(int32_t M, int32_t N, int32_t K, int32_t* out, double* time) {
  const Plan8 p = plan_of(M, N, K, false);
  const int v[7] = {p.kind, p.mt, p.shares, p.waves, p.n_rest, p.mt_rest, p.shares_rest};
  for (int i = 0; i < 7; ++i) out[i] = v[i];
  *time = p.time;
}

// Whether there are kernels for a plan, and rows that they reach.
static bool can_run(const Plan8& p, const Gemm8Args& a) {
  auto block = [](int mt, int shares) { return (mt == 1 || mt == 2 || mt == 4) && shares >= 1 && shares <= 64; };
  if (p.n_rest != 0 && (p.kind != kBlock || p.n_rest < 0 || p.n_rest % 256 != 0 || p.n_rest >= a.N || p.shares != 1 || !block(p.mt_rest, p.shares_rest))) return false;
  if (p.kind == kFew) return p.shares == 1 && (p.mt == 4 ? p.waves == 4 : p.mt == 1 && (p.waves == 4 || p.waves == 16));
  if (p.kind == kStream)
    return (p.mt == 6 ? !a.x16 : p.mt >= 1 && p.mt <= 4) && p.shares >= 1 && p.shares <= 64 && stream_lds(p.mt, stream_blocks(a.blocks, p.shares)) <= kMostLds;
  return p.kind == kBlock && block(p.mt, p.shares) && !a.x16 && a.ldw <= kFarRows && a.ldx <= kFarRows;
}

// The same: a call as a named plan.  x without scales: bf16 rows.  (`workspace` is as large as the plan's partial results.)
int launch_gemm8_as(const ccq_weight8* w, const ccq_rows8* x, int M, void* y, int64_t ldy, void* workspace, const int32_t* plan, void* stream) {
  Plan8 p;
  p.kind = plan[0], p.mt = plan[1], p.shares = plan[2], p.waves = plan[3], p.n_rest = plan[4], p.mt_rest = plan[5], p.shares_rest = plan[6];
  Gemm8Args a = args_of(w, x, M, y, ldy, workspace);
  if (!x->scales) a.x16 = static_cast<const uint16_t*>(x->codes), a.ldx16 = x->ld;
  if (!can_run(p, a)) return CCQ_ERR_BAD_PARAM;
  if (workspace_of(p, M, w->N) > 0 && !workspace) return CCQ_ERR_WORKSPACE;
  return run(a, p, stream);
}

}  // namespace ccq
