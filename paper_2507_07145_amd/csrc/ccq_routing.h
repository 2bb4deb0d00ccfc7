// What the kernels around rows that choose their weights share: their limits, and the launchers that the host checks (ccq_routing.cpp) call.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "ccq.h"
#include "ccq_layer.h"

namespace ccq {

constexpr int kMostSorted = 4096;    // experts of an order
constexpr int kMostExperts = 1024;   // of a router
constexpr int kMostChosen = 32;
constexpr int kMostRank = 256;

int64_t sort_workspace(int T, int k, int experts);
int launch_sort(const int32_t* ids, int64_t ld_ids, int T, int k, int first, int experts, const ccq_order* order, void* workspace, void* stream);
int64_t route_workspace(const ccq_router* r);
int launch_route(const ccq_router* r, const ccq_order* order, void* workspace, void* stream);
int launch_combine(const ccq_combination* c, void* stream);
int64_t adapters_workspace(const ccq_adapter_set* set, int T);
int launch_adapters(const ccq_adapter_set* set, int T, const int32_t* rows, const int32_t* experts, const void* x, int64_t ldx, const void* y, int64_t ldy, void* out,
                    int64_t ld_out, void* workspace, void* stream);

}  // namespace ccq
