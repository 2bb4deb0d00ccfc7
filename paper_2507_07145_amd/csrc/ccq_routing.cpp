// Argument checks of the operators around rows that choose their weights: everything is checked before the first launch.  No device code in this file.
#include "ccq_routing.h"

#include <cmath>

using namespace ccq;

namespace {

bool off(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
bool is_type(int32_t t) { return t == CCQ_BF16 || t == CCQ_FP32; }
unsigned bytes_of(int32_t t) { return t == CCQ_FP32 ? 4 : 2; }

constexpr int64_t kMostEntries = 1 << 30;   // of an order; rows and columns elsewhere

int check_sort(int32_t T, int32_t k, int32_t experts) {
  if (T < 0 || k < 1 || experts < 1 || (int64_t)T * k > kMostEntries) return CCQ_ERR_BAD_PARAM;
  return experts > kMostSorted ? CCQ_ERR_UNSUPPORTED : CCQ_OK;
}

int check_order(const ccq_order* o, int32_t T) {
  if (!o->offsets || (T > 0 && !o->rows)) return CCQ_ERR_NULL;
  return off(o->rows, 16) || off(o->offsets, 16) || off(o->experts, 4) || off(o->places, 4) ? CCQ_ERR_ALIGN : CCQ_OK;
}

int check_workspace(int64_t need, const void* workspace, int64_t bytes) {
  if (off(workspace, 16)) return CCQ_ERR_ALIGN;
  return need > 0 && (!workspace || bytes < need) ? CCQ_ERR_WORKSPACE : CCQ_OK;
}

int check_router(const ccq_router* r) {
  if (!r) return CCQ_ERR_NULL;
  if (r->T < 0 || r->experts < 1 || r->top_k < 1 || r->groups < 1) return CCQ_ERR_BAD_PARAM;
  if (r->experts % r->groups != 0 || r->top_groups < 1 || r->top_groups > r->groups || r->group_best < 1 || r->group_best > 2) return CCQ_ERR_BAD_PARAM;
  if (r->top_k > (int64_t)r->top_groups * (r->experts / r->groups) || (r->scoring != CCQ_SOFTMAX && r->scoring != CCQ_SIGMOID)) return CCQ_ERR_BAD_PARAM;
  if (!std::isfinite(r->scale) || !is_type(r->logits_type) || (int64_t)r->T * r->top_k > kMostEntries) return CCQ_ERR_BAD_PARAM;
  return r->experts > kMostExperts || r->top_k > kMostChosen ? CCQ_ERR_UNSUPPORTED : CCQ_OK;
}

int check_set(const ccq_adapter_set* s, int32_t T) {
  if (!s) return CCQ_ERR_NULL;
  if (s->count < 1 || s->rank < 1 || s->K < 1 || s->N < 1 || s->K > kMostEntries || s->N > kMostEntries || T < 0 || T > kMostEntries) return CCQ_ERR_BAD_PARAM;
  if (s->rank > kMostRank) return CCQ_ERR_UNSUPPORTED;
  return s->rank % 8 != 0 || s->K % 8 != 0 ? CCQ_ERR_ALIGN : CCQ_OK;
}

}  // namespace

extern "C" int64_t ccq_sort_rows_workspace_bytes(int32_t T, int32_t k, int32_t experts) {
  return check_sort(T, k, experts) == CCQ_OK ? sort_workspace(T, k, experts) : -1;
}

extern "C" int ccq_sort_rows(const int32_t* ids, int64_t ld_ids, int32_t T, int32_t k, int32_t first, int32_t experts, const ccq_order* order, void* workspace,
                             int64_t workspace_bytes, void* hip_stream) {
  if (!order) return CCQ_ERR_NULL;
  int rc = check_sort(T, k, experts);
  if (rc != CCQ_OK) return rc;
  if (first < 0 || ld_ids < k) return CCQ_ERR_BAD_PARAM;
  if ((rc = check_order(order, T)) != CCQ_OK) return rc;
  if (T > 0 && !ids) return CCQ_ERR_NULL;
  if (off(ids, 4)) return CCQ_ERR_ALIGN;
  if ((rc = check_workspace(sort_workspace(T, k, experts), workspace, workspace_bytes)) != CCQ_OK) return rc;
  return launch_sort(ids, ld_ids, T, k, first, experts, order, workspace, hip_stream);
}

extern "C" int64_t ccq_route_workspace_bytes(const ccq_router* r, int32_t with_order) {
  if (check_router(r) != CCQ_OK) return -1;
  return with_order ? route_workspace(r) : 0;
}

extern "C" int ccq_route(const ccq_router* r, const ccq_order* order, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  int rc = check_router(r);
  if (rc != CCQ_OK) return rc;
  if (r->T > 0) {
    if (r->ld < r->experts) return CCQ_ERR_BAD_PARAM;
    if (!r->logits || !r->ids || !r->weights) return CCQ_ERR_NULL;
    if (off(r->logits, bytes_of(r->logits_type)) || off(r->bias, 4) || off(r->ids, 4) || off(r->weights, 4)) return CCQ_ERR_ALIGN;
  }
  if (order && ((rc = check_order(order, r->T)) != CCQ_OK || (rc = check_workspace(route_workspace(r), workspace, workspace_bytes)) != CCQ_OK)) return rc;
  return launch_route(r, order, workspace, hip_stream);
}

extern "C" int ccq_combine(const ccq_combination* c, void* hip_stream) {
  if (!c) return CCQ_ERR_NULL;
  if (c->T < 0 || c->k < 1 || c->N < 1 || c->P < 0 || c->N > kMostEntries || !is_type(c->base_type) || !is_type(c->y_type)) return CCQ_ERR_BAD_PARAM;
  if (c->T == 0) return CCQ_OK;
  if (!c->places || !c->weights || !c->y || (c->P > 0 && !c->rows)) return CCQ_ERR_NULL;
  if (c->ld_rows < c->N || c->ld_places < c->k || c->ld_weights < c->k || c->ldy < c->N || (c->base && c->ld_base < c->N)) return CCQ_ERR_BAD_PARAM;
  if (c->y == c->base && ((c->T > 1 && c->ldy != c->ld_base) || c->y_type != c->base_type)) return CCQ_ERR_BAD_PARAM;
  if (off(c->rows, 2) || off(c->places, 4) || off(c->weights, 4) || off(c->base, bytes_of(c->base_type)) || off(c->y, bytes_of(c->y_type))) return CCQ_ERR_ALIGN;
  return launch_combine(c, hip_stream);
}

extern "C" int64_t ccq_adapters_workspace_bytes(const ccq_adapter_set* set, int32_t T) { return check_set(set, T) == CCQ_OK ? adapters_workspace(set, T) : -1; }

extern "C" int ccq_adapters(const ccq_adapter_set* set, int32_t T, const int32_t* rows, const int32_t* experts, const void* x, int64_t ldx, const void* y, int64_t ldy,
                            void* out, int64_t ld_out, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  int rc = check_set(set, T);
  if (rc != CCQ_OK) return rc;
  if (ldx < set->K || ldy < set->N || ld_out < set->N) return CCQ_ERR_BAD_PARAM;
  if (T == 0) return CCQ_OK;
  if (!set->a || !set->b || !rows || !experts || !x || !y || !out) return CCQ_ERR_NULL;
  if (T > 1 && y == out && ldy != ld_out) return CCQ_ERR_BAD_PARAM;
  if (off(set->a, 16) || off(set->b, 16) || off(set->scales, 4) || off(set->ranks, 4) || off(rows, 4) || off(experts, 4) || off(x, 2) || off(y, 2) || off(out, 2))
    return CCQ_ERR_ALIGN;
  if ((rc = check_workspace(adapters_workspace(set, T), workspace, workspace_bytes)) != CCQ_OK) return rc;
  return launch_adapters(set, T, rows, experts, x, ldx, y, ldy, out, ld_out, workspace, hip_stream);
}
