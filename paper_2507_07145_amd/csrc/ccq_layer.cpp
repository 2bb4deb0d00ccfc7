// Argument checks of the 8-bit layer operators: everything is checked before the first launch.  No device code in this file.
#include <cmath>

#include "ccq_layer.h"

using namespace ccq;

namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool off(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }
int64_t blocks_of(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock; }

int check_rows8(const ccq_rows8& r, int N) {
  if (!r.codes || !r.scales) return CCQ_ERR_NULL;
  if (r.ld < N || r.ld_scales < blocks_of(N)) return CCQ_ERR_BAD_PARAM;
  if (off16(r.codes) || r.ld % 16 != 0) return CCQ_ERR_ALIGN;
  return CCQ_OK;
}

bool is_type(int32_t t) { return t == CCQ_BF16 || t == CCQ_FP32; }
unsigned bytes_of(int32_t t) { return t == CCQ_FP32 ? 4 : 2; }

int check_norm(const ccq_norm* n, bool norm) {
  if (n->M < 0 || n->N < 1) return CCQ_ERR_BAD_PARAM;
  if (norm && (!(n->eps >= 0.f) || std::isinf(n->eps) || !is_type(n->residual_type) || !is_type(n->weight_type))) return CCQ_ERR_BAD_PARAM;
  if (n->M == 0) return CCQ_OK;
  if (!n->x || (!n->y && !n->y8.codes)) return CCQ_ERR_NULL;
  if (n->ldx < n->N || (n->residual && n->ld_residual < n->N) || (n->sum && n->ld_sum < n->N) || (n->y && n->ldy < n->N)) return CCQ_ERR_BAD_PARAM;
  // results may lie on an input exactly, row on row
  if ((n->sum && n->sum == n->residual && n->ld_sum != n->ld_residual) || (n->y && n->y == n->x && n->ldy != n->ldx)) return CCQ_ERR_BAD_PARAM;
  if (off(n->x, 2) || off(n->y, 2) || off(n->residual, bytes_of(n->residual_type)) || off(n->sum, bytes_of(n->residual_type)) ||
      off(n->weight, bytes_of(n->weight_type)))
    return CCQ_ERR_ALIGN;
  if (n->y8.codes || n->y8.scales) return check_rows8(n->y8, n->N);
  return CCQ_OK;
}

constexpr int kMostRows = 0x7FFFFF00;   // (rounded up to blocks they stay within 31 bits)
int check_weight8(const ccq_weight8* w) {
  if (!w) return CCQ_ERR_NULL;
  if (w->K <= 0 || w->N <= 0 || w->K > 0x7FFFFF00 || w->N > 0x7FFFFF00 || w->ldw < w->K || w->ld_scales < blocks_of(w->K)) return CCQ_ERR_BAD_PARAM;
  if (w->K % 16 != 0 || w->ldw % 16 != 0) return CCQ_ERR_ALIGN;
  return CCQ_OK;
}

int check_cache(const ccq_cache* c) {
  if (!c) return CCQ_ERR_NULL;
  if (c->pages < 1 || c->kv_heads < 1) return CCQ_ERR_BAD_PARAM;
  if (c->page_tokens < 1 || c->head_dim < 1) return CCQ_ERR_BAD_PARAM;
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)) != 0) return CCQ_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return CCQ_ERR_UNSUPPORTED;
  return CCQ_OK;
}
int check_cache_pointers(const ccq_cache* c) {
  if (!c->k || !c->v || !c->k_scales || !c->v_scales) return CCQ_ERR_NULL;
  return off16(c->k) || off16(c->v) ? CCQ_ERR_ALIGN : CCQ_OK;
}

constexpr int kMostTokens = 1 << 30;
int check_batch(const ccq_batch* b) {
  if (!b) return CCQ_ERR_NULL;
  if (b->batch < 0 || b->batch > 65535 || b->tokens < 0 || b->max_new < 0 || b->max_len < 0 || b->table_width < 0 || b->ld_table < b->table_width) return CCQ_ERR_BAD_PARAM;
  if (b->max_len > kMostTokens || b->max_new > kMostTokens || b->tokens > kMostTokens) return CCQ_ERR_BAD_PARAM;
  return CCQ_OK;
}
bool nothing(const ccq_batch* b) { return b->batch == 0 || b->tokens == 0 || b->max_new == 0; }
int check_batch_pointers(const ccq_batch* b) {
  if (!b->offsets || !b->lens || (!b->table && b->table_width > 0)) return CCQ_ERR_NULL;
  return off(b->offsets, 4) || off(b->lens, 4) || off(b->table, 4) ? CCQ_ERR_ALIGN : CCQ_OK;
}

int check_heads(const ccq_heads* h, int heads, int head_dim) {
  if (!h->data) return CCQ_ERR_NULL;
  if (h->head_stride < (heads > 1 ? head_dim : 0) || h->token_stride < (int64_t)(heads - 1) * h->head_stride + head_dim) return CCQ_ERR_BAD_PARAM;
  if (off16(h->data) || h->token_stride % 8 != 0 || h->head_stride % 8 != 0) return CCQ_ERR_ALIGN;
  return CCQ_OK;
}

int check_attn(const ccq_cache* c, const ccq_batch* b, const ccq_attn* a) {
  int rc = check_cache(c);
  if (rc == CCQ_OK) rc = check_batch(b);
  if (rc != CCQ_OK) return rc;
  if (!a) return CCQ_ERR_NULL;
  if (a->q_heads < 1 || a->q_heads % c->kv_heads != 0 || a->window < 0 || (a->window > 0 && !a->causal) || !(a->scale > 0.f) || std::isinf(a->scale))
    return CCQ_ERR_BAD_PARAM;
  // rows of a sequence and key head, heads of all tokens
  if ((int64_t)b->max_new * a->q_heads > 0x7FFFFFFF || (int64_t)b->tokens * a->q_heads > 0x7FFFFFFF) return CCQ_ERR_BAD_PARAM;
  return CCQ_OK;
}

}  // namespace

extern "C" int ccq_rms_norm(const ccq_norm* n, void* hip_stream) {
  if (!n) return CCQ_ERR_NULL;
  const int rc = check_norm(n, true);
  if (rc != CCQ_OK || n->M == 0) return rc;
  return launch_norm(n, true, hip_stream);
}

extern "C" int ccq_quantize8(const void* x, int64_t ldx, int32_t M, int32_t N, const ccq_rows8* out, void* hip_stream) {
  if (!out) return CCQ_ERR_NULL;
  ccq_norm n = {};
  n.M = M, n.N = N, n.x = x, n.ldx = ldx, n.y8 = *out;
  const int rc = check_norm(&n, false);
  if (rc != CCQ_OK || M == 0) return rc;
  return launch_norm(&n, false, hip_stream);
}

extern "C" int64_t ccq_gemm8_workspace_bytes(const ccq_weight8* w, int32_t M) {
  if (check_weight8(w) != CCQ_OK || M < 0 || M > kMostRows) return -1;
  return gemm8_workspace(w, M);
}

static int check_gemm8(const ccq_weight8* w, int32_t M, const void* y, int64_t ldy, const void* workspace) {
  const int rc = check_weight8(w);
  if (rc != CCQ_OK) return rc;
  if (M < 0 || M > kMostRows || ldy < w->N) return CCQ_ERR_BAD_PARAM;
  if (ldy % 8 != 0) return CCQ_ERR_ALIGN;
  if (M == 0) return CCQ_OK;
  if (!w->codes || !w->scales || !y) return CCQ_ERR_NULL;
  return off16(w->codes) || off16(w->scales) || off16(y) || off16(workspace) ? CCQ_ERR_ALIGN : CCQ_OK;
}

extern "C" int ccq_gemm8(const ccq_weight8* w, const ccq_rows8* x, int32_t M, void* y, int64_t ldy, void* workspace, int64_t workspace_bytes,
                         void* hip_stream) {
  if (w && !x && check_weight8(w) == CCQ_OK) return CCQ_ERR_NULL;
  int rc = check_gemm8(w, M, y, ldy, workspace);
  if (rc != CCQ_OK || M == 0) return rc;
  if ((rc = check_rows8(*x, w->K)) != CCQ_OK) return rc;
  const int64_t need = gemm8_workspace(w, M);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CCQ_ERR_WORKSPACE;
  return launch_gemm8(w, x, M, y, ldy, workspace, hip_stream);
}

extern "C" int64_t ccq_gemm8_bf16_workspace_bytes(const ccq_weight8* w, int32_t M) {
  if (check_weight8(w) != CCQ_OK || M < 0 || M > kMostRows) return -1;
  return gemm8_bf16_workspace(w, M);
}

extern "C" int ccq_gemm8_bf16(const ccq_weight8* w, const void* x, int64_t ldx, int32_t M, void* y, int64_t ldy, void* workspace, int64_t workspace_bytes,
                              void* hip_stream) {
  const int rc = check_gemm8(w, M, y, ldy, workspace);
  if (rc != CCQ_OK) return rc;
  if (ldx < w->K) return CCQ_ERR_BAD_PARAM;
  if (M == 0) return CCQ_OK;
  if (!x) return CCQ_ERR_NULL;
  if (off(x, 2)) return CCQ_ERR_ALIGN;
  const int64_t need = gemm8_bf16_workspace(w, M);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CCQ_ERR_WORKSPACE;
  return launch_gemm8_bf16(w, x, ldx, M, y, ldy, workspace, hip_stream);
}

// For tests, no part of the interface: ccq_gemm8 (x without scales: ccq_gemm8_bf16) as a named plan.
extern "C" int ccq_gemm8_as(const ccq_weight8* w, const ccq_rows8* x, int32_t M, void* y, int64_t ldy, void* workspace, const int32_t* plan, void* hip_stream) {
  if (!x || !plan) return CCQ_ERR_NULL;
  int rc = check_gemm8(w, M, y, ldy, workspace);
  if (rc != CCQ_OK || M == 0) return rc;
  if (x->scales) {
    if ((rc = check_rows8(*x, w->K)) != CCQ_OK) return rc;
  } else {
    if (!x->codes) return CCQ_ERR_NULL;
    if (x->ld < w->K) return CCQ_ERR_BAD_PARAM;
    if (off(x->codes, 2)) return CCQ_ERR_ALIGN;
  }
  return launch_gemm8_as(w, x, M, y, ldy, workspace, plan, hip_stream);
}

extern "C" int ccq_rope_table(const ccq_rope_scaling* s, int32_t rows, int32_t dims, float* table, void* hip_stream) {
  if (!s || !table) return CCQ_ERR_NULL;
  if (rows < 0 || dims < 2 || dims % 2 != 0 || s->kind < 0 || s->kind > 3) return CCQ_ERR_BAD_PARAM;
  if (!(s->base > 0.0) || std::isinf(s->base) || !std::isfinite(s->magnitude)) return CCQ_ERR_BAD_PARAM;
  if (s->kind != 0 && (!(s->factor > 0.0) || std::isinf(s->factor))) return CCQ_ERR_BAD_PARAM;
  if (s->kind == 2 && dims < 4) return CCQ_ERR_BAD_PARAM;
  if (s->kind == 3 && (!(s->base > 1.0) || !(s->original_length > 0.0) || !(s->slow > 0.0) || !(s->fast >= s->slow) || std::isinf(s->original_length) || std::isinf(s->fast)))
    return CCQ_ERR_BAD_PARAM;
  if (off(table, 4)) return CCQ_ERR_ALIGN;
  if (rows == 0) return CCQ_OK;
  return launch_rope_table(s, rows, dims, table, hip_stream);
}

extern "C" int ccq_cache_append(const ccq_cache* c, const ccq_batch* b, const ccq_rope* rope, const ccq_heads* k, const ccq_heads* v, const ccq_heads* q,
                                const ccq_heads* q_out, int32_t q_heads, void* hip_stream) {
  int rc = check_cache(c);
  if (rc == CCQ_OK) rc = check_batch(b);
  if (rc != CCQ_OK) return rc;
  if (!k != !v || !q != !q_out || (!k && !q)) return CCQ_ERR_NULL;
  if (q && (q_heads < 1 || q_heads > 0x7FFFFF)) return CCQ_ERR_BAD_PARAM;
  if (rope) {
    if (rope->rows < 1 || rope->dims < 2 || rope->dims % 2 != 0 || rope->dims > c->head_dim) return CCQ_ERR_BAD_PARAM;
    if (!rope->table) return CCQ_ERR_NULL;
    if (off(rope->table, 4) || off(rope->positions, 4)) return CCQ_ERR_ALIGN;
  }
  if (nothing(b)) return CCQ_OK;
  if (k && (rc = check_cache_pointers(c)) != CCQ_OK) return rc;
  if ((rc = check_batch_pointers(b)) != CCQ_OK) return rc;
  if (k && ((rc = check_heads(k, c->kv_heads, c->head_dim)) != CCQ_OK || (rc = check_heads(v, c->kv_heads, c->head_dim)) != CCQ_OK)) return rc;
  if (q && ((rc = check_heads(q, q_heads, c->head_dim)) != CCQ_OK || (rc = check_heads(q_out, q_heads, c->head_dim)) != CCQ_OK)) return rc;
  if (q && q->data == q_out->data && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride)) return CCQ_ERR_BAD_PARAM;
  return launch_cache_append(c, b, rope, k, v, q, q_out, q_heads, hip_stream);
}

extern "C" int64_t ccq_attention_workspace_bytes(const ccq_cache* c, const ccq_batch* b, const ccq_attn* a) {
  if (check_attn(c, b, a) != CCQ_OK) return -1;
  return nothing(b) ? 0 : attention_workspace(c, b, a);
}

extern "C" int ccq_attention(const ccq_cache* c, const ccq_batch* b, const ccq_attn* a, const ccq_heads* q, const ccq_heads* out, void* workspace,
                             int64_t workspace_bytes, void* hip_stream) {
  int rc = check_attn(c, b, a);
  if (rc != CCQ_OK) return rc;
  if (nothing(b)) return CCQ_OK;
  if (!q || !out) return CCQ_ERR_NULL;
  if ((rc = check_cache_pointers(c)) != CCQ_OK || (rc = check_batch_pointers(b)) != CCQ_OK) return rc;
  if ((rc = check_heads(q, a->q_heads, c->head_dim)) != CCQ_OK || (rc = check_heads(out, a->q_heads, c->head_dim)) != CCQ_OK) return rc;
  if (off16(workspace)) return CCQ_ERR_ALIGN;
  const int64_t need = attention_workspace(c, b, a);
  if (need > 0 && (!workspace || workspace_bytes < need)) return CCQ_ERR_WORKSPACE;
  return launch_attention(c, b, a, q, out, workspace, hip_stream);
}
