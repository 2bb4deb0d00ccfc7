// The host path of the functions of layer.py: as ccq_call.cpp for the multiply calls, with the same answers: outputs, a
// negative ccq_status as an int, or None for arguments that the general path has to look at.
#include "call.h"
#include "descriptor.h"

namespace {

struct Entry {
  decltype(&ccq_rms_norm) norm = nullptr;
  decltype(&ccq_quantize8) quantize = nullptr;
  decltype(&ccq_gemm8) gemm = nullptr;
  decltype(&ccq_gemm8_workspace_bytes) gemm_workspace = nullptr;
  decltype(&ccq_gemm8_bf16) gemm_bf16 = nullptr;
  decltype(&ccq_gemm8_bf16_workspace_bytes) gemm_bf16_workspace = nullptr;
  decltype(&ccq_cache_append) append = nullptr;
  decltype(&ccq_attention) attention = nullptr;
  decltype(&ccq_attention_workspace_bytes) attention_workspace = nullptr;
} entry;

bool is_codes(const at::Tensor* t) { return t->scalar_type() == at::kByte || t->scalar_type() == at::kFloat8_e4m3fn; }
bool is_scales(const at::Tensor* t) { return t->scalar_type() == at::kByte || t->scalar_type() == at::kFloat8_e8m0fnu; }
bool rows_like(const at::Tensor* t, const at::Tensor* x) {
  return t && t->dim() == 2 && t->device() == x->device() && t->size(0) == x->size(0) && t->size(1) == x->size(1) && t->stride(1) == 1;
}
// (a single row's stride is whatever it is; a row is at least as far from the next as it is long)
int64_t ld(const at::Tensor* t) { return t->size(0) > 1 ? t->stride(0) : std::max(t->stride(0), (t->size(1) + 15) / 16 * 16); }
int32_t type_of(const at::Tensor* t) { return t->scalar_type() == at::kFloat ? CCQ_FP32 : CCQ_BF16; }
bool is_type(const at::Tensor* t) { return t->scalar_type() == at::kFloat || t->scalar_type() == at::kBFloat16; }

struct Made8 {
  at::Tensor codes, scales;
  void make(int64_t M, int64_t N, c10::Device device) {
    const int64_t wide = (N + 15) / 16 * 16;
    codes = at::detail::empty_cuda({M, wide}, at::kByte, device, std::nullopt);
    if (wide != N) {
      const int64_t size[2] = {M, N}, stride[2] = {wide, 1};
      codes.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef(size, 2), at::IntArrayRef(stride, 2));
    }
    scales = at::detail::empty_cuda({M, (N + 127) / 128}, at::kByte, device, std::nullopt);
  }
  ccq_rows8 rows() const { return {codes.data_ptr(), codes.stride(0), static_cast<uint8_t*>(scales.data_ptr()), scales.stride(0)}; }
  PyObject* pair() { return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(codes)), THPVariable_Wrap(std::move(scales))); }
};

// rms_norm(x, weight or None, eps, residual or None, residual_out or None, out or None, rows8)
PyObject* call_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 || !entry.norm || looked_on()) return general();
  const at::Tensor *x = tensor(a[0]), *w = tensor(a[1]), *r = tensor(a[3]), *sum = tensor(a[4]), *y = tensor(a[5]);
  if (!plain_bf16(x) || !here(x) || !PyFloat_Check(a[2]) || !is_flag(a[6])) return general();
  const int64_t M = x->size(0), N = x->size(1);
  if (M > INT32_MAX || N > INT32_MAX || N < 1) return general();
  if (a[1] != Py_None && (!w || w->dim() != 1 || w->size(0) != N || w->device() != x->device() || !is_type(w) || (N > 1 && w->stride(0) != 1))) return general();
  if (a[3] != Py_None && (!rows_like(r, x) || !is_type(r))) return general();
  if (a[4] != Py_None && (!r || !rows_like(sum, x) || sum->scalar_type() != r->scalar_type())) return general();
  if (a[5] != Py_None && (!rows_like(y, x) || y->scalar_type() != at::kBFloat16)) return general();
  const bool rows8 = a[6] == Py_True;
  if (!sum) sum = r;
  ccq_norm c = {};
  c.M = (int32_t)M, c.N = (int32_t)N, c.eps = (float)PyFloat_AS_DOUBLE(a[2]);
  c.x = x->data_ptr(), c.ldx = ld(x);
  if (w) c.weight = w->data_ptr(), c.weight_type = type_of(w);
  if (r) c.residual = r->data_ptr(), c.ld_residual = ld(r), c.sum = sum->data_ptr(), c.ld_sum = ld(sum), c.residual_type = type_of(r);
  at::Tensor made;
  Made8 made8;
  int rc;
  {
    Unlocked u;
    if (!y && !rows8) y = &(made = new_output(M, N, x->device()));
    if (y) c.y = y->data_ptr(), c.ldy = ld(y);
    if (rows8) {
      made8.make(M, N, x->device());
      c.y8 = made8.rows();
    }
    rc = entry.norm(&c, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  if (rows8) return made8.pair();
  if (a[5] == Py_None) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[5]);
  return a[5];
  END_HANDLE_TH_ERRORS
}

// quantize8(x)
PyObject* call_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 1 || !entry.quantize || looked_on()) return general();
  const at::Tensor* x = tensor(a[0]);
  if (!plain_bf16(x) || !here(x) || x->size(0) > INT32_MAX || x->size(1) > INT32_MAX || x->size(1) < 1) return general();
  Made8 made8;
  int rc;
  {
    Unlocked u;
    made8.make(x->size(0), x->size(1), x->device());
    const ccq_rows8 rows = made8.rows();
    rc = entry.quantize(x->data_ptr(), ld(x), (int32_t)x->size(0), (int32_t)x->size(1), &rows, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  return made8.pair();
  END_HANDLE_TH_ERRORS
}

// gemm8(weight's descriptor, its GPU, x (bf16) or codes, None or scales, out or None, workspace or None)
PyObject* call_gemm8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6 || !entry.gemm || looked_on()) return general();
  const Struct<ccq_weight8> w(a[0]);
  const at::Tensor *x = tensor(a[2]), *scales = tensor(a[3]), *y = tensor(a[4]);
  if (!w.p || !here(a[1]) || !x || x->dim() != 2 || !here(x) || x->size(1) != w.p->K || x->stride(1) != 1) return general();
  const int64_t M = x->size(0);
  if (M > INT32_MAX) return general();
  const bool wide = a[3] == Py_None;
  if (wide ? x->scalar_type() != at::kBFloat16
           : !is_codes(x) || !scales || scales->dim() != 2 || !is_scales(scales) || scales->device() != x->device() || scales->size(0) != M ||
                 scales->size(1) != (w.p->K + 127) / 128 || (scales->size(1) > 1 && scales->stride(1) != 1))
    return general();
  if (a[4] != Py_None && (!plain_bf16(y) || y->device() != x->device() || y->size(0) != M || y->size(1) != w.p->N)) return general();
  Workspace ws;
  if (a[5] != Py_None && !ws.of(a[5], x)) return general();
  const int64_t need = a[5] != Py_None ? 0 : wide ? entry.gemm_bf16_workspace(w.p, (int32_t)M) : entry.gemm_workspace(w.p, (int32_t)M);
  if (need < 0) return general();
  at::Tensor made;
  int rc;
  {
    Unlocked u;
    if (!y) y = &(made = new_output(M, w.p->N, x->device()));
    ws.make(need, x->device());
    const int64_t ldy = a[4] == Py_None || M > 1 ? y->stride(0) : (w.p->N + 7) / 8 * 8;
    if (wide) {
      rc = entry.gemm_bf16(w.p, x->data_ptr(), ld(x), (int32_t)M, y->data_ptr(), ldy, ws.ptr, ws.bytes, current_stream());
    } else {
      const int64_t ld_scales = M > 1 ? scales->stride(0) : std::max(scales->stride(0), scales->size(1));
      const ccq_rows8 rows = {x->data_ptr(), ld(x), static_cast<uint8_t*>(scales->data_ptr()), ld_scales};
      rc = entry.gemm(w.p, &rows, (int32_t)M, y->data_ptr(), ldy, ws.ptr, ws.bytes, current_stream());
    }
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  if (a[4] == Py_None) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[4]);
  return a[4];
  END_HANDLE_TH_ERRORS
}

// bf16 [tokens][heads][dim]
bool heads_of(const at::Tensor* t, int64_t tokens, int64_t heads, int64_t dim, ccq_heads* out) {
  if (!t || t->dim() != 3 || t->scalar_type() != at::kBFloat16 || !here(t) || t->size(0) != tokens || t->size(2) != dim || t->stride(2) != 1) return false;
  if (heads > 0 && t->size(1) != heads) return false;
  const int64_t n = t->size(1), head = n > 1 ? t->stride(1) : dim;
  *out = {t->data_ptr(), tokens > 1 ? t->stride(0) : std::max(t->stride(0), (n - 1) * head + dim), head};
  return true;
}
at::Tensor new_heads(const at::Tensor* like) {
  return at::detail::empty_cuda(like->sizes(), at::kBFloat16, like->device(), std::nullopt);
}

// append(cache's descriptor and GPU, batch's, k or None, v or None, q or None, q_out or None, rope's descriptor or None, its GPU)
PyObject* call_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10 || !entry.append || looked_on()) return general();
  const Struct<ccq_cache> c(a[0]);
  const Struct<ccq_batch> b(a[2]);
  std::optional<Struct<ccq_rope>> rope;
  if (a[8] != Py_None) rope.emplace(a[8]);
  if (!here(a[1]) || !here(a[3]) || !here(a[9]) || !c.p || !b.p || (rope && !rope->p)) return general();
  const at::Tensor *k = tensor(a[4]), *v = tensor(a[5]), *q = tensor(a[6]), *out = tensor(a[7]);
  ccq_heads hk, hv, hq, ho;
  const int64_t T = b.p->tokens, D = c.p->head_dim;
  if (a[4] != Py_None && !heads_of(k, T, c.p->kv_heads, D, &hk)) return general();
  if (a[5] != Py_None && !heads_of(v, T, c.p->kv_heads, D, &hv)) return general();
  if (a[6] != Py_None && (!heads_of(q, T, 0, D, &hq) || q->size(1) > INT32_MAX)) return general();
  if (a[7] != Py_None && (!q || !heads_of(out, T, q->size(1), D, &ho))) return general();
  at::Tensor made;
  int rc;
  {
    Unlocked u;
    if (q && !out) {
      made = new_heads(q);
      heads_of(&made, T, q->size(1), D, &ho);
    }
    rc = entry.append(c.p, b.p, rope ? rope->p : nullptr, k ? &hk : nullptr, v ? &hv : nullptr, q ? &hq : nullptr, q ? &ho : nullptr, q ? (int32_t)q->size(1) : 0,
                      current_stream());
  }
  if (rc != CCQ_OK || !q) return PyLong_FromLong(rc);
  if (a[7] == Py_None) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[7]);
  return a[7];
  END_HANDLE_TH_ERRORS
}

// attention(cache's descriptor and GPU, batch's, q, scale, window, causal, out or None, workspace or None)
PyObject* call_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10 || !entry.attention || looked_on()) return general();
  const Struct<ccq_cache> c(a[0]);
  const Struct<ccq_batch> b(a[2]);
  const at::Tensor *q = tensor(a[4]), *out = tensor(a[8]);
  ccq_heads hq, ho;
  if (!here(a[1]) || !here(a[3]) || !c.p || !b.p || !heads_of(q, b.p->tokens, 0, c.p->head_dim, &hq) || q->size(1) > INT32_MAX) return general();
  if (!PyFloat_Check(a[5]) || !PyLong_Check(a[6]) || !is_flag(a[7])) return general();
  int overflow = 0;
  const long window = PyLong_AsLongAndOverflow(a[6], &overflow);
  if (overflow || window < 0 || window > INT32_MAX) return general();
  if (a[8] != Py_None && !heads_of(out, b.p->tokens, q->size(1), c.p->head_dim, &ho)) return general();
  ccq_attn at = {(int32_t)q->size(1), a[7] == Py_True, (int32_t)window, (float)PyFloat_AS_DOUBLE(a[5])};
  Workspace ws;
  if (a[9] != Py_None && !ws.of(a[9], q)) return general();
  const int64_t need = a[9] == Py_None ? entry.attention_workspace(c.p, b.p, &at) : 0;
  if (need < 0) return general();
  at::Tensor made;
  int rc;
  {
    Unlocked u;
    if (!out) {
      made = new_heads(q);
      heads_of(&made, b.p->tokens, q->size(1), c.p->head_dim, &ho);
    }
    ws.make(need, q->device());
    rc = entry.attention(c.p, b.p, &at, &hq, &ho, ws.ptr, ws.bytes, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  if (a[8] == Py_None) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[8]);
  return a[8];
  END_HANDLE_TH_ERRORS
}

// bind(addresses of ccq_rms_norm, ccq_quantize8, ccq_gemm8, ccq_gemm8_workspace_bytes, ccq_cache_append, ccq_attention,
// ccq_attention_workspace_bytes, ccq_gemm8_bf16, ccq_gemm8_bf16_workspace_bytes)
PyObject* call_bind(PyObject*, PyObject* args) {
  unsigned long long p[9];
  if (!PyArg_ParseTuple(args, "KKKKKKKKK", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6], &p[7], &p[8])) return nullptr;
  entry.norm = reinterpret_cast<decltype(entry.norm)>(p[0]);
  entry.quantize = reinterpret_cast<decltype(entry.quantize)>(p[1]);
  entry.gemm = reinterpret_cast<decltype(entry.gemm)>(p[2]);
  entry.gemm_workspace = reinterpret_cast<decltype(entry.gemm_workspace)>(p[3]);
  entry.append = reinterpret_cast<decltype(entry.append)>(p[4]);
  entry.attention = reinterpret_cast<decltype(entry.attention)>(p[5]);
  entry.attention_workspace = reinterpret_cast<decltype(entry.attention_workspace)>(p[6]);
  entry.gemm_bf16 = reinterpret_cast<decltype(entry.gemm_bf16)>(p[7]);
  entry.gemm_bf16_workspace = reinterpret_cast<decltype(entry.gemm_bf16_workspace)>(p[8]);
  Py_RETURN_NONE;
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", call_bind, METH_VARARGS, "addresses of the C entry points"},
    {"rms_norm", fast(call_norm), METH_FASTCALL, nullptr},
    {"quantize8", fast(call_quantize), METH_FASTCALL, nullptr},
    {"gemm8", fast(call_gemm8), METH_FASTCALL, nullptr},
    {"append", fast(call_append), METH_FASTCALL, nullptr},
    {"attention", fast(call_attention), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ccq_layer", "host path of the layer operators", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__ccq_layer() { return PyModule_Create(&module); }
