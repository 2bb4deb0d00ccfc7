// The host path of the functions of routing.py: as ccq_layer_call.cpp for those of layer.py, with the same answers: outputs, a negative ccq_status
// as an int, or None for arguments that the general path has to look at.
#include "call.h"
#include "descriptor.h"

namespace {

struct Entry {
  decltype(&ccq_route) route = nullptr;
  decltype(&ccq_route_workspace_bytes) route_workspace = nullptr;
  decltype(&ccq_sort_rows) sort = nullptr;
  decltype(&ccq_sort_rows_workspace_bytes) sort_workspace = nullptr;
  decltype(&ccq_combine) combine = nullptr;
  decltype(&ccq_adapters) adapters = nullptr;
  decltype(&ccq_adapters_workspace_bytes) adapters_workspace = nullptr;
} entry;

bool small(PyObject* o, int64_t lo, int64_t hi, int32_t* out) {
  int overflow = 0;
  if (!PyLong_Check(o)) return false;
  const long v = PyLong_AsLongAndOverflow(o, &overflow);
  if (overflow || v < lo || v > hi) return false;
  *out = (int32_t)v;
  return true;
}
bool is_type(const at::Tensor* t) { return t->scalar_type() == at::kFloat || t->scalar_type() == at::kBFloat16; }
int32_t type_of(const at::Tensor* t) { return t->scalar_type() == at::kFloat ? CCQ_FP32 : CCQ_BF16; }
bool rows_of(const at::Tensor* t, at::ScalarType type) { return t && t->dim() == 2 && t->scalar_type() == type && here(t) && (t->size(1) <= 1 || t->stride(1) == 1); }
// (a single row's stride is whatever it is)
int64_t ld(const at::Tensor* t) { return t->size(0) > 1 ? t->stride(0) : std::max(t->stride(0), t->size(1)); }

// The four tensors of an order, in one piece of memory: offsets first, each from a multiple of 16 bytes on.
struct MadeOrder {
  at::Tensor rows, experts, offsets, places;
  void make(int64_t T, int64_t k, int64_t E, c10::Device device) {
    rows = at::detail::empty_cuda({T * k}, at::kInt, device, std::nullopt);
    experts = at::detail::empty_cuda({T * k}, at::kInt, device, std::nullopt);
    offsets = at::detail::empty_cuda({E + 1}, at::kInt, device, std::nullopt);
    places = at::detail::empty_cuda({T, k}, at::kInt, device, std::nullopt);
  }
  ccq_order order() const {
    return {static_cast<int32_t*>(rows.data_ptr()), static_cast<int32_t*>(experts.data_ptr()), static_cast<int32_t*>(offsets.data_ptr()),
            static_cast<int32_t*>(places.data_ptr())};
  }
};

// route(logits, top_k, scoring, bias or None, groups, top_groups, group_best, renormalize, scale, order) -> (ids, weights[, rows, experts, offsets, places])
PyObject* call_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10 || !entry.route || looked_on()) return general();
  const at::Tensor *x = tensor(a[0]), *bias = tensor(a[3]);
  if (!x || x->dim() != 2 || !is_type(x) || !here(x) || x->size(1) < 1 || (x->size(1) > 1 && x->stride(1) != 1) || x->size(0) > INT32_MAX || x->size(1) > INT32_MAX) return general();
  const int64_t T = x->size(0), E = x->size(1);
  ccq_router r = {};
  if (!small(a[1], 1, INT32_MAX, &r.top_k) || !small(a[2], 0, 1, &r.scoring) || !small(a[4], 1, INT32_MAX, &r.groups) || !small(a[5], 1, INT32_MAX, &r.top_groups) ||
      !small(a[6], 1, 2, &r.group_best) || !is_flag(a[7]) || !PyFloat_Check(a[8]) || !is_flag(a[9]))
    return general();
  if (a[3] != Py_None && (!bias || bias->dim() != 1 || bias->size(0) != E || bias->scalar_type() != at::kFloat || !here(bias) || (E > 1 && bias->stride(0) != 1))) return general();
  const bool ordered = a[9] == Py_True;
  r.T = (int32_t)T, r.experts = (int32_t)E, r.renormalize = a[7] == Py_True, r.scale = (float)PyFloat_AS_DOUBLE(a[8]);
  r.logits = x->data_ptr(), r.ld = ld(x), r.logits_type = type_of(x);
  r.bias = bias ? static_cast<const float*>(bias->data_ptr()) : nullptr;
  const int64_t need = entry.route_workspace(&r, ordered);
  if (need < 0) return general();
  at::Tensor ids, weights;
  MadeOrder made;
  Workspace ws;
  int rc;
  {
    Unlocked u;
    ids = at::detail::empty_cuda({T, r.top_k}, at::kInt, x->device(), std::nullopt);
    weights = at::detail::empty_cuda({T, r.top_k}, at::kFloat, x->device(), std::nullopt);
    r.ids = static_cast<int32_t*>(ids.data_ptr()), r.weights = static_cast<float*>(weights.data_ptr());
    ccq_order order;
    if (ordered) {
      made.make(T, r.top_k, E, x->device());
      order = made.order();
    }
    ws.make(need, x->device());
    rc = entry.route(&r, ordered ? &order : nullptr, ws.ptr, ws.bytes, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  if (!ordered) return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(ids)), THPVariable_Wrap(std::move(weights)));
  return Py_BuildValue("(NNNNNN)", THPVariable_Wrap(std::move(ids)), THPVariable_Wrap(std::move(weights)), THPVariable_Wrap(std::move(made.rows)),
                       THPVariable_Wrap(std::move(made.experts)), THPVariable_Wrap(std::move(made.offsets)), THPVariable_Wrap(std::move(made.places)));
  END_HANDLE_TH_ERRORS
}

// sort(ids, experts, first) -> (rows, experts, offsets, places)
PyObject* call_sort(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 3 || !entry.sort || looked_on()) return general();
  const at::Tensor* ids = tensor(a[0]);
  int32_t E, first;
  if (!rows_of(ids, at::kInt) || !small(a[1], 1, INT32_MAX, &E) || !small(a[2], 0, INT32_MAX, &first)) return general();
  const int64_t T = ids->size(0), k = ids->size(1);
  if (T > INT32_MAX || k > INT32_MAX) return general();
  const int64_t need = entry.sort_workspace((int32_t)T, (int32_t)k, E);
  if (need < 0) return general();
  MadeOrder made;
  Workspace ws;
  int rc;
  {
    Unlocked u;
    made.make(T, k, E, ids->device());
    const ccq_order order = made.order();
    ws.make(need, ids->device());
    rc = entry.sort(static_cast<const int32_t*>(ids->data_ptr()), ld(ids), (int32_t)T, (int32_t)k, first, E, &order, ws.ptr, ws.bytes, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("(NNNN)", THPVariable_Wrap(std::move(made.rows)), THPVariable_Wrap(std::move(made.experts)), THPVariable_Wrap(std::move(made.offsets)),
                       THPVariable_Wrap(std::move(made.places)));
  END_HANDLE_TH_ERRORS
}

// combine(rows, places, weights, base or None, out or None)
PyObject* call_combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5 || !entry.combine || looked_on()) return general();
  const at::Tensor *rows = tensor(a[0]), *places = tensor(a[1]), *weights = tensor(a[2]), *base = tensor(a[3]), *out = tensor(a[4]);
  if (!rows_of(rows, at::kBFloat16) || !rows_of(places, at::kInt) || !rows_of(weights, at::kFloat)) return general();
  const int64_t T = places->size(0), k = places->size(1), N = rows->size(1);
  if (T > INT32_MAX || k > INT32_MAX || N > INT32_MAX || rows->size(0) > INT32_MAX || weights->size(0) != T || weights->size(1) != k) return general();
  if (a[3] != Py_None && (!base || !is_type(base) || !rows_of(base, base->scalar_type()) || base->size(0) != T || base->size(1) != N)) return general();
  if (a[4] != Py_None && (!out || !is_type(out) || !rows_of(out, out->scalar_type()) || out->size(0) != T || out->size(1) != N || (T > 1 && out->stride(0) < N))) return general();
  ccq_combination c = {};
  c.T = (int32_t)T, c.k = (int32_t)k, c.N = (int32_t)N, c.P = (int32_t)rows->size(0);
  c.rows = rows->data_ptr(), c.ld_rows = ld(rows);
  c.places = static_cast<const int32_t*>(places->data_ptr()), c.ld_places = ld(places);
  c.weights = static_cast<const float*>(weights->data_ptr()), c.ld_weights = ld(weights);
  if (base) c.base = base->data_ptr(), c.ld_base = ld(base), c.base_type = type_of(base);
  at::Tensor made;
  int rc;
  {
    Unlocked u;
    if (!out) out = &(made = new_output(T, N, rows->device()));
    c.y = out->data_ptr(), c.ldy = ld(out), c.y_type = type_of(out);
    rc = entry.combine(&c, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  if (a[4] == Py_None) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[4]);
  return a[4];
  END_HANDLE_TH_ERRORS
}

// adapters(y, x, set's descriptor and GPU, order's rows and experts, out or None, workspace or None)
PyObject* call_adapters(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8 || !entry.adapters || looked_on()) return general();
  const at::Tensor *y = tensor(a[0]), *x = tensor(a[1]), *rows = tensor(a[4]), *experts = tensor(a[5]), *out = tensor(a[6]);
  const Struct<ccq_adapter_set> set(a[2]);
  if (!set.p || !here(a[3]) || !rows_of(y, at::kBFloat16) || !rows_of(x, at::kBFloat16)) return general();
  const int64_t T = x->size(0), N = set.p->N;
  if (T > INT32_MAX || x->size(1) != set.p->K || y->size(0) != T || y->size(1) != N) return general();
  for (const at::Tensor* t : {rows, experts})
    if (!t || t->dim() != 1 || t->scalar_type() != at::kInt || !here(t) || t->size(0) != T || (T > 1 && t->stride(0) != 1)) return general();
  if (a[6] != Py_None && (!rows_of(out, at::kBFloat16) || out->size(0) != T || out->size(1) != N || (T > 1 && out->stride(0) < N))) return general();
  Workspace ws;
  if (a[7] != Py_None && !ws.of(a[7], x)) return general();
  const int64_t need = a[7] == Py_None ? entry.adapters_workspace(set.p, (int32_t)T) : 0;
  if (need < 0) return general();
  at::Tensor made;
  int rc;
  {
    Unlocked u;
    if (!out) out = &(made = new_output(T, N, x->device()));
    ws.make(need, x->device());
    rc = entry.adapters(set.p, (int32_t)T, static_cast<const int32_t*>(rows->data_ptr()), static_cast<const int32_t*>(experts->data_ptr()), x->data_ptr(), ld(x), y->data_ptr(),
                        ld(y), out->data_ptr(), ld(out), ws.ptr, ws.bytes, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  if (a[6] == Py_None) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[6]);
  return a[6];
  END_HANDLE_TH_ERRORS
}

// bind(addresses of ccq_route, ccq_route_workspace_bytes, ccq_sort_rows, ccq_sort_rows_workspace_bytes, ccq_combine, ccq_adapters, ccq_adapters_workspace_bytes)
PyObject* call_bind(PyObject*, PyObject* args) {
  unsigned long long p[7];
  if (!PyArg_ParseTuple(args, "KKKKKKK", &p[0], &p[1], &p[2], &p[3], &p[4], &p[5], &p[6])) return nullptr;
  entry.route = reinterpret_cast<decltype(entry.route)>(p[0]);
  entry.route_workspace = reinterpret_cast<decltype(entry.route_workspace)>(p[1]);
  entry.sort = reinterpret_cast<decltype(entry.sort)>(p[2]);
  entry.sort_workspace = reinterpret_cast<decltype(entry.sort_workspace)>(p[3]);
  entry.combine = reinterpret_cast<decltype(entry.combine)>(p[4]);
  entry.adapters = reinterpret_cast<decltype(entry.adapters)>(p[5]);
  entry.adapters_workspace = reinterpret_cast<decltype(entry.adapters_workspace)>(p[6]);
  Py_RETURN_NONE;
}

PyCFunction fast(PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", call_bind, METH_VARARGS, "addresses of the C entry points"},
    {"route", fast(call_route), METH_FASTCALL, nullptr},
    {"sort", fast(call_sort), METH_FASTCALL, nullptr},
    {"combine", fast(call_combine), METH_FASTCALL, nullptr},
    {"adapters", fast(call_adapters), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ccq_routing", "host path of the operators of rows that choose their weights", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__ccq_routing() { return PyModule_Create(&module); }
