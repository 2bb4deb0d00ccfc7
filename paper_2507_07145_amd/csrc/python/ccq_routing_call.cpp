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

// Tensors in one piece of memory, each from a multiple of 16 bytes on: one allocation costs the host what each of six would.
class Pieces {
 public:
  int64_t add(int64_t bytes) {
    const int64_t at = bytes_;
    bytes_ += (bytes + 15) / 16 * 16;
    return at;
  }
  void make(c10::Device device) { held_ = at::detail::empty_cuda({std::max<int64_t>(bytes_, 16)}, at::kByte, device, std::nullopt); }
  void* at(int64_t offset) const { return static_cast<char*>(held_.data_ptr()) + offset; }
  PyObject* tensor(int64_t offset, at::ScalarType type, at::IntArrayRef sizes) const {
    auto impl = c10::make_intrusive<at::TensorImpl>(c10::Storage(held_.storage()), held_.key_set(), c10::scalarTypeToTypeMeta(type));
    impl->set_storage_offset(offset / 4);   // (all are of four bytes)
    impl->set_sizes_contiguous(sizes);
    return THPVariable_Wrap(at::Tensor(std::move(impl)));
  }

 private:
  at::Tensor held_;
  int64_t bytes_ = 0;
};

// The four tensors of an order among them.
struct MadeOrder {
  int64_t T, k, E, rows, experts, offsets, places;
  MadeOrder(Pieces& p, int64_t T_, int64_t k_, int64_t E_) : T(T_), k(k_), E(E_) {
    rows = p.add(T * k * 4), experts = p.add(T * k * 4), offsets = p.add((E + 1) * 4), places = p.add(T * k * 4);
  }
  ccq_order order(const Pieces& p) const {
    return {static_cast<int32_t*>(p.at(rows)), static_cast<int32_t*>(p.at(experts)), static_cast<int32_t*>(p.at(offsets)), static_cast<int32_t*>(p.at(places))};
  }
  // new references, or an exception and NULL for what could not be made
  void tensors(const Pieces& p, PyObject* (&out)[4]) const {
    out[0] = p.tensor(rows, at::kInt, {T * k});
    out[1] = p.tensor(experts, at::kInt, {T * k});
    out[2] = p.tensor(offsets, at::kInt, {E + 1});
    out[3] = p.tensor(places, at::kInt, {T, k});
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
  Pieces pieces;
  const int64_t ids = pieces.add(T * r.top_k * 4), weights = pieces.add(T * r.top_k * 4);
  std::optional<MadeOrder> made;
  if (ordered) made.emplace(pieces, T, r.top_k, E);
  Workspace ws;
  int rc;
  {
    Unlocked u;
    pieces.make(x->device());
    r.ids = static_cast<int32_t*>(pieces.at(ids)), r.weights = static_cast<float*>(pieces.at(weights));
    ccq_order order;
    if (ordered) order = made->order(pieces);
    ws.make(need, x->device());
    rc = entry.route(&r, ordered ? &order : nullptr, ws.ptr, ws.bytes, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  PyObject *made_ids = pieces.tensor(ids, at::kInt, {T, r.top_k}), *made_weights = pieces.tensor(weights, at::kFloat, {T, r.top_k});
  if (!ordered) return Py_BuildValue("(NN)", made_ids, made_weights);
  PyObject* o[4];
  made->tensors(pieces, o);
  return Py_BuildValue("(NNNNNN)", made_ids, made_weights, o[0], o[1], o[2], o[3]);
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
  Pieces pieces;
  const MadeOrder made(pieces, T, k, E);
  Workspace ws;
  int rc;
  {
    Unlocked u;
    pieces.make(ids->device());
    const ccq_order order = made.order(pieces);
    ws.make(need, ids->device());
    rc = entry.sort(static_cast<const int32_t*>(ids->data_ptr()), ld(ids), (int32_t)T, (int32_t)k, first, E, &order, ws.ptr, ws.bytes, current_stream());
  }
  if (rc != CCQ_OK) return PyLong_FromLong(rc);
  PyObject* o[4];
  made.tensors(pieces, o);
  return Py_BuildValue("(NNNN)", o[0], o[1], o[2], o[3]);
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
