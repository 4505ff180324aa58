// torch_binding.cpp -- argument marshalling of the device calls for the
// Python binding: torch tensors are checked for device, dtype, shape and
// contiguity and passed to the C ABI of include/sla.h as raw device pointers,
// on the calling thread's current stream.  Each function returns the ABI's
// status code; a bad argument raises TypeError or ValueError before anything
// is launched.
//
// Native because a call's marshalling bounds every launch shorter than it:
// with tensors checked and ctypes structures filled in Python, one eager
// sla_verify took 31 us of host time against 7 us on the GPU for one sequence
// of eight nodes (conv 20 us, commit 21 us, prune 17 us).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>

#include "sla.h"

namespace {

using Dims = std::initializer_list<int64_t>;

const at::Tensor &tensor(PyObject *o, const char *name) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a torch tensor");
  return THPVariable_Unpack(o);
}

void *device_pointer(const at::Tensor &t, at::ScalarType dtype, Dims shape, const char *name) {
  TORCH_CHECK_VALUE(t.is_cuda(), name, " must live on the GPU");
  TORCH_CHECK_TYPE(t.scalar_type() == dtype, name, " must be ", dtype, ", got ", t.scalar_type());
  const at::IntArrayRef want(shape.begin(), shape.size());
  TORCH_CHECK_VALUE(t.sizes() == want, name, " has shape ", t.sizes(), ", expected ", want);
  TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
  return t.data_ptr();
}

void *pointer(PyObject *o, at::ScalarType dtype, Dims shape, const char *name) {
  return device_pointer(tensor(o, name), dtype, shape, name);
}

void *optional_pointer(PyObject *o, at::ScalarType dtype, Dims shape, const char *name) {
  return o == Py_None ? nullptr : pointer(o, dtype, shape, name);
}

const at::Tensor &sized(PyObject *o, int64_t dims, const char *name) {
  const at::Tensor &t = tensor(o, name);
  TORCH_CHECK_VALUE(t.dim() == dims, name, " must have ", dims, " dimensions, got ", t.dim());
  return t;
}

int activation_code(const at::Tensor &t) {
  TORCH_CHECK_TYPE(t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat,
                   "q/k/v must be bfloat16 or float32, got ", t.scalar_type());
  return t.scalar_type() == at::kBFloat16 ? SLA_DTYPE_BF16 : SLA_DTYPE_F32;
}

hipStream_t stream_of(const at::Tensor &t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

long number(PyObject *o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}

int32_t number32(PyObject *o, const char *name) {
  const long v = number(o);
  TORCH_CHECK_VALUE(v >= INT32_MIN && v <= INT32_MAX, name, " is out of range: ", v);
  return (int32_t)v;
}

bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}

// other Python threads run while the library enqueues (a launch can wait for
// room in the queue)
template <typename F>
int unlocked(F call) {
  PyThreadState *const ts = PyEval_SaveThread();
  const int code = call();
  PyEval_RestoreThread(ts);
  return code;
}

void count_args(Py_ssize_t got, Py_ssize_t want) {
  TORCH_CHECK_TYPE(got == want, "expected ", want, " arguments, got ", got);
}

// the four tensors of a factor store, from o[0..3]
sla_factors factors(PyObject *const *o, at::ScalarType act, int64_t B, int64_t n, int64_t H, int64_t dk, int64_t dv,
                    bool gates) {
  sla_factors f;
  f.k = pointer(o[0], act, {B, n, H, dk}, "factors.k");
  f.u = static_cast<float *>(pointer(o[1], at::kFloat, {B, n, H, dv}, "factors.u"));
  f.alpha = static_cast<float *>(gates ? pointer(o[2], at::kFloat, {B, n, H, dk}, "factors.alpha")
                                       : pointer(o[2], at::kFloat, {B, n, H}, "factors.alpha"));
  f.parent = static_cast<int32_t *>(pointer(o[3], at::kInt, {B, n}, "factors.parent"));
  return f;
}

// verify(state, q, k, v, alpha, beta, parent_idx, out, f.k, f.u, f.alpha, f.parent,
//        p.k, p.u, p.alpha, p.parent, path, len, pending, status, topology, family, route)
// pending: whether p.k .. len are a pending round's (each is then required)
PyObject *verify(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 23);
  const at::Tensor &q = sized(o[1], 4, "q");
  const at::Tensor &v = tensor(o[3], "v");
  TORCH_CHECK_VALUE(v.dim() > 0, "v has no dimensions");
  const int64_t B = q.size(0), n = q.size(1), H = q.size(2), dk = q.size(3), dv = v.size(-1);
  const at::ScalarType act = q.scalar_type();
  sla_shape shape;
  shape.batch = (int32_t)B;
  shape.heads = (int32_t)H;
  shape.d_k = (int32_t)dk;
  shape.d_v = (int32_t)dv;
  shape.n_nodes = (int32_t)n;
  shape.qkv_dtype = activation_code(q);
  shape.topology = (int32_t)number(o[20]);
  shape.family = (int32_t)number(o[21]);
  shape.route = (int32_t)number(o[22]);
  const bool gates = shape.family == SLA_FAMILY_GLA;
  const sla_factors f = factors(o + 8, act, B, n, H, dk, dv, gates);
  sla_pending pend;
  const bool pending = truth(o[18]);
  if (pending) {
    const int64_t pn = sized(o[15], 2, "pending parent").size(1);
    pend.f = factors(o + 12, act, B, pn, H, dk, dv, gates);
    pend.n_nodes = (int32_t)pn;
    pend.path = static_cast<const int32_t *>(pointer(o[16], at::kInt, {B, pn}, "pending.path"));
    pend.len = static_cast<const int32_t *>(pointer(o[17], at::kInt, {B}, "pending.len"));
  }
  int32_t *status = static_cast<int32_t *>(optional_pointer(o[19], at::kInt, {B}, "status"));
  float *state = static_cast<float *>(pointer(o[0], at::kFloat, {B, H, dk, dv}, "state"));
  const void *qp = device_pointer(q, act, {B, n, H, dk}, "q");
  const void *kp = pointer(o[2], act, {B, n, H, dk}, "k");
  const void *vp = device_pointer(v, act, {B, n, H, dv}, "v");
  const void *alpha = gates ? optional_pointer(o[4], at::kFloat, {B, n, H, dk}, "alpha")
                            : optional_pointer(o[4], at::kFloat, {B, n, H}, "alpha");
  const void *beta = optional_pointer(o[5], at::kFloat, {B, n, H}, "beta");
  const void *parent = pointer(o[6], at::kInt, {B, n}, "parent_idx");
  float *out = static_cast<float *>(pointer(o[7], at::kFloat, {B, n, H, dv}, "out"));
  const hipStream_t stream = stream_of(q);
  return PyLong_FromLong(unlocked([&] {
    return sla_verify(&shape, state, pending ? &pend : nullptr, qp, kp, vp, static_cast<const float *>(alpha),
        static_cast<const float *>(beta), static_cast<const int32_t *>(parent), out, &f, status, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// commit(state, f.k, f.u, f.alpha, f.parent, path, len, status, family)
PyObject *commit(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 9);
  const at::Tensor &k = sized(o[1], 4, "factors.k");
  const at::Tensor &u = tensor(o[2], "factors.u");
  TORCH_CHECK_VALUE(u.dim() > 0, "factors.u has no dimensions");
  const int64_t B = k.size(0), n = k.size(1), H = k.size(2), dk = k.size(3), dv = u.size(-1);
  sla_shape shape;
  shape.batch = (int32_t)B;
  shape.heads = (int32_t)H;
  shape.d_k = (int32_t)dk;
  shape.d_v = (int32_t)dv;
  shape.n_nodes = (int32_t)n;
  shape.qkv_dtype = activation_code(k);
  shape.topology = SLA_TOPO_TREE;
  shape.family = (int32_t)number(o[8]);
  shape.route = SLA_ROUTE_AUTO;
  const sla_factors f = factors(o + 1, k.scalar_type(), B, n, H, dk, dv, shape.family == SLA_FAMILY_GLA);
  int32_t *status = static_cast<int32_t *>(optional_pointer(o[7], at::kInt, {B}, "status"));
  const at::Tensor &state = tensor(o[0], "state");
  float *sp = static_cast<float *>(device_pointer(state, at::kFloat, {B, H, dk, dv}, "state"));
  const void *path = pointer(o[5], at::kInt, {B, n}, "path");
  const void *len = pointer(o[6], at::kInt, {B}, "len");
  const hipStream_t stream = stream_of(state);
  return PyLong_FromLong(unlocked([&] {
    return sla_commit(&shape, sp, &f, static_cast<const int32_t *>(path), static_cast<const int32_t *>(len), status,
        stream);
  }));
  END_HANDLE_TH_ERRORS
}

sla_conv_shape conv_shape(const at::Tensor &x, int64_t K, bool silu) {
  sla_conv_shape s;
  s.batch = (int32_t)x.size(0);
  s.channels = (int32_t)x.size(2);
  s.kernel_size = (int32_t)K;
  s.n_nodes = (int32_t)x.size(1);
  s.x_dtype = activation_code(x);
  s.activation = silu ? SLA_ACT_SILU : SLA_ACT_NONE;
  return s;
}

// conv_verify(conv_state | None, x, weight, parent_idx, y, bias | None,
//             px, pparent, path, len, pending, status, activation)
PyObject *conv_verify(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 13);
  const at::Tensor &x = sized(o[1], 3, "x");
  const at::Tensor &weight = sized(o[2], 2, "weight");
  const int64_t B = x.size(0), n = x.size(1), D = x.size(2), K = weight.size(1);
  const at::ScalarType act = x.scalar_type();
  const sla_conv_shape shape = conv_shape(x, K, truth(o[12]));
  float *cs = static_cast<float *>(optional_pointer(o[0], at::kFloat, {B, K - 1, D}, "conv_state"));
  sla_conv_pending pend;
  const bool pending = truth(o[10]);
  if (pending) {
    const int64_t pn = sized(o[7], 2, "pending parent").size(1);
    pend.x = pointer(o[6], act, {B, pn, D}, "pending.x");
    pend.parent = static_cast<const int32_t *>(pointer(o[7], at::kInt, {B, pn}, "pending.parent"));
    pend.n_nodes = (int32_t)pn;
    pend.path = static_cast<const int32_t *>(pointer(o[8], at::kInt, {B, pn}, "pending.path"));
    pend.len = static_cast<const int32_t *>(pointer(o[9], at::kInt, {B}, "pending.len"));
  }
  const void *bias = optional_pointer(o[5], at::kFloat, {D}, "bias");
  int32_t *status = static_cast<int32_t *>(optional_pointer(o[11], at::kInt, {B}, "status"));
  const void *xp = device_pointer(x, act, {B, n, D}, "x");
  const void *wp = device_pointer(weight, at::kFloat, {D, K}, "weight");
  const void *parent = pointer(o[3], at::kInt, {B, n}, "parent_idx");
  void *y = pointer(o[4], act, {B, n, D}, "y");
  const hipStream_t stream = stream_of(x);
  return PyLong_FromLong(unlocked([&] {
    return sla_conv_verify(&shape, cs, pending ? &pend : nullptr, xp, static_cast<const float *>(wp),
        static_cast<const float *>(bias), static_cast<const int32_t *>(parent), y, status, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// conv_commit(conv_state | None, x, parent_idx, path, len, kernel_size | None, status)
PyObject *conv_commit(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 7);
  const at::Tensor &x = sized(o[1], 3, "x");
  const int64_t B = x.size(0), n = x.size(1), D = x.size(2);
  const int64_t K = o[5] != Py_None ? number(o[5]) : sized(o[0], 3, "conv_state").size(1) + 1;
  const sla_conv_shape shape = conv_shape(x, K, true);
  float *cs = static_cast<float *>(optional_pointer(o[0], at::kFloat, {B, K - 1, D}, "conv_state"));
  int32_t *status = static_cast<int32_t *>(optional_pointer(o[6], at::kInt, {B}, "status"));
  const void *xp = device_pointer(x, x.scalar_type(), {B, n, D}, "x");
  const void *parent = pointer(o[2], at::kInt, {B, n}, "parent_idx");
  const void *path = pointer(o[3], at::kInt, {B, n}, "path");
  const void *len = pointer(o[4], at::kInt, {B}, "len");
  const hipStream_t stream = stream_of(x);
  return PyLong_FromLong(unlocked([&] {
    return sla_conv_commit(&shape, cs, xp, static_cast<const int32_t *>(parent), static_cast<const int32_t *>(path),
        static_cast<const int32_t *>(len), status, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// prune(parent, logp, tau, budget, with_scores) ->
//   (code, packed_parent, index_map, count, status, scores | None)
PyObject *prune(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 5);
  const at::Tensor &parent = sized(o[0], 2, "parent");
  const int64_t B = parent.size(0), n = parent.size(1);
  const double tau = PyFloat_AsDouble(o[2]);
  if (tau == -1.0 && PyErr_Occurred()) throw python_error();
  const long budget = number(o[3]);
  const bool scored = truth(o[4]);
  const void *pp = device_pointer(parent, at::kInt, {B, n}, "parent");
  const void *lp = pointer(o[1], at::kFloat, {B, n}, "logp");
  const auto ints = parent.options().dtype(at::kInt);
  const at::Tensor packed = at::empty({B, n}, ints), map = at::empty({B, n}, ints), count = at::empty({B}, ints),
                   status = at::empty({B}, ints);
  at::Tensor scores;
  if (scored) scores = at::empty({B, n}, ints.dtype(at::kFloat));
  const hipStream_t stream = stream_of(parent);
  const int code = unlocked([&] {
    return sla_prune(static_cast<const int32_t *>(pp), static_cast<const float *>(lp), (int32_t)B, (int32_t)n,
        (float)tau, (int32_t)budget, packed.data_ptr<int32_t>(), map.data_ptr<int32_t>(), count.data_ptr<int32_t>(),
            scored ? scores.data_ptr<float>() : nullptr, status.data_ptr<int32_t>(), stream);
  });
  PyObject *r = PyTuple_New(6);
  if (!r) throw python_error();
  PyTuple_SET_ITEM(r, 0, PyLong_FromLong(code));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(packed));
  PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(map));
  PyTuple_SET_ITEM(r, 3, THPVariable_Wrap(count));
  PyTuple_SET_ITEM(r, 4, THPVariable_Wrap(status));
  if (scored) {
    PyTuple_SET_ITEM(r, 5, THPVariable_Wrap(scores));
  } else {
    Py_INCREF(Py_None);
    PyTuple_SET_ITEM(r, 5, Py_None);
  }
  return r;
  END_HANDLE_TH_ERRORS
}

// A layer's pool, or several layers': [layers][pages][kv heads][page size][D].
struct Pool {
  sla_attn_shape shape;
  int32_t layers;
  void *k, *v;
  const at::Tensor *tensor;
};

Pool pool(PyObject *ko, PyObject *vo, bool layered) {
  const at::Tensor &k = tensor(ko, "k_cache");
  TORCH_CHECK_VALUE(k.dim() == 4 || (layered && k.dim() == 5), "k_cache must have ", layered ? "4 or 5" : "4",
                    " dimensions, got ", k.dim());
  const int64_t at0 = k.dim() - 4;
  Pool p = {};
  p.tensor = &k;
  p.shape.qkv_dtype = activation_code(k);
  for (int64_t i = 0; i < k.dim(); ++i)
    TORCH_CHECK_VALUE(k.size(i) <= INT32_MAX, "k_cache has shape ", k.sizes(), ", too large");
  p.layers = at0 ? (int32_t)k.size(0) : 1;
  p.shape.n_pages = (int32_t)k.size(at0);
  p.shape.kv_heads = (int32_t)k.size(at0 + 1);
  p.shape.page_size = (int32_t)k.size(at0 + 2);
  p.shape.head_dim = (int32_t)k.size(at0 + 3);
  TORCH_CHECK_VALUE(k.is_cuda(), "k_cache must live on the GPU");
  TORCH_CHECK_VALUE(k.is_contiguous(), "k_cache must be contiguous");
  const at::Tensor &v = tensor(vo, "v_cache");
  TORCH_CHECK_VALUE(v.is_cuda(), "v_cache must live on the GPU");
  TORCH_CHECK_TYPE(v.scalar_type() == k.scalar_type(), "v_cache must be ", k.scalar_type(), ", got ", v.scalar_type());
  TORCH_CHECK_VALUE(v.sizes() == k.sizes(), "v_cache has shape ", v.sizes(), ", expected ", k.sizes());
  TORCH_CHECK_VALUE(v.is_contiguous(), "v_cache must be contiguous");
  p.k = k.data_ptr();
  p.v = v.data_ptr();
  return p;
}

struct Rows {
  const int32_t *parent, *table, *len;
  int32_t *status;
};

// parent_idx [B][n], page_table [B][max_pages], cache_len [B], status [B] or None
Rows cache_rows(sla_attn_shape &s, PyObject *parent, PyObject *table, PyObject *len, PyObject *status) {
  const at::Tensor &p = sized(parent, 2, "parent_idx");
  const at::Tensor &t = sized(table, 2, "page_table");
  const int64_t B = p.size(0), n = p.size(1), pages = t.size(1);
  TORCH_CHECK_VALUE(B <= INT32_MAX && n <= INT32_MAX && pages <= INT32_MAX, "parent_idx and page_table have shapes ",
                    p.sizes(), " and ", t.sizes(), ", too large");
  s.batch = (int32_t)B;
  s.n_nodes = (int32_t)n;
  s.max_pages = (int32_t)pages;
  Rows r;
  r.parent = static_cast<const int32_t *>(device_pointer(p, at::kInt, {B, n}, "parent_idx"));
  r.table = static_cast<const int32_t *>(device_pointer(t, at::kInt, {B, pages}, "page_table"));
  r.len = static_cast<const int32_t *>(pointer(len, at::kInt, {B}, "cache_len"));
  r.status = static_cast<int32_t *>(optional_pointer(status, at::kInt, {B}, "status"));
  return r;
}

// a draft's projection [B][n][heads][D]: the heads of a node dense, the nodes a
// constant step apart (a part of a wider projection)
const void *strided(PyObject *o, at::ScalarType dtype, Dims shape, const char *name, int64_t &step) {
  const at::Tensor &t = sized(o, 4, name);
  TORCH_CHECK_VALUE(t.is_cuda(), name, " must live on the GPU");
  TORCH_CHECK_TYPE(t.scalar_type() == dtype, name, " must be ", dtype, ", got ", t.scalar_type());
  const at::IntArrayRef want(shape.begin(), shape.size());
  TORCH_CHECK_VALUE(t.sizes() == want, name, " has shape ", t.sizes(), ", expected ", want);
  const int64_t B = t.size(0), n = t.size(1), H = t.size(2), D = t.size(3);
  step = n > 1 ? t.stride(1) : B > 1 ? t.stride(0) : H * D;
  TORCH_CHECK_VALUE((D == 1 || t.stride(3) == 1) && (H == 1 || t.stride(2) == D) && (B == 1 || t.stride(0) == n * step) &&
                        step >= H * D,
                    name, " must hold each node's heads contiguously, its nodes a constant step apart; strides are ",
                    t.strides());
  return t.data_ptr();
}

// attn_append(q, k, v, parent_idx, page_table, cache_len, q_out, k_cache, v_cache, q_norm, k_norm, eps, rope, layout,
//             status, topology)
PyObject *attn_append(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 16);
  Pool c = pool(o[7], o[8], false);
  const at::ScalarType act = c.tensor->scalar_type();
  const Rows r = cache_rows(c.shape, o[3], o[4], o[5], o[14]);
  const int64_t B = c.shape.batch, n = c.shape.n_nodes, D = c.shape.head_dim, kh = c.shape.kv_heads;
  const at::Tensor &q = sized(o[0], 4, "q");
  const int64_t qh = q.size(2);
  TORCH_CHECK_VALUE(qh <= INT32_MAX, "q has shape ", q.sizes(), ", too large");
  c.shape.q_heads = (int32_t)qh;
  c.shape.topology = (int32_t)number(o[15]);
  int64_t qs, ks, vs;
  const void *qp = strided(o[0], act, {B, n, qh, D}, "q", qs);
  const void *kp = strided(o[1], act, {B, n, kh, D}, "k", ks);
  const void *vp = strided(o[2], act, {B, n, kh, D}, "v", vs);
  void *out = pointer(o[6], act, {B, n, qh, D}, "q_out");
  sla_attn_transform t = {};
  t.q_norm = static_cast<const float *>(optional_pointer(o[9], at::kFloat, {D}, "q_norm"));
  t.k_norm = static_cast<const float *>(optional_pointer(o[10], at::kFloat, {D}, "k_norm"));
  const double eps = PyFloat_AsDouble(o[11]);
  if (eps == -1.0 && PyErr_Occurred()) throw python_error();
  t.eps = (float)eps;
  if (o[12] != Py_None) {
    const at::Tensor &rope = sized(o[12], 2, "rope");
    t.rope = static_cast<const float *>(device_pointer(rope, at::kFloat, {rope.size(0), rope.size(1)}, "rope"));
    TORCH_CHECK_VALUE(rope.size(0) <= INT32_MAX && rope.size(1) <= D, "rope has shape ", rope.sizes(), ", expected [positions][up to ", D, "]");
    t.rope_len = (int32_t)rope.size(0);
    t.rope_dim = (int32_t)rope.size(1);
  }
  t.layout = (int32_t)number(o[13]);
  const hipStream_t stream = stream_of(*c.tensor);
  return PyLong_FromLong(unlocked([&] {
    return sla_attn_append(&c.shape, &t, qp, qs, kp, ks, vp, vs, r.parent, r.table, r.len, out, c.k, c.v, r.status,
        stream);
  }));
  END_HANDLE_TH_ERRORS
}

// q [B][n][q heads][D] of a verification over this pool
const void *queries(Pool &c, PyObject *qo, PyObject *max_len) {
  const at::Tensor &q = sized(qo, 4, "q");
  TORCH_CHECK_VALUE(q.size(2) <= INT32_MAX, "q has shape ", q.sizes(), ", too large");
  c.shape.q_heads = (int32_t)q.size(2);
  c.shape.max_len = number32(max_len, "max_len");
  const int64_t B = c.shape.batch, n = c.shape.n_nodes, D = c.shape.head_dim;
  return device_pointer(q, c.tensor->scalar_type(), {B, n, q.size(2), D}, "q");
}

// attn_verify(q, k_cache, v_cache, parent_idx, page_table, cache_len, out, scale | None, max_len, workspace, status, topology)
PyObject *attn_verify(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 12);
  Pool c = pool(o[1], o[2], false);
  const Rows r = cache_rows(c.shape, o[3], o[4], o[5], o[10]);
  const void *q = queries(c, o[0], o[8]);
  c.shape.topology = (int32_t)number(o[11]);
  const int64_t B = c.shape.batch, n = c.shape.n_nodes, D = c.shape.head_dim;
  void *out = pointer(o[6], c.tensor->scalar_type(), {B, n, (int64_t)c.shape.q_heads, D}, "out");
  const double scale = o[7] == Py_None ? 1.0 / std::sqrt((double)D) : PyFloat_AsDouble(o[7]);
  if (scale == -1.0 && PyErr_Occurred()) throw python_error();
  void *ws = nullptr;
  size_t bytes = 0;
  if (o[9] != Py_None) {
    const at::Tensor &w = sized(o[9], 1, "workspace");
    ws = device_pointer(w, at::kByte, {w.size(0)}, "workspace");
    bytes = (size_t)w.size(0);
  }
  const hipStream_t stream = stream_of(*c.tensor);
  return PyLong_FromLong(unlocked([&] {
    return sla_attn_verify(&c.shape, (float)scale, q, c.k, c.v, r.parent, r.table, r.len, out, ws, bytes, r.status, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// attn_workspace_bytes(batch, n, q_heads, k_cache, max_pages, max_len)
PyObject *attn_workspace_bytes(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 6);
  Pool c = pool(o[3], o[3], false);
  c.shape.batch = number32(o[0], "batch");
  c.shape.n_nodes = number32(o[1], "n_nodes");
  c.shape.q_heads = number32(o[2], "q_heads");
  c.shape.max_pages = number32(o[4], "max_pages");
  c.shape.max_len = number32(o[5], "max_len");
  return PyLong_FromSize_t(sla_attn_workspace_bytes(&c.shape));
  END_HANDLE_TH_ERRORS
}

// attn_commit(k_cache, v_cache, parent_idx, path, len, page_table, cache_len, new_len | None, status)
PyObject *attn_commit(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 9);
  Pool c = pool(o[0], o[1], true);
  const Rows r = cache_rows(c.shape, o[2], o[5], o[6], o[8]);
  const int64_t B = c.shape.batch, n = c.shape.n_nodes;
  const void *path = pointer(o[3], at::kInt, {B, n}, "path");
  const void *len = pointer(o[4], at::kInt, {B}, "len");
  void *new_len = optional_pointer(o[7], at::kInt, {B}, "new_len");
  const hipStream_t stream = stream_of(*c.tensor);
  return PyLong_FromLong(unlocked([&] {
    return sla_attn_commit(&c.shape, c.layers, c.k, c.v, r.parent, static_cast<const int32_t *>(path),
        static_cast<const int32_t *>(len), r.table, r.len, static_cast<int32_t *>(new_len), r.status, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// page_copy(k_cache, v_cache, src, dst, rows | None, status | None)
PyObject *page_copy(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 6);
  Pool c = pool(o[0], o[1], true);
  const at::Tensor &src = sized(o[2], 1, "src");
  const int64_t m = src.size(0);
  TORCH_CHECK_VALUE(m <= INT32_MAX, "src has shape ", src.sizes(), ", too large");
  const void *sp = device_pointer(src, at::kInt, {m}, "src");
  const void *dp = pointer(o[3], at::kInt, {m}, "dst");
  const void *rp = optional_pointer(o[4], at::kInt, {m}, "rows");
  void *status = optional_pointer(o[5], at::kInt, {m}, "status");
  const hipStream_t stream = stream_of(*c.tensor);
  return PyLong_FromLong(unlocked([&] {
    return sla_page_copy(&c.shape, c.layers, c.k, c.v, static_cast<const int32_t *>(sp), static_cast<const int32_t *>(dp),
        static_cast<const int32_t *>(rp), (int32_t)m, static_cast<int32_t *>(status), stream);
  }));
  END_HANDLE_TH_ERRORS
}

// The tensors of a prompt-pass call, all on the device of the first.
class Packed {
 public:
  explicit Packed(const at::Tensor &first) : device_(first.device()) {
    TORCH_CHECK_VALUE(first.is_cuda(), "the tensors must live on the GPU");
  }
  c10::Device device() const { return device_; }
  template <typename P = void>
  P *dense(PyObject *o, at::ScalarType dtype, Dims shape, const char *name) const {
    void *const p = pointer(o, dtype, shape, name);
    same(THPVariable_Unpack(o), name);
    return static_cast<P *>(p);
  }
  template <typename P = void>
  P *optional(PyObject *o, at::ScalarType dtype, Dims shape, const char *name) const {
    return o == Py_None ? nullptr : dense<P>(o, dtype, shape, name);
  }
  // [rows][..] whose rows are dense and a constant step apart (parts of a wider row)
  const void *rows(PyObject *o, at::ScalarType dtype, Dims shape, const char *name, int64_t &step) const {
    const at::Tensor &t = tensor(o, name);
    same(t, name);
    TORCH_CHECK_TYPE(t.scalar_type() == dtype, name, " must be ", dtype, ", got ", t.scalar_type());
    const at::IntArrayRef want(shape.begin(), shape.size());
    TORCH_CHECK_VALUE(t.sizes() == want, name, " has shape ", t.sizes(), ", expected ", want);
    int64_t width = 1;
    bool dense = true;
    for (int64_t d = t.dim() - 1; d > 0; --d) {
      dense = dense && (t.size(d) == 1 || t.stride(d) == width);
      width *= t.size(d);
    }
    step = t.size(0) > 1 ? t.stride(0) : width;
    TORCH_CHECK_VALUE(t.numel() == 0 || (dense && step >= width), name,
                      " must hold each row contiguously, its rows a constant step apart; strides are ", t.strides());
    if (t.numel() == 0) step = width;
    return t.data_ptr();
  }

 private:
  void same(const at::Tensor &t, const char *name) const {
    TORCH_CHECK_VALUE(t.device() == device_, name, " must live on ", device_, ", not ", t.device());
  }
  c10::Device device_;
};

int32_t size32(int64_t n, const char *name) {
  TORCH_CHECK_VALUE(n <= INT32_MAX, name, " is too large: ", n);
  return (int32_t)n;
}

float real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}

sla_prefill_shape prefill_shape(const at::Tensor &q, const at::Tensor &v, int64_t batch, int32_t family) {
  sla_prefill_shape s;
  s.tokens = size32(q.size(0), "tokens");
  s.batch = size32(batch, "batch");
  s.heads = size32(v.size(1), "heads");
  s.k_heads = size32(q.size(1), "k_heads");
  s.d_k = size32(q.size(2), "d_k");
  s.d_v = size32(v.size(2), "d_v");
  s.qkv_dtype = activation_code(q);
  s.family = family;
  return s;
}

// prefill(q, k, v, alpha | None, beta | None, seq_start, out, state_out, state | None, workspace | None, status | None,
//         family)
PyObject *prefill(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 12);
  const at::Tensor &q = sized(o[0], 3, "q"), &v = sized(o[2], 3, "v"), &starts = sized(o[5], 1, "seq_start");
  TORCH_CHECK_VALUE(starts.size(0) > 1, "seq_start has shape ", starts.sizes(), ", expected [sequences + 1]");
  const int64_t T = q.size(0), kh = q.size(1), dk = q.size(2), H = v.size(1), dv = v.size(2), B = starts.size(0) - 1;
  const at::ScalarType act = q.scalar_type();
  const sla_prefill_shape shape = prefill_shape(q, v, B, number32(o[11], "family"));
  const Packed r(q);
  int64_t qs, ks, vs;
  const void *qp = r.rows(o[0], act, {T, kh, dk}, "q", qs);
  const void *kp = r.rows(o[1], act, {T, kh, dk}, "k", ks);
  const void *vp = r.rows(o[2], act, {T, H, dv}, "v", vs);
  const float *alpha = r.optional<float>(o[3], at::kFloat, {T, H}, "alpha");
  const float *beta = r.optional<float>(o[4], at::kFloat, {T, H}, "beta");
  const int32_t *start = r.dense<int32_t>(o[5], at::kInt, {B + 1}, "seq_start");
  void *out = r.dense(o[6], act, {T, H, dv}, "out");
  float *state_out = r.dense<float>(o[7], at::kFloat, {B, H, dk, dv}, "state_out");
  const float *state = r.optional<float>(o[8], at::kFloat, {B, H, dk, dv}, "state");
  void *ws = nullptr;
  size_t bytes = 0;
  if (o[9] != Py_None) {
    bytes = (size_t)sized(o[9], 1, "workspace").size(0);
    ws = r.dense(o[9], at::kByte, {(int64_t)bytes}, "workspace");
  }
  int32_t *status = r.optional<int32_t>(o[10], at::kInt, {B}, "status");
  const c10::DeviceGuard guard(r.device());
  const hipStream_t stream = stream_of(q);
  return PyLong_FromLong(unlocked([&] {
    return sla_prefill(&shape, state, qp, qs, kp, ks, vp, vs, alpha, beta, start, out, state_out, ws, bytes, status,
        stream);
  }));
  END_HANDLE_TH_ERRORS
}

// prefill_workspace_bytes(q, v, batch, family)
PyObject *prefill_workspace_bytes(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 4);
  const at::Tensor &q = sized(o[0], 3, "q"), &v = sized(o[1], 3, "v");
  const sla_prefill_shape shape = prefill_shape(q, v, number(o[2]), number32(o[3], "family"));
  const c10::DeviceGuard guard(Packed(q).device());
  return PyLong_FromSize_t(sla_prefill_workspace_bytes(&shape));
  END_HANDLE_TH_ERRORS
}

// conv_prefill(x, weight, seq_start, y, conv_state_out | None, conv_state | None, bias | None, status | None, activation)
PyObject *conv_prefill(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 9);
  const at::Tensor &x = sized(o[0], 2, "x"), &w = sized(o[1], 2, "weight"), &starts = sized(o[2], 1, "seq_start");
  TORCH_CHECK_VALUE(starts.size(0) > 1, "seq_start has shape ", starts.sizes(), ", expected [sequences + 1]");
  const int64_t T = x.size(0), D = x.size(1), K = w.size(1), B = starts.size(0) - 1;
  const at::ScalarType act = x.scalar_type();
  sla_conv_prefill_shape shape;
  shape.tokens = size32(T, "tokens");
  shape.batch = size32(B, "batch");
  shape.channels = size32(D, "channels");
  shape.kernel_size = size32(K, "kernel_size");
  shape.x_dtype = activation_code(x);
  shape.activation = truth(o[8]) ? SLA_ACT_SILU : SLA_ACT_NONE;
  const Packed r(x);
  int64_t xs;
  const void *xp = r.rows(o[0], act, {T, D}, "x", xs);
  const float *wp = r.dense<float>(o[1], at::kFloat, {D, K}, "weight");
  const int32_t *start = r.dense<int32_t>(o[2], at::kInt, {B + 1}, "seq_start");
  void *y = r.dense(o[3], act, {T, D}, "y");
  float *state_out = r.optional<float>(o[4], at::kFloat, {B, K - 1, D}, "conv_state_out");
  const float *state = r.optional<float>(o[5], at::kFloat, {B, K - 1, D}, "conv_state");
  const float *bias = r.optional<float>(o[6], at::kFloat, {D}, "bias");
  int32_t *status = r.optional<int32_t>(o[7], at::kInt, {B}, "status");
  const c10::DeviceGuard guard(r.device());
  const hipStream_t stream = stream_of(x);
  return PyLong_FromLong(unlocked([&] {
    return sla_conv_prefill(&shape, state, xp, xs, wp, bias, start, y, state_out, status, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// recurrent_inputs(q, k, a | None, b | None, a_log | None, dt_bias | None, q_out, k_out, alpha | None, beta | None,
//                  q_scale | None, eps)
PyObject *recurrent_inputs(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 12);
  const at::Tensor &q = sized(o[0], 3, "q"), &qo = sized(o[6], 3, "q_out");
  const int64_t N = q.size(0), kh = q.size(1), dk = q.size(2), oh = qo.size(1);
  TORCH_CHECK_VALUE(kh > 0 && oh % kh == 0, "q_out has ", oh, " heads, expected a multiple of q's ", kh);
  PyObject *const gate = o[8] != Py_None ? o[8] : o[9];
  const int64_t H = gate != Py_None ? sized(gate, 2, "alpha or beta").size(1) : 1;
  const at::ScalarType act = q.scalar_type();
  sla_inputs_shape shape;
  shape.rows = size32(N, "rows");
  shape.heads = size32(H, "heads");
  shape.k_heads = size32(kh, "k_heads");
  shape.repeat = size32(oh / kh, "repeat");
  shape.d_k = size32(dk, "d_k");
  shape.dtype = activation_code(q);
  shape.q_scale = o[10] == Py_None ? (float)(1.0 / std::sqrt((double)dk)) : real(o[10]);
  shape.eps = real(o[11]);
  const Packed r(q);
  int64_t qs, ks, as = H, bs = H;
  const void *qp = r.rows(o[0], act, {N, kh, dk}, "q", qs);
  const void *kp = r.rows(o[1], act, {N, kh, dk}, "k", ks);
  const void *ap = o[2] == Py_None ? nullptr : r.rows(o[2], act, {N, H}, "a", as);
  const void *bp = o[3] == Py_None ? nullptr : r.rows(o[3], act, {N, H}, "b", bs);
  const float *a_log = r.optional<float>(o[4], at::kFloat, {H}, "a_log");
  const float *dt_bias = r.optional<float>(o[5], at::kFloat, {H}, "dt_bias");
  void *q_out = r.dense(o[6], act, {N, oh, dk}, "q_out");
  void *k_out = r.dense(o[7], act, {N, oh, dk}, "k_out");
  float *alpha = r.optional<float>(o[8], at::kFloat, {N, H}, "alpha");
  float *beta = r.optional<float>(o[9], at::kFloat, {N, H}, "beta");
  const c10::DeviceGuard guard(r.device());
  const hipStream_t stream = stream_of(q);
  return PyLong_FromLong(unlocked([&] {
    return sla_recurrent_inputs(&shape, qp, qs, kp, ks, ap, as, bp, bs, a_log, dt_bias, q_out, k_out, alpha, beta, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// gated_norm(x, z | None, weight | None, y, eps, gate)
PyObject *gated_norm(PyObject *, PyObject *const *o, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  count_args(nargs, 6);
  const at::Tensor &x = sized(o[0], 3, "x"), &y = sized(o[3], 3, "y");
  const int64_t N = x.size(0), H = x.size(1), dv = x.size(2);
  const at::ScalarType act = y.scalar_type();
  sla_norm_shape shape;
  shape.rows = size32(N, "rows");
  shape.heads = size32(H, "heads");
  shape.d_v = size32(dv, "d_v");
  shape.x_dtype = activation_code(x);
  shape.dtype = activation_code(y);
  shape.eps = real(o[4]);
  shape.gate = number32(o[5], "gate");
  const Packed r(x);
  int64_t zs = H * dv;
  const void *xp = r.dense(o[0], x.scalar_type(), {N, H, dv}, "x");
  const void *zp = o[1] == Py_None ? nullptr : r.rows(o[1], act, {N, H, dv}, "z", zs);
  const float *w = r.optional<float>(o[2], at::kFloat, {dv}, "weight");
  void *yp = r.dense(o[3], act, {N, H, dv}, "y");
  const c10::DeviceGuard guard(r.device());
  const hipStream_t stream = stream_of(x);
  return PyLong_FromLong(unlocked([&] { return sla_gated_norm(&shape, xp, zp, zs, w, yp, stream); }));
  END_HANDLE_TH_ERRORS
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
constexpr PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<verify>("verify"),
                         method<commit>("commit"),
                         method<conv_verify>("conv_verify"),
                         method<conv_commit>("conv_commit"),
                         method<prune>("prune"),
                         method<attn_append>("attn_append"),
                         method<attn_verify>("attn_verify"),
                         method<attn_workspace_bytes>("attn_workspace_bytes"),
                         method<attn_commit>("attn_commit"),
                         method<page_copy>("page_copy"),
                         method<prefill>("prefill"),
                         method<prefill_workspace_bytes>("prefill_workspace_bytes"),
                         method<conv_prefill>("conv_prefill"),
                         method<recurrent_inputs>("recurrent_inputs"),
                         method<gated_norm>("gated_norm"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Argument marshalling of libsla's device calls.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
