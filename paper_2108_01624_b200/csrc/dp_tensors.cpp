// CPython module _dp_tensors: torch tensors into the C ABI of include/dp.h for the calls on small tensors (global norm,
// rows, relative position bias, query/key norms), where reading a tensor's address, sizes and strides from Python takes
// several times as long as the launch.  Argument marshalling only: every function checks its tensors, fills the
// descriptors and calls the entry point whose address bind() was given, on the current stream of the tensors' device (or
// the stream it is handed).  A tensor that does not fit raises ValueError before anything is launched; the entry point's
// status is returned.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "../../include/dp.h"

namespace {

struct Refused {                  // becomes a ValueError
  std::string what;
};
struct Raised {};                 // a Python error is already set

struct Api {
  decltype(&dp_global_sqnorm) global_sqnorm;
  decltype(&dp_clip_by_global_norm) clip_by_global_norm;
  decltype(&dp_clip_adamw_step) clip_adamw_step;
  decltype(&dp_rows_sqnorms) rows_sqnorms;
  decltype(&dp_rows_clipped_accumulate) rows_clipped_accumulate;
  decltype(&dp_relpos_bias) relpos_bias;
  decltype(&dp_relpos_workspace_bytes) relpos_workspace_bytes;
  decltype(&dp_relpos_bias_grad) relpos_bias_grad;
  decltype(&dp_qknorm_rope) qknorm_rope;
  decltype(&dp_qknorm_workspace_bytes) qknorm_workspace_bytes;
  decltype(&dp_qknorm_rope_backward) qknorm_rope_backward;
};
Api api = {};

// ---- arguments ------------------------------------------------------------------------------------------------------
const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refused{std::string(what) + ": tensor expected"};
  return THPVariable_Unpack(o);
}
double number(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Raised{};
  return x;
}
int64_t integer(PyObject* o) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Raised{};
  return x;
}
int32_t small_integer(PyObject* o, const char* what) {
  const int64_t x = integer(o);
  if (x < INT32_MIN || x > INT32_MAX) throw Refused{std::string(what) + ": out of range"};
  return (int32_t)x;
}
int truth(PyObject* o) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw Raised{};
  return x;
}

std::string shape_text(c10::IntArrayRef s) {
  std::string t = "[";
  for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + "]";
}

int dp_dtype_of(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kFloat) return DP_F32;
  if (t.scalar_type() == at::kBFloat16) return DP_BF16;
  throw Refused{std::string(what) + ": fp32 or bf16 tensor expected"};
}

// The device that a call's first tensor is on; later ones are held to it.
int device_of(const at::Tensor& t, const char* what) {
  if (!t.is_cuda()) throw Refused{std::string(what) + ": device tensor expected"};
  return t.get_device();
}
void on_device(const at::Tensor& t, int device, const char* what) {
  if (!t.is_cuda() || t.get_device() != device)
    throw Refused{std::string(what) + ": not on the device of the other tensors, cuda:" + std::to_string(device)};
}

// Address of an optional dense argument (None: null) after the checks that every argument gets.
void* dense(PyObject* o, int device, at::ScalarType type, const char* what, int64_t numel = -1, c10::IntArrayRef shape = {}) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  on_device(t, device, what);
  if (t.scalar_type() != type) throw Refused{std::string(what) + ": " + c10::toString(type) + " expected"};
  if (!t.is_contiguous()) throw Refused{std::string(what) + ": contiguous tensor expected"};
  if (numel >= 0 && t.numel() != numel)
    throw Refused{std::string(what) + ": " + std::to_string(numel) + " elements expected, got " + std::to_string(t.numel())};
  if (!shape.empty() && t.sizes() != shape)
    throw Refused{std::string(what) + ": shape " + shape_text(shape) + " expected, got " + shape_text(t.sizes())};
  return t.data_ptr();
}

struct Workspace { void* p = nullptr; size_t n = 0; };
Workspace workspace_of(PyObject* o, int device) {
  Workspace w;
  if (o == Py_None) return w;
  const at::Tensor& t = tensor(o, "workspace");
  on_device(t, device, "workspace");
  if (!t.is_contiguous()) throw Refused{"workspace: contiguous tensor expected"};
  w.p = t.data_ptr();
  w.n = t.nbytes();
  return w;
}

// The stream to launch on (None: the device's current one), with the device made current while it lives: a launch goes to
// the current device.
struct On {
  c10::cuda::CUDAGuard guard;
  void* stream;
  On(int device, PyObject* given) : guard((c10::DeviceIndex)device) {
    if (given == Py_None) stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    else stream = reinterpret_cast<void*>((uintptr_t)integer(given));
  }
};

// Addresses and sizes of a list of dense tensors of one dtype on one device.
struct List {
  std::vector<void*> address;
  std::vector<int64_t> size;
  int dtype = DP_F32, device = -1;
  List(PyObject* seq) {
    PyObject* fast = PySequence_Fast(seq, "a sequence of tensors expected");
    if (!fast) throw Raised{};
    try {
      const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
      PyObject** items = PySequence_Fast_ITEMS(fast);
      address.resize(n);
      size.resize(n);
      for (Py_ssize_t k = 0; k < n; ++k) {
        const at::Tensor& t = tensor(items[k], "tensors");
        if (k == 0) {
          device = device_of(t, "tensors");
          dtype = dp_dtype_of(t, "tensors");
        } else if (!t.is_cuda() || t.get_device() != device || dp_dtype_of(t, "tensors") != dtype) {
          throw Refused{"the tensors of a list share one dtype and one device"};
        }
        if (!t.is_contiguous()) throw Refused{"contiguous tensor expected"};
        address[k] = t.data_ptr();
        size[k] = t.numel();
      }
    } catch (...) {
      Py_DECREF(fast);
      throw;
    }
    Py_DECREF(fast);
  }
};

// ---- calls ------------------------------------------------------------------------------------------------------------
using Args = PyObject* const*;

int global_sqnorm(Args a) {       // tensors, sqsum, accumulate_into, workspace, stream
  const List L(a[0]);
  const int device = L.device >= 0 ? L.device : device_of(tensor(a[1], "sqsum"), "sqsum");
  auto* out = static_cast<double*>(dense(a[1], device, at::kDouble, "sqsum", 1));
  const Workspace w = workspace_of(a[3], device);
  const On on(device, a[4]);
  return api.global_sqnorm(L.address.data(), L.size.data(), (int)L.size.size(), L.dtype, truth(a[2]), out, w.p, w.n, on.stream);
}

int clip_by_global_norm(Args a) {  // tensors, outs or None, sqsum, max_norm, norm_and_factor, stream
  List L(a[0]);
  if (L.size.empty()) throw Refused{"at least one tensor expected"};
  void* const* outs = L.address.data();
  std::vector<void*> other;
  if (a[1] != Py_None) {
    List O(a[1]);
    if (O.size != L.size || O.dtype != L.dtype || O.device != L.device)
      throw Refused{"outputs must have their tensors' number, sizes, dtype and device"};
    other = std::move(O.address);
    outs = other.data();
  }
  auto* sqsum = static_cast<double*>(dense(a[2], L.device, at::kDouble, "sqsum", 1));
  auto* told = static_cast<float*>(dense(a[4], L.device, at::kFloat, "norm_and_factor", 2));
  const On on(L.device, a[5]);
  return api.clip_by_global_norm(L.address.data(), outs, L.size.data(), (int)L.size.size(), L.dtype, sqsum, number(a[3]),
                                 told, on.stream);
}

int clip_adamw_step(Args a) {     // theta, m, v, g, zero_g, sqsum, max_norm, lr, beta1, beta2, xi, weight_decay, t, stream
  const at::Tensor& theta = tensor(a[0], "theta");
  const int device = device_of(theta, "theta");
  const int64_t n = theta.numel();
  const char* names[4] = {"theta", "m", "v", "g"};
  float* p[4];
  for (int k = 0; k < 4; ++k) {
    if (a[k] == Py_None) throw Refused{std::string(names[k]) + ": tensor expected"};
    p[k] = static_cast<float*>(dense(a[k], device, at::kFloat, names[k], n));
  }
  auto* sqsum = static_cast<double*>(dense(a[5], device, at::kDouble, "sqsum", 1));
  const On on(device, a[13]);
  return api.clip_adamw_step(p[0], p[1], p[2], p[3], truth(a[4]), n, sqsum, number(a[6]), number(a[7]), number(a[8]),
                             number(a[9]), number(a[10]), number(a[11]), integer(a[12]), on.stream);
}

// Rows descriptors live in a bytes object: (device, B, descriptors).
PyObject* rows_list(Args a) {     // sequence of (gradients, accumulator or None)
  PyObject* fast = PySequence_Fast(a[0], "a sequence of pairs expected");
  if (!fast) throw Raised{};
  PyObject* out = nullptr;
  try {
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
    if (n == 0) throw Refused{"at least one tensor expected"};
    std::vector<dp_rows> rows(n);
    int device = -1;
    int64_t B = 0;
    for (Py_ssize_t k = 0; k < n; ++k) {
      PyObject* pair = PySequence_Fast_GET_ITEM(fast, k);
      if (!PyTuple_Check(pair) || PyTuple_GET_SIZE(pair) != 2) throw Refused{"(gradients, accumulator) pairs expected"};
      PyObject *g = PyTuple_GET_ITEM(pair, 0), *acc = PyTuple_GET_ITEM(pair, 1);
      const at::Tensor& t = tensor(g, "per-example gradients");
      if (t.dim() < 1) throw Refused{"per-example gradients: [B, ...] expected"};
      if (k == 0) {
        device = device_of(t, "per-example gradients");
        B = t.size(0);
        if (B > INT32_MAX) throw Refused{"per-example gradients: too many examples"};
      } else if (t.size(0) != B) {
        throw Refused{"the tensors of a list share the number of examples"};
      }
      rows[k].grad = static_cast<float*>(dense(g, device, at::kFloat, "per-example gradients"));
      rows[k].width = B ? t.numel() / B : 0;
      if (acc != Py_None && tensor(acc, "accumulator").sizes() != t.sizes().slice(1))
        throw Refused{"accumulator: shape " + shape_text(t.sizes().slice(1)) + " expected, got " + shape_text(tensor(acc, "accumulator").sizes())};
      rows[k].acc = static_cast<float*>(dense(acc, device, at::kFloat, "accumulator"));
    }
    out = Py_BuildValue("(iLy#)", device, (long long)B, reinterpret_cast<const char*>(rows.data()),
                        (Py_ssize_t)(n * sizeof(dp_rows)));
  } catch (...) {
    Py_DECREF(fast);
    throw;
  }
  Py_DECREF(fast);
  if (!out) throw Raised{};
  return out;
}
struct Rows { int device, B, n; const dp_rows* p; };
Rows rows_of(PyObject* o) {       // what rows_list returned
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3 || !PyBytes_Check(PyTuple_GET_ITEM(o, 2))) throw Refused{"row list expected"};
  PyObject* bytes = PyTuple_GET_ITEM(o, 2);
  return {(int)integer(PyTuple_GET_ITEM(o, 0)), (int)integer(PyTuple_GET_ITEM(o, 1)),
          (int)(PyBytes_GET_SIZE(bytes) / (Py_ssize_t)sizeof(dp_rows)), reinterpret_cast<const dp_rows*>(PyBytes_AS_STRING(bytes))};
}
int rows_sqnorms(Args a) {        // rows, sqnorm, accumulate_into, stream
  const Rows r = rows_of(a[0]);
  auto* sqnorm = static_cast<float*>(dense(a[1], r.device, at::kFloat, "sqnorm", r.B));
  const On on(r.device, a[3]);
  return api.rows_sqnorms(r.p, r.n, r.B, sqnorm, truth(a[2]), on.stream);
}
int rows_clipped_accumulate(Args a) {  // rows, clip, stream
  const Rows r = rows_of(a[0]);
  auto* clip = static_cast<float*>(dense(a[1], r.device, at::kFloat, "clip", r.B));
  const On on(r.device, a[2]);
  return api.rows_clipped_accumulate(r.p, r.n, r.B, clip, on.stream);
}

int32_t extent(int64_t n) { return n > INT32_MAX ? -1 : (int32_t)n; }     // -1 is refused by the entry point

int relpos_bias(Args a) {         // table, out, max_distance, bidirectional, offset, stream
  const at::Tensor &table = tensor(a[0], "table"), &out = tensor(a[1], "out");
  const int device = device_of(table, "table");
  on_device(out, device, "out");
  if (table.dim() != 2 || !table.is_contiguous()) throw Refused{"table: contiguous [num_buckets, heads] expected"};
  if (out.dim() != 3 || out.size(0) != table.size(1))
    throw Refused{"out: [" + std::to_string(table.size(1)) + ", Tq, Tk] expected, got " + shape_text(out.sizes())};
  if (out.size(2) > 1 && out.stride(2) != 1) throw Refused{"out: unit stride along the keys expected"};
  const dp_relpos p = {extent(table.size(0)), small_integer(a[2], "max_distance"), truth(a[3]), extent(table.size(1)),
                       extent(out.size(1)), extent(out.size(2)), integer(a[4])};
  const On on(device, a[5]);
  return api.relpos_bias(&p, table.data_ptr(), dp_dtype_of(table, "table"), out.data_ptr(), dp_dtype_of(out, "out"),
                         out.size(0) > 1 ? out.stride(0) : 0, out.size(1) > 1 ? out.stride(1) : out.size(2), on.stream);
}

PyObject* relpos_workspace_bytes(Args a) {   // G, num_buckets
  const at::Tensor& G = tensor(a[0], "G");
  if (G.dim() != 4) throw Refused{"G: [B, heads, Tq, Tk] expected"};
  // the size depends on neither the distances nor the sides: one side and a distance that is always valid
  const int32_t nb = small_integer(a[1], "num_buckets");
  const dp_relpos p = {nb, nb < (1 << 20) ? nb + 1 : nb, 0, extent(G.size(1)), extent(G.size(2)), extent(G.size(3)), 0};
  const size_t n = api.relpos_workspace_bytes(&p, extent(G.size(0)));
  return PyLong_FromSize_t(n < 256 ? 256 : n);
}

int relpos_bias_grad(Args a) {    // G, rows, max_distance, bidirectional, offset, causal, q_len, k_len, accumulate, workspace, stream
  const at::Tensor &G = tensor(a[0], "G"), &rows = tensor(a[1], "rows");
  const int device = device_of(G, "G");
  if (G.dim() != 4 || rows.dim() != 3) throw Refused{"G [B, heads, Tq, Tk] and rows [B, num_buckets, heads] expected"};
  if (G.size(3) > 1 && G.stride(3) != 1) throw Refused{"G: unit stride along the keys expected"};
  const int64_t B = G.size(0), H = G.size(1), nb = rows.size(1);
  const int64_t rows_shape[3] = {B, nb, H}, len_shape[1] = {B};
  const dp_relpos p = {extent(nb), small_integer(a[2], "max_distance"), truth(a[3]), extent(H), extent(G.size(2)),
                       extent(G.size(3)), integer(a[4])};
  auto* out = static_cast<float*>(dense(a[1], device, at::kFloat, "rows", -1, rows_shape));
  auto* ql = static_cast<int32_t*>(dense(a[6], device, at::kInt, "q_len", -1, len_shape));
  auto* kl = static_cast<int32_t*>(dense(a[7], device, at::kInt, "k_len", -1, len_shape));
  const Workspace w = workspace_of(a[9], device);
  const On on(device, a[10]);
  return api.relpos_bias_grad(&p, extent(B), truth(a[5]), G.data_ptr(), dp_dtype_of(G, "G"), G.stride(0), G.stride(1),
                              G.stride(2), ql, kl, out, truth(a[8]), w.p, w.n, on.stream);
}

// Queries and keys [B, T, heads, dim] of one call, either None, and what belongs to them.
struct Heads {
  dp_qknorm p = {};
  int device = -1;
  const at::Tensor* x[2] = {nullptr, nullptr};
  Heads(PyObject* q, PyObject* k) {
    PyObject* o[2] = {q, k};
    const char* names[2] = {"q", "k"};
    for (int i = 0; i < 2; ++i) {
      if (o[i] == Py_None) continue;
      const at::Tensor& t = tensor(o[i], names[i]);
      if (t.dim() != 4) throw Refused{std::string(names[i]) + ": [B, T, heads, dim] expected"};
      if (device < 0) {
        device = device_of(t, names[i]);
        p.dtype = dp_dtype_of(t, names[i]);
        p.B = extent(t.size(0));
        p.T = extent(t.size(1));
        p.dim = extent(t.size(3));
      } else {
        on_device(t, device, names[i]);
        if (dp_dtype_of(t, names[i]) != p.dtype) throw Refused{"queries and keys share one dtype"};
        if (t.size(0) != p.B || t.size(1) != p.T || t.size(3) != p.dim)
          throw Refused{"queries and keys share examples, tokens and width"};
      }
      (i ? p.n_k : p.n_q) = extent(t.size(2));
      x[i] = &t;
    }
    if (device < 0) throw Refused{"queries or keys [B, T, heads, dim] expected"};
  }
  void more(PyObject* gain_q, PyObject* gain_k, PyObject* eps, PyObject* inv_freq, PyObject* positions, PyObject* lengths,
            PyObject* interleaved) {
    const int64_t dim[1] = {p.dim}, pos[2] = {p.B, p.T}, len[1] = {p.B};
    p.gain_q = static_cast<float*>(dense(gain_q, device, at::kFloat, "gain_q", -1, dim));
    p.gain_k = static_cast<float*>(dense(gain_k, device, at::kFloat, "gain_k", -1, dim));
    p.positions = static_cast<int32_t*>(dense(positions, device, at::kInt, "positions", -1, pos));
    p.lengths = static_cast<int32_t*>(dense(lengths, device, at::kInt, "lengths", -1, len));
    p.eps = number(eps);
    p.interleaved = truth(interleaved);
    if (inv_freq != Py_None) {
      const at::Tensor& f = tensor(inv_freq, "inv_freq");
      if (f.is_cuda() || f.scalar_type() != at::kDouble || !f.is_contiguous())
        throw Refused{"inv_freq: contiguous float64 tensor on the host expected"};
      p.rot = extent(2 * f.numel());
      p.inv_freq = p.rot ? static_cast<const double*>(f.data_ptr()) : nullptr;
    }
  }
  // dp_heads of a tensor shaped like the queries (i = 0) or keys (1); null where there are none.
  const dp_heads* view(PyObject* o, int i, const char* what, dp_heads& h) const {
    if (!x[i]) return nullptr;
    if (o == Py_None) throw Refused{std::string(what) + " expected"};
    const at::Tensor& t = tensor(o, what);
    on_device(t, device, what);
    if (t.scalar_type() != x[i]->scalar_type() || t.sizes() != x[i]->sizes())
      throw Refused{std::string(what) + ": " + shape_text(x[i]->sizes()) + " of the same dtype expected, got " + shape_text(t.sizes())};
    if (t.stride(3) != 1) throw Refused{std::string(what) + ": unit stride along the width expected"};
    h = {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
    return &h;
  }
};

int qknorm_rope(Args a) {         // q, k, out_q, out_k, gain_q, gain_k, eps, inv_freq, positions, lengths, interleaved, stream
  Heads H(a[0], a[1]);
  H.more(a[4], a[5], a[6], a[7], a[8], a[9], a[10]);
  dp_heads h[4];
  const dp_heads *q = H.view(a[0], 0, "q", h[0]), *k = H.view(a[1], 1, "k", h[1]);
  const dp_heads *oq = H.view(a[2], 0, "out_q", h[2]), *ok = H.view(a[3], 1, "out_k", h[3]);
  const On on(H.device, a[11]);
  return api.qknorm_rope(&H.p, q, k, oq, ok, on.stream);
}

PyObject* qknorm_workspace_bytes(Args a) {   // q, k
  const Heads H(a[0], a[1]);
  const size_t n = api.qknorm_workspace_bytes(&H.p);
  return PyLong_FromSize_t(n < 256 ? 256 : n);
}

int qknorm_rope_backward(Args a) {  // q, k, dout_q, dout_k, dq, dk, gain_q, gain_k, rows_q, rows_k, eps, inv_freq, positions, lengths, interleaved, accumulate, workspace, stream
  Heads H(a[0], a[1]);
  H.more(a[6], a[7], a[10], a[11], a[12], a[13], a[14]);
  if ((!H.x[0] && a[8] != Py_None) || (!H.x[1] && a[9] != Py_None))
    throw Refused{"gradients of a gain need the heads that it scales"};
  dp_heads h[6];
  const dp_heads *q = H.view(a[0], 0, "q", h[0]), *k = H.view(a[1], 1, "k", h[1]);
  const dp_heads *gq = H.view(a[2], 0, "dout_q", h[2]), *gk = H.view(a[3], 1, "dout_k", h[3]);
  const dp_heads *dq = H.view(a[4], 0, "dq", h[4]), *dk = H.view(a[5], 1, "dk", h[5]);
  const int64_t shape[2] = {H.p.B, H.p.dim};
  auto* rq = static_cast<float*>(dense(a[8], H.device, at::kFloat, "rows_q", -1, shape));
  auto* rk = static_cast<float*>(dense(a[9], H.device, at::kFloat, "rows_k", -1, shape));
  const Workspace w = workspace_of(a[16], H.device);
  const On on(H.device, a[17]);
  return api.qknorm_rope_backward(&H.p, q, k, gq, gk, dq, dk, rq, rk, truth(a[15]), w.p, w.n, on.stream);
}

// ---- module -------------------------------------------------------------------------------------------------------------
PyObject* as_object(int rc) { return PyLong_FromLong(rc); }
PyObject* as_object(PyObject* o) { return o; }

template <auto F, int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
    return nullptr;
  }
  if (!api.global_sqnorm) {
    PyErr_SetString(PyExc_RuntimeError, "bind() first");
    return nullptr;
  }
  try {
    return as_object(F(args));
  } catch (const Raised&) {
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what.c_str());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// bind(addresses): the entry points in the order of Api.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr Py_ssize_t count = sizeof(Api) / sizeof(void*);
  if (n != count) {
    PyErr_Format(PyExc_TypeError, "%zd addresses expected, got %zd", count, n);
    return nullptr;
  }
  void* p[count];
  for (Py_ssize_t k = 0; k < count; ++k) {
    p[k] = PyLong_AsVoidPtr(args[k]);
    if (PyErr_Occurred()) return nullptr;
  }
  memcpy(&api, p, sizeof(api));
  Py_RETURN_NONE;
}

#define ENTRY(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&bind)), METH_FASTCALL, nullptr},
    ENTRY(global_sqnorm, 5), ENTRY(clip_by_global_norm, 6), ENTRY(clip_adamw_step, 14),
    ENTRY(rows_list, 1), ENTRY(rows_sqnorms, 4), ENTRY(rows_clipped_accumulate, 3),
    ENTRY(relpos_bias, 6), ENTRY(relpos_workspace_bytes, 2), ENTRY(relpos_bias_grad, 11),
    ENTRY(qknorm_rope, 12), ENTRY(qknorm_workspace_bytes, 2), ENTRY(qknorm_rope_backward, 18),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dp_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// DP_MODULE_KEY names the torch and the Python that this file was compiled against; build.py looks for it in the built file.
PyMODINIT_FUNC PyInit__dp_tensors(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", DP_MODULE_KEY) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
