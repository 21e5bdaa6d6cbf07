// CPython module `_qwam_call`: the per-token calls of qwam.py (quantize_act,
// quantize_act_deflated, asp_linear, asp_layer, asp_matvec) and block.py
// (block_norm, block_norm_backward, kv_append, kv_read, paged_attention) and
// rotary.py (rope) without ctypes.
//
// A few-token call runs for 5-10 us on the GPU; marshalling one through ctypes
// took 14 us of Python (nine tensor checks of the layer, four or five of the
// arguments, the struct, the stream lookup), which was the whole time of such
// a call.  The same checks here take under 1 us.  Every check runs on every
// call, on the tensors that the layer holds at that time; nothing is kept
// between calls.
//
// Each function returns its outputs, the library's status as an int when the
// library refused the call, or None when an argument is not what the fast path
// takes (a wrong device, type, shape or stride): qwam.py then goes the long
// way, which names the argument that is wrong.  asp_linear, asp_layer and the
// calls of a token's step go there with an explicit stream too; an activation call does not, because the
// workspace of its stream made it dearer there than without one (26 us of host
// time against 16).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <memory>

#include "../../include/qwam.h"

namespace {

// entry points of the libqwam that qwam.py loaded
decltype(&qwam_quantize_act_ws) g_quantize;
decltype(&qwam_quantize_act_workspace) g_workspace;
decltype(&qwam_asp_linear) g_linear;
decltype(&qwam_asp_layer) g_layer;
decltype(&qwam_asp_matvec) g_matvec;
decltype(&qwam_asp_matvec_workspace) g_matvec_workspace;
decltype(&qwam_block_norm) g_norm;
decltype(&qwam_block_norm_backward) g_norm_bwd;
decltype(&qwam_block_norm_backward_workspace) g_norm_workspace;
decltype(&qwam_kv_append) g_append;
decltype(&qwam_paged_attention) g_attention;
decltype(&qwam_paged_attention_workspace) g_attention_workspace;
decltype(&qwam_kv_read) g_read;
decltype(&qwam_rope) g_rope;

enum Attr { kK, kN, kR, kGroup, kHadamard, kWq, kWs, kInv, kL1t, kL2t, kBias, kL1, kWsp, kL1f, kAttrs };
const char* const kAttrNames[kAttrs] = {"K",   "N",   "r",    "group", "hadamard", "wq",  "ws",
                                        "inv_smooth", "L1t", "L2t", "bias",  "L1",       "wsp", "L1f"};
PyObject* g_names[kAttrs];
PyObject *g_cuda_stream, *g_device_index;
enum CacheAttr { kCacheK, kCacheV, kCacheTable, kCacheKScale, kCacheVScale, kCacheAttrs };
const char* const kCacheAttrNames[kCacheAttrs] = {"k", "v", "table", "k_scale", "v_scale"};
PyObject* g_cache_names[kCacheAttrs];
PyObject *g_inv_freq, *g_axis, *g_interleaved;
enum Grad { kDx, kDbranch, kDgate, kDpostWeight, kDweight, kDscale, kDshift, kGrads };
const char* const kGradNames[kGrads] = {"dx", "dbranch", "dgate", "dpost_weight", "dweight", "dscale", "dshift"};
PyObject* g_grad_names[kGrads];

// the data pointer of a contiguous GPU tensor of this type and shape; false otherwise
bool data_of(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, void** out) {
  if (!THPVariable_Check(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != type || t.dim() != static_cast<int64_t>(shape.size())) return false;
  int64_t i = 0;
  for (const int64_t s : shape)
    if (t.size(i++) != s) return false;
  if (!t.is_contiguous()) return false;
  *out = t.data_ptr();
  return true;
}

// a GPU tensor; null for anything else
const at::Tensor* tensor_of(PyObject* o) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() ? &t : nullptr;
}

// whether the kernels, which run on the current device, may take these (GPU tensors)
bool on_current_device(std::initializer_list<const at::Tensor*> tensors) {
  const auto now = c10::hip::current_device();
  for (const at::Tensor* t : tensors)
    if (t->get_device() != now) return false;
  return true;
}

// the same of what may be None, or no tensor (which is refused elsewhere)
bool on_current_device(std::initializer_list<PyObject*> objects) {
  const auto now = c10::hip::current_device();
  for (PyObject* o : objects) {
    const at::Tensor* const t = o == nullptr ? nullptr : tensor_of(o);
    if (t != nullptr && t->get_device() != now) return false;
  }
  return true;
}

// A layer's struct, and references that keep its tensors alive during the call.
struct Layer {
  PyObject* held[kAttrs] = {};
  qwam_layer c = {};
  ~Layer() {
    for (PyObject* o : held) Py_XDECREF(o);
  }
  bool read_int(Attr a, int32_t& v) {
    if (!PyLong_Check(held[a])) return false;
    const long x = PyLong_AsLong(held[a]);
    if (x == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      return false;
    }
    v = static_cast<int32_t>(x);
    return v == x;
  }
  template <typename T>
  bool read(Attr a, at::ScalarType type, std::initializer_list<int64_t> shape, const T*& p, bool optional) {
    if (optional && held[a] == Py_None) return true;
    void* q = nullptr;
    if (!data_of(held[a], type, shape, &q)) return false;
    p = static_cast<const T*>(q);
    return true;
  }
  // matvec: a layer may do without smoothing, and with r = 0 without a branch
  bool load(PyObject* o, bool matvec = false) {
    for (int a = 0; a < kAttrs; ++a) {
      held[a] = PyObject_GetAttr(o, g_names[a]);
      if (held[a] == nullptr) {
        PyErr_Clear();
        return false;
      }
    }
    if (!read_int(kK, c.K) || !read_int(kN, c.N) || !read_int(kR, c.r) || !read_int(kGroup, c.group) ||
        !read_int(kHadamard, c.hadamard) || c.K <= 0 || c.group <= 0)
      return false;
    const int64_t G = c.K / c.group;
    if (!on_current_device({held[kWq], held[kWs], held[kInv], held[kL1t], held[kL2t], held[kBias], held[kL1], held[kWsp], held[kL1f]}))
      return false;
    return read(kWq, at::kByte, {c.N, c.K / 2}, c.wq, false) && read(kWs, at::kFloat, {G, c.N}, c.ws, false) &&
           read(kInv, at::kFloat, {c.K}, c.inv_smooth, matvec) &&
           ((matvec && c.r == 0) || (read(kL1t, at::kBFloat16, {c.r, c.K}, c.L1t, false) &&
                                     read(kL2t, at::kBFloat16, {c.N, c.r}, c.L2t, false))) && read(kBias, at::kBFloat16, {c.N}, c.bias, true) &&
           read(kL1, at::kBFloat16, {c.K, c.r}, c.L1, true) && read(kWsp, at::kInt, {G, c.N}, c.wsp, true) &&
           read(kL1f, at::kBFloat16, {c.K / 64, c.r / 16, 2, 64, 8}, c.L1f, true);
  }
};

// the number of rows of a 2-d GPU tensor; -1 for anything else
int64_t rows_of(PyObject* o) {
  if (!THPVariable_Check(o)) return -1;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.dim() == 2 && t.size(0) <= INT32_MAX ? t.size(0) : -1;
}

// the rows of `like` and an output of `cols` columns on its device, or `given`
bool output(PyObject* given, const at::Tensor& like, at::ScalarType type, int64_t rows, int64_t cols, PyObject** obj,
            void** data) {
  if (given == nullptr || given == Py_None) {
    const at::Tensor t = at::empty({rows, cols}, like.options().dtype(type));
    *data = t.data_ptr();
    *obj = THPVariable_Wrap(t);
    return *obj != nullptr;
  }
  if (!data_of(given, type, {rows, cols}, data)) return false;
  Py_INCREF(given);
  *obj = given;
  return true;
}

struct Held {
  PyObject* o = nullptr;
  ~Held() { Py_XDECREF(o); }
  PyObject* release() {
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};

// What the call wrote into tensors that the caller gave, told to autograd, which may have saved them: as after torch's own
// operations in place (a tensor of inference mode has no version).  None, and what is null, is no tensor.
void written(std::initializer_list<PyObject*> objects) {
  for (PyObject* o : objects)
    if (o != nullptr && THPVariable_Check(o) && !THPVariable_Unpack(o).is_inference())
      THPVariable_Unpack(o).unsafeGetTensorImpl()->bump_version();
}

PyObject* none_or_error() {
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// the handle of a torch.cuda.Stream of the current device; false for another device's
bool stream_of(PyObject* o, hipStream_t* out) {
  Held handle, device;
  handle.o = PyObject_GetAttr(o, g_cuda_stream);
  device.o = handle.o == nullptr ? nullptr : PyObject_GetAttr(o, g_device_index);
  if (device.o == nullptr) return false;
  *out = static_cast<hipStream_t>(PyLong_AsVoidPtr(handle.o));
  const long index = PyLong_AsLong(device.o);
  return !PyErr_Occurred() && index == c10::hip::current_device();
}

// quantize(layer, x, out, deflated, stream) -> (xq, xs, t); stream a torch.cuda.Stream or None
PyObject* py_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5) Py_RETURN_NONE;
  Layer L;
  const int64_t M = rows_of(args[1]);
  void* x;
  if (M < 0 || !L.load(args[0]) || !data_of(args[1], at::kBFloat16, {M, L.c.K}, &x)) return none_or_error();
  PyObject* given[3] = {nullptr, nullptr, nullptr};
  if (args[2] != Py_None) {
    if (!PyTuple_Check(args[2]) || PyTuple_GET_SIZE(args[2]) != 3) return none_or_error();
    for (int i = 0; i < 3; ++i) given[i] = PyTuple_GET_ITEM(args[2], i);
  }
  const at::Tensor& xt = THPVariable_Unpack(args[1]);
  hipStream_t given_stream = nullptr;
  const bool explicit_stream = args[4] != Py_None;
  if (!on_current_device({args[1], given[0], given[1], given[2]}) || (explicit_stream && !stream_of(args[4], &given_stream)))
    return none_or_error();
  Held xq, xs, t;
  void *pq, *ps, *pt;
  if (!output(given[0], xt, at::kByte, M, L.c.K / 2, &xq.o, &pq) ||
      !output(given[1], xt, at::kFloat, L.c.K / L.c.group, M, &xs.o, &ps) ||
      !output(given[2], xt, at::kBFloat16, M, L.c.r, &t.o, &pt))
    return none_or_error();
  const int32_t deflated = PyObject_IsTrue(args[3]) == 1;
  // few tokens and a large K: the call splits K over workgroups through a
  // workspace, from the pool of the stream the call runs on (dropped below: the
  // next user of that memory runs behind the call's kernels)
  const int64_t need = g_workspace(&L.c, static_cast<int32_t>(M), deflated);
  at::Tensor ws;
  std::unique_ptr<void, void (*)(void*)> ws_stream(nullptr, c10::hip::HIPCachingAllocator::raw_delete);
  if (need > 0) {
    if (explicit_stream)
      ws_stream.reset(c10::hip::HIPCachingAllocator::raw_alloc_with_stream(static_cast<size_t>(need), given_stream));
    else
      ws = at::empty({need}, xt.options().dtype(at::kByte));
  }
  void* const pw = need <= 0 ? nullptr : explicit_stream ? ws_stream.get() : ws.data_ptr();
  void* stream = explicit_stream ? given_stream : current_stream();
  qwam_status st;
  Py_BEGIN_ALLOW_THREADS
  st = g_quantize(&L.c, static_cast<int32_t>(M), deflated, static_cast<const uint16_t*>(x), static_cast<uint8_t*>(pq),
                  static_cast<float*>(ps), static_cast<uint16_t*>(pt), pw, need > 0 ? need : 0, stream);
  Py_END_ALLOW_THREADS
  if (st != QWAM_OK) return PyLong_FromLong(st);
  written({given[0], given[1], given[2]});
  return PyTuple_Pack(3, xq.o, xs.o, t.o);
  END_HANDLE_TH_ERRORS
}

// linear(layer, xq, xs, t, out) -> y
PyObject* py_linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5) Py_RETURN_NONE;
  Layer L;
  const int64_t M = rows_of(args[1]);
  void *xq, *xs, *t, *py;
  if (M < 0 || !L.load(args[0]) || !data_of(args[1], at::kByte, {M, L.c.K / 2}, &xq) ||
      !data_of(args[2], at::kFloat, {L.c.K / L.c.group, M}, &xs) || !data_of(args[3], at::kBFloat16, {M, L.c.r}, &t))
    return none_or_error();
  if (!on_current_device({args[1], args[2], args[3], args[4]})) Py_RETURN_NONE;
  Held y;
  if (!output(args[4], THPVariable_Unpack(args[1]), at::kBFloat16, M, L.c.N, &y.o, &py)) return none_or_error();
  void* stream = current_stream();
  qwam_status st;
  Py_BEGIN_ALLOW_THREADS
  st = g_linear(&L.c, static_cast<int32_t>(M), static_cast<const uint8_t*>(xq), static_cast<const float*>(xs),
                static_cast<const uint16_t*>(t), static_cast<uint16_t*>(py), stream);
  Py_END_ALLOW_THREADS
  if (st != QWAM_OK) return PyLong_FromLong(st);
  written({args[4]});
  return y.release();
  END_HANDLE_TH_ERRORS
}

// layer(layer, x, out) -> y (without the optional activation outputs)
PyObject* py_layer(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 3) Py_RETURN_NONE;
  Layer L;
  const int64_t M = rows_of(args[1]);
  void *x, *py;
  if (M < 0 || !L.load(args[0]) || !data_of(args[1], at::kBFloat16, {M, L.c.K}, &x)) return none_or_error();
  if (!on_current_device({args[1], args[2]})) Py_RETURN_NONE;
  Held y;
  if (!output(args[2], THPVariable_Unpack(args[1]), at::kBFloat16, M, L.c.N, &y.o, &py)) return none_or_error();
  void* stream = current_stream();
  qwam_status st;
  Py_BEGIN_ALLOW_THREADS
  st = g_layer(&L.c, static_cast<int32_t>(M), static_cast<const uint16_t*>(x), static_cast<uint16_t*>(py), nullptr,
               nullptr, nullptr, stream);
  Py_END_ALLOW_THREADS
  if (st != QWAM_OK) return PyLong_FromLong(st);
  written({args[2]});
  return y.release();
  END_HANDLE_TH_ERRORS
}

// device memory for the call about to be made on the current stream
at::Tensor workspace_of(int64_t need, const at::Tensor& like) {
  return need > 0 ? at::empty({need}, like.options().dtype(at::kByte)) : at::Tensor();
}

bool tangent(PyObject* o) { return THPVariable_Check(o) && THPVariable_Unpack(o)._fw_grad(0).defined(); }

// whether autograd follows this argument (a tensor, or None): backwards, or forwards through a tangent
bool tracked(PyObject* o) {
  return tangent(o) || (THPVariable_Check(o) && c10::GradMode::is_enabled() && THPVariable_Unpack(o).requires_grad());
}
bool tracked(std::initializer_list<PyObject*> objects) {
  for (PyObject* o : objects)
    if (tracked(o)) return true;
  return false;
}

// matvec(layer, x, out) -> y
PyObject* py_matvec(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 3) Py_RETURN_NONE;
  Layer L;
  const int64_t M = rows_of(args[1]);
  void *x, *py;
  if (M < 0 || !L.load(args[0], true) || !data_of(args[1], at::kBFloat16, {M, L.c.K}, &x)) return none_or_error();
  if (tracked({args[1], args[2], L.held[kWs], L.held[kInv], L.held[kL1t], L.held[kL2t], L.held[kBias], L.held[kL1f]}) ||
      !on_current_device({args[1], args[2]}))
    Py_RETURN_NONE;
  const at::Tensor& xt = THPVariable_Unpack(args[1]);
  Held y;
  if (!output(args[2], xt, at::kBFloat16, M, L.c.N, &y.o, &py)) return none_or_error();
  const int64_t need = g_matvec_workspace(&L.c, static_cast<int32_t>(M));
  if (need < 0) Py_RETURN_NONE;
  const at::Tensor ws = workspace_of(need, xt);
  void* stream = current_stream();
  qwam_status st;
  Py_BEGIN_ALLOW_THREADS
  st = g_matvec(&L.c, static_cast<int32_t>(M), static_cast<const uint16_t*>(x), static_cast<uint16_t*>(py),
                need > 0 ? ws.data_ptr() : nullptr, need, stream);
  Py_END_ALLOW_THREADS
  if (st != QWAM_OK) return PyLong_FromLong(st);
  written({args[2]});
  return y.release();
  END_HANDLE_TH_ERRORS
}

// the arguments that the norm's calls share, from `a`: norm ("rms" or "layer"), eps, residual_scale, gate, post_norm, post_weight,
// weight, scale, shift
constexpr int kNormArgs = 9;
bool norm_of(PyObject* const* a, int64_t T, int64_t D, bool f32, qwam_norm& p) {
  if (!PyUnicode_Check(a[0]) || !PyFloat_Check(a[1]) || !PyFloat_Check(a[2]) || !PyBool_Check(a[4]) || T > INT32_MAX || D > INT32_MAX)
    return false;
  p = {};
  p.T = static_cast<int32_t>(T);
  p.D = static_cast<int32_t>(D);
  p.S = 1;
  if (PyUnicode_CompareWithASCIIString(a[0], "rms") == 0) p.kind = QWAM_NORM_RMS;
  else if (PyUnicode_CompareWithASCIIString(a[0], "layer") == 0) p.kind = QWAM_NORM_LAYER;
  else return false;
  p.post = a[4] == Py_True;
  p.x_f32 = f32;
  p.eps = static_cast<float>(PyFloat_AS_DOUBLE(a[1]));
  p.residual_scale = static_cast<float>(PyFloat_AS_DOUBLE(a[2]));
  bool first = true;
  auto per_sample = [&](PyObject* o, const uint16_t*& q, int64_t& stride) {
    if (o == Py_None) return true;
    const at::Tensor* t = tensor_of(o);
    if (t == nullptr || t->scalar_type() != at::kBFloat16 || t->dim() != 2 || t->size(1) != D || (D > 1 && t->stride(1) != 1) ||
        t->size(0) > INT32_MAX || (!first && t->size(0) != p.S))
      return false;
    first = false;
    p.S = static_cast<int32_t>(t->size(0));
    q = static_cast<const uint16_t*>(t->data_ptr());
    stride = t->stride(0);
    return true;
  };
  auto per_channel = [&](PyObject* o, const uint16_t*& q) {
    void* d = nullptr;
    if (o == Py_None) return true;
    if (!data_of(o, at::kBFloat16, {D}, &d)) return false;
    q = static_cast<const uint16_t*>(d);
    return true;
  };
  return per_sample(a[3], p.gate, p.gate_stride) && per_sample(a[7], p.scale, p.scale_stride) &&
         per_sample(a[8], p.shift, p.shift_stride) && per_channel(a[5], p.post_weight) && per_channel(a[6], p.weight) &&
         (p.post_weight == nullptr || p.post != 0);
}

// norm(x, branch, <norm_of's>) -> (x', h); None under autograd too
PyObject* py_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 2 + kNormArgs) Py_RETURN_NONE;
  const at::Tensor* x = tensor_of(args[0]);
  if (x == nullptr || x->dim() != 2 || !x->is_contiguous()) Py_RETURN_NONE;
  const bool f32 = x->scalar_type() == at::kFloat;
  if (!f32 && x->scalar_type() != at::kBFloat16) Py_RETURN_NONE;
  const int64_t T = x->size(0), D = x->size(1);
  qwam_norm p;
  void* branch = nullptr;
  if (!norm_of(args + 2, T, D, f32, p) || (args[1] != Py_None && !data_of(args[1], at::kBFloat16, {T, D}, &branch)))
    return none_or_error();
  if (tracked({args[0], args[1], args[5], args[7], args[8], args[9], args[10]}) ||
      !on_current_device({args[0], args[1], args[5], args[7], args[8], args[9], args[10]}))
    Py_RETURN_NONE;
  const at::Tensor h = at::empty({T, D}, x->options().dtype(at::kBFloat16));
  const at::Tensor xo = branch != nullptr ? at::empty({T, D}, x->options()) : at::Tensor();
  const qwam_status st = g_norm(&p, x->data_ptr(), static_cast<const uint16_t*>(branch), branch != nullptr ? xo.data_ptr() : nullptr,
                                static_cast<uint16_t*>(h.data_ptr()), current_stream());
  if (st != QWAM_OK) return PyLong_FromLong(st);
  Held ho, xoo;
  ho.o = THPVariable_Wrap(h);
  xoo.o = branch != nullptr ? THPVariable_Wrap(xo) : Py_NewRef(Py_None);
  return PyTuple_Pack(2, xoo.o, ho.o);
  END_HANDLE_TH_ERRORS
}

// norm_backward(dx_out, dh, x_out, branch, <norm_of's>) -> the dict of all gradients
PyObject* py_norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 4 + kNormArgs) Py_RETURN_NONE;
  const at::Tensor* x = tensor_of(args[2]);
  if (x == nullptr || x->dim() != 2 || !x->is_contiguous()) Py_RETURN_NONE;
  const bool f32 = x->scalar_type() == at::kFloat;
  if (!f32 && x->scalar_type() != at::kBFloat16) Py_RETURN_NONE;
  const int64_t T = x->size(0), D = x->size(1);
  qwam_norm p;
  void *dxo = nullptr, *dh = nullptr, *branch = nullptr;
  if (!norm_of(args + 4, T, D, f32, p) || (args[0] != Py_None && !data_of(args[0], x->scalar_type(), {T, D}, &dxo)) ||
      !data_of(args[1], at::kBFloat16, {T, D}, &dh) || (args[3] != Py_None && !data_of(args[3], at::kBFloat16, {T, D}, &branch)))
    return none_or_error();
  for (Py_ssize_t i = 0; i < nargs; ++i)
    if (tangent(args[i])) Py_RETURN_NONE;      // (false of what is no tensor)
  if (!on_current_device({args[0], args[1], args[2], args[3], args[7], args[9], args[10], args[11], args[12]})) Py_RETURN_NONE;
  const int64_t need = g_norm_workspace(&p);
  if (need < 0) Py_RETURN_NONE;
  at::Tensor g[kGrads];
  const auto f = x->options().dtype(at::kFloat);
  g[kDx] = at::empty({T, D}, x->options());
  if (branch != nullptr) {
    g[kDbranch] = at::empty({T, D}, x->options().dtype(at::kBFloat16));
    if (p.gate != nullptr) g[kDgate] = at::empty({p.S, D}, f);
    if (p.post_weight != nullptr) g[kDpostWeight] = at::empty({D}, f);
  }
  if (p.weight != nullptr) g[kDweight] = at::empty({D}, f);
  if (p.scale != nullptr) g[kDscale] = at::empty({p.S, D}, f);
  if (p.shift != nullptr) g[kDshift] = at::empty({p.S, D}, f);
  const at::Tensor ws = workspace_of(need, *x);
  auto ptr = [&](Grad i) -> void* { return g[i].defined() ? g[i].data_ptr() : nullptr; };
  auto fptr = [&](Grad i) { return static_cast<float*>(ptr(i)); };
  const qwam_status st = g_norm_bwd(&p, dxo, static_cast<const uint16_t*>(dh), x->data_ptr(), static_cast<const uint16_t*>(branch),
                                    ptr(kDx), static_cast<uint16_t*>(ptr(kDbranch)), fptr(kDgate), fptr(kDscale), fptr(kDshift),
                                    fptr(kDpostWeight), fptr(kDweight), need > 0 ? ws.data_ptr() : nullptr, need, current_stream());
  if (st != QWAM_OK) return PyLong_FromLong(st);
  Held d;
  d.o = PyDict_New();
  if (d.o == nullptr) return nullptr;
  for (int i = 0; i < kGrads; ++i) {
    Held v;
    v.o = g[i].defined() ? THPVariable_Wrap(g[i]) : Py_NewRef(Py_None);
    if (v.o == nullptr || PyDict_SetItem(d.o, g_grad_names[i], v.o) != 0) return nullptr;
  }
  return d.release();
  END_HANDLE_TH_ERRORS
}

// A cache's struct, and references that keep its tensors alive during the call.
struct Cache {
  PyObject* held[kCacheAttrs] = {};
  qwam_cache c = {};
  const at::Tensor* k = nullptr;
  ~Cache() {
    for (PyObject* o : held) Py_XDECREF(o);
  }
  bool load(PyObject* o) {
    for (int a = 0; a < kCacheAttrs; ++a) {
      held[a] = PyObject_GetAttr(o, g_cache_names[a]);
      if (held[a] == nullptr) {
        PyErr_Clear();
        return false;
      }
    }
    k = tensor_of(held[kCacheK]);
    const at::Tensor *v = tensor_of(held[kCacheV]), *t = tensor_of(held[kCacheTable]);
    if (k == nullptr || v == nullptr || t == nullptr || k->dim() != 4 || k->sizes() != v->sizes() || k->strides() != v->strides() ||
        k->scalar_type() != v->scalar_type() || k->stride(3) != 1 || t->dim() != 2)
      return false;
    const bool fp8 = k->scalar_type() == at::kFloat8_e4m3fn, fp4 = k->scalar_type() == at::ScalarType::Float4_e2m1fn_x2;
    if ((!fp8 && !fp4 && k->scalar_type() != at::kBFloat16) || !on_current_device({k, v, t})) return false;
    for (int i = 0; i < 4; ++i)
      if (k->size(i) > INT32_MAX) return false;
    if (t->size(0) > INT32_MAX || t->size(1) > INT32_MAX) return false;
    c.pages = static_cast<int32_t>(k->size(0));
    c.heads = static_cast<int32_t>(k->size(1));
    c.page_size = static_cast<int32_t>(k->size(2));
    if (fp4 && k->size(3) > INT32_MAX / 2) return false;
    c.dim = static_cast<int32_t>(fp4 ? 2 * k->size(3) : k->size(3));
    c.type = fp4 ? QWAM_CACHE_FP4 : fp8 ? QWAM_CACHE_FP8 : QWAM_CACHE_BF16;
    c.seqs = static_cast<int32_t>(t->size(0));
    c.table_width = static_cast<int32_t>(t->size(1));
    c.page_stride = k->stride(0);
    c.head_stride = k->stride(1);
    c.row_stride = k->stride(2);
    c.k = k->data_ptr();
    c.v = v->data_ptr();
    void *table, *ks, *vs;
    if (!data_of(held[kCacheTable], at::kInt, {c.seqs, c.table_width}, &table)) return false;
    c.table = static_cast<const int32_t*>(table);
    if (!fp8 && !fp4) return true;
    if (fp4) {
      const std::initializer_list<int64_t> shape = {c.pages, c.heads, c.dim / 32, c.page_size};
      constexpr auto type = at::ScalarType::Float8_e8m0fnu;
      if (!data_of(held[kCacheKScale], type, shape, &ks) || !data_of(held[kCacheVScale], type, shape, &vs)) return false;
    } else if (!data_of(held[kCacheKScale], at::kFloat, {c.heads}, &ks) || !data_of(held[kCacheVScale], at::kFloat, {c.heads}, &vs)) {
      return false;
    }
    if (!on_current_device({&THPVariable_Unpack(held[kCacheKScale]), &THPVariable_Unpack(held[kCacheVScale])})) return false;
    c.k_scale = ks;
    c.v_scale = vs;
    return true;
  }
  bool followed() const { return tracked({held[kCacheK], held[kCacheV], held[kCacheKScale], held[kCacheVScale]}); }
};

// a bf16 [rows][heads][dim] whose rows may be apart
const at::Tensor* rows3_of(PyObject* o, int64_t rows, int64_t heads, int64_t dim) {
  const at::Tensor* t = tensor_of(o);
  if (t == nullptr || t->scalar_type() != at::kBFloat16 || t->dim() != 3 || t->size(0) != rows || t->size(1) != heads ||
      t->size(2) != dim || (dim > 1 && t->stride(2) != 1) || (heads > 1 && t->stride(1) != dim))
    return nullptr;
  return t;
}

// append(cache, k, v, seq, pos) -> 0
PyObject* py_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5) Py_RETURN_NONE;
  Cache C;
  const at::Tensor* k = tensor_of(args[1]);
  if (k == nullptr || k->dim() != 3 || k->size(0) > INT32_MAX || !C.load(args[0])) return none_or_error();
  const int64_t n = k->size(0);
  void *seq, *pos;
  const at::Tensor* v = rows3_of(args[2], n, C.c.heads, C.c.dim);
  if (v == nullptr || rows3_of(args[1], n, C.c.heads, C.c.dim) == nullptr || !data_of(args[3], at::kInt, {n}, &seq) ||
      !data_of(args[4], at::kInt, {n}, &pos))
    return none_or_error();
  if (C.followed() || tracked({args[1], args[2]})) Py_RETURN_NONE;
  if (!on_current_device({k, v, &THPVariable_Unpack(args[3]), &THPVariable_Unpack(args[4])})) Py_RETURN_NONE;
  const qwam_status st = g_append(&C.c, static_cast<int32_t>(n), static_cast<const uint16_t*>(k->data_ptr()), n > 1 ? k->stride(0) : 0,
                                  static_cast<const uint16_t*>(v->data_ptr()), n > 1 ? v->stride(0) : 0,
                                  static_cast<const int32_t*>(seq), static_cast<const int32_t*>(pos), current_stream());
  if (st == QWAM_OK) {
    written({C.held[kCacheK], C.held[kCacheV]});
    if (C.c.type == QWAM_CACHE_FP4) written({C.held[kCacheKScale], C.held[kCacheVScale]});
  }
  return PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// attention(cache, q, lengths, starts, scale, max_len, out) -> out; scale, max_len and out may be None
PyObject* py_attention(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 7) Py_RETURN_NONE;
  Cache C;
  const at::Tensor* q = tensor_of(args[1]);
  if (q == nullptr || q->dim() != 3 || q->size(1) > INT32_MAX || !C.load(args[0]) ||
      rows3_of(args[1], C.c.seqs, q->size(1), C.c.dim) == nullptr)
    return none_or_error();
  if (C.followed() || tracked({args[1], args[6]})) Py_RETURN_NONE;
  const int32_t heads = static_cast<int32_t>(q->size(1));
  void *lengths, *starts = nullptr, *po;
  if (!data_of(args[2], at::kInt, {C.c.seqs}, &lengths) || (args[3] != Py_None && !data_of(args[3], at::kInt, {C.c.seqs}, &starts)))
    return none_or_error();
  double scale;
  if (args[4] == Py_None) scale = 1.0 / std::sqrt(static_cast<double>(C.c.dim));
  else if (PyFloat_Check(args[4])) scale = PyFloat_AS_DOUBLE(args[4]);
  else Py_RETURN_NONE;
  int64_t max_len = static_cast<int64_t>(C.c.table_width) * C.c.page_size;
  if (args[5] != Py_None) {
    if (!PyLong_Check(args[5])) Py_RETURN_NONE;
    max_len = PyLong_AsLongLong(args[5]);
  }
  if (PyErr_Occurred() || max_len < 1 || max_len > INT32_MAX) return none_or_error();
  if (!on_current_device({q, &THPVariable_Unpack(args[2])}) || (starts != nullptr && !on_current_device({&THPVariable_Unpack(args[3])})))
    Py_RETURN_NONE;
  Held o;
  if (args[6] == Py_None) {
    const at::Tensor t = at::empty({C.c.seqs, heads, C.c.dim}, q->options());
    po = t.data_ptr();
    o.o = THPVariable_Wrap(t);
  } else {
    if (!data_of(args[6], at::kBFloat16, {C.c.seqs, heads, C.c.dim}, &po) || !on_current_device({&THPVariable_Unpack(args[6])}))
      return none_or_error();
    o.o = Py_NewRef(args[6]);
  }
  const int64_t need = g_attention_workspace(&C.c, heads, static_cast<int32_t>(max_len));
  if (need < 0) Py_RETURN_NONE;
  const at::Tensor ws = workspace_of(need, *q);
  const qwam_status st = g_attention(&C.c, heads, static_cast<const uint16_t*>(q->data_ptr()), C.c.seqs > 1 ? q->stride(0) : 0,
                                     static_cast<const int32_t*>(lengths), static_cast<const int32_t*>(starts),
                                     static_cast<int32_t>(max_len), static_cast<float>(scale), static_cast<uint16_t*>(po),
                                     need > 0 ? ws.data_ptr() : nullptr, need, current_stream());
  if (st != QWAM_OK) return PyLong_FromLong(st);
  written({args[6]});
  return o.release();
  END_HANDLE_TH_ERRORS
}

// read(cache, seq, pos, out) -> (k, v); out may be None
PyObject* py_read(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 4) Py_RETURN_NONE;
  Cache C;
  const at::Tensor* at_pos = tensor_of(args[2]);
  if (at_pos == nullptr || at_pos->dim() != 1 || at_pos->size(0) > INT32_MAX || !C.load(args[0])) return none_or_error();
  const int64_t n = at_pos->size(0);
  void *seq, *pos;
  if (!data_of(args[1], at::kInt, {n}, &seq) || !data_of(args[2], at::kInt, {n}, &pos) || C.followed() ||
      !on_current_device({&THPVariable_Unpack(args[1]), at_pos}))
    return none_or_error();
  Held o[2];
  const at::Tensor* t[2];
  for (int i = 0; i < 2; ++i) {
    if (args[3] == Py_None) {
      o[i].o = THPVariable_Wrap(at::empty({n, C.c.heads, C.c.dim}, C.k->options().dtype(at::kBFloat16)));
      if (o[i].o == nullptr) return nullptr;
    } else {
      if (!PyTuple_Check(args[3]) || PyTuple_GET_SIZE(args[3]) != 2) Py_RETURN_NONE;
      o[i].o = Py_NewRef(PyTuple_GET_ITEM(args[3], i));
    }
    t[i] = rows3_of(o[i].o, n, C.c.heads, C.c.dim);
    if (t[i] == nullptr || tracked(o[i].o) || !on_current_device({t[i]})) return none_or_error();
  }
  const qwam_status st = g_read(&C.c, static_cast<int32_t>(n), static_cast<const int32_t*>(seq), static_cast<const int32_t*>(pos),
                                static_cast<uint16_t*>(t[0]->data_ptr()), n > 1 ? t[0]->stride(0) : 0,
                                static_cast<uint16_t*>(t[1]->data_ptr()), n > 1 ? t[1]->stride(0) : 0, current_stream());
  if (st != QWAM_OK) return PyLong_FromLong(st);
  if (args[3] != Py_None) written({o[0].o, o[1].o});
  return PyTuple_Pack(2, o[0].o, o[1].o);
  END_HANDLE_TH_ERRORS
}

// rope(x, positions, plan, inverse, out) -> y; None with an out that is not x (its overlap is looked at there) and where
// autograd follows x
PyObject* py_rope(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5 || !PyBool_Check(args[3]) || (args[4] != Py_None && args[4] != args[0])) Py_RETURN_NONE;
  Held freq, axis, interleaved;
  freq.o = PyObject_GetAttr(args[2], g_inv_freq);
  axis.o = freq.o == nullptr ? nullptr : PyObject_GetAttr(args[2], g_axis);
  interleaved.o = axis.o == nullptr ? nullptr : PyObject_GetAttr(args[2], g_interleaved);
  if (interleaved.o == nullptr) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  const at::Tensor *x = tensor_of(args[0]), *pos = tensor_of(args[1]), *f = tensor_of(freq.o);
  if (!PyBool_Check(interleaved.o) || x == nullptr || pos == nullptr || f == nullptr || x->dim() != 3 || pos->dim() != 2 || f->dim() != 1)
    Py_RETURN_NONE;
  for (int i = 0; i < 3; ++i)
    if (x->size(i) > INT32_MAX) Py_RETURN_NONE;
  if (pos->size(0) > INT32_MAX || pos->size(1) > INT32_MAX || f->size(0) > INT32_MAX) Py_RETURN_NONE;
  qwam_rope_plan p = {};
  p.heads = static_cast<int32_t>(x->size(1));
  p.dim = static_cast<int32_t>(x->size(2));
  p.pairs = static_cast<int32_t>(f->size(0));
  p.interleaved = interleaved.o == Py_True;
  p.positions = static_cast<int32_t>(pos->size(0));
  p.axes = static_cast<int32_t>(pos->size(1));
  p.pos_f32 = pos->scalar_type() == at::kFloat;
  p.x_f32 = x->scalar_type() == at::kFloat;
  if ((!p.x_f32 && x->scalar_type() != at::kBFloat16) || (!p.pos_f32 && pos->scalar_type() != at::kInt) || !pos->is_contiguous() ||
      (x->size(2) > 1 && x->stride(2) != 1) || (x->size(1) > 1 && x->stride(1) != x->size(2)))
    Py_RETURN_NONE;
  void *fp, *ap;
  if (!data_of(freq.o, at::kFloat, {p.pairs}, &fp) || !data_of(axis.o, at::kInt, {p.pairs}, &ap)) return none_or_error();
  if (!on_current_device({x, pos, f, &THPVariable_Unpack(axis.o)}) || tracked({args[0], args[1], freq.o})) Py_RETURN_NONE;
  p.pos = pos->data_ptr();
  p.inv_freq = static_cast<const float*>(fp);
  p.axis = static_cast<const int32_t*>(ap);
  const int64_t T = x->size(0), stride = T > 1 ? x->stride(0) : 0;
  Held y;
  void* py = x->data_ptr();
  int64_t y_stride = stride;
  if (args[4] == Py_None) {
    const at::Tensor t = at::empty(x->sizes(), x->options());
    py = t.data_ptr();
    y_stride = T > 1 ? t.stride(0) : 0;
    y.o = THPVariable_Wrap(t);
    if (y.o == nullptr) return nullptr;
  } else {
    y.o = Py_NewRef(args[4]);
  }
  const qwam_status st = g_rope(&p, static_cast<int32_t>(T), args[3] == Py_True, x->data_ptr(), stride, py, y_stride, current_stream());
  if (st != QWAM_OK) return PyLong_FromLong(st);
  written({args[4]});
  return y.release();
  END_HANDLE_TH_ERRORS
}

// bind(the addresses of the library's entry points, in the order below)
PyObject* py_bind(PyObject*, PyObject* args) {
  void** const to[] = {reinterpret_cast<void**>(&g_quantize), reinterpret_cast<void**>(&g_workspace),
                       reinterpret_cast<void**>(&g_linear),   reinterpret_cast<void**>(&g_layer),
                       reinterpret_cast<void**>(&g_matvec),   reinterpret_cast<void**>(&g_matvec_workspace),
                       reinterpret_cast<void**>(&g_norm),     reinterpret_cast<void**>(&g_norm_bwd),
                       reinterpret_cast<void**>(&g_norm_workspace), reinterpret_cast<void**>(&g_append),
                       reinterpret_cast<void**>(&g_attention), reinterpret_cast<void**>(&g_attention_workspace),
                       reinterpret_cast<void**>(&g_read), reinterpret_cast<void**>(&g_rope)};
  constexpr Py_ssize_t n = sizeof(to) / sizeof(to[0]);
  if (PyTuple_GET_SIZE(args) != n) {
    PyErr_Format(PyExc_TypeError, "bind takes %zd addresses", n);
    return nullptr;
  }
  void* p[n];
  for (Py_ssize_t i = 0; i < n; ++i) {
    p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
    if (PyErr_Occurred()) return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) *to[i] = p[i];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(py_quantize), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(py_linear), METH_FASTCALL, nullptr},
    {"layer", reinterpret_cast<PyCFunction>(py_layer), METH_FASTCALL, nullptr},
    {"matvec", reinterpret_cast<PyCFunction>(py_matvec), METH_FASTCALL, nullptr},
    {"norm", reinterpret_cast<PyCFunction>(py_norm), METH_FASTCALL, nullptr},
    {"norm_backward", reinterpret_cast<PyCFunction>(py_norm_bwd), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(py_append), METH_FASTCALL, nullptr},
    {"attention", reinterpret_cast<PyCFunction>(py_attention), METH_FASTCALL, nullptr},
    {"read", reinterpret_cast<PyCFunction>(py_read), METH_FASTCALL, nullptr},
    {"rope", reinterpret_cast<PyCFunction>(py_rope), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qwam_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qwam_call() {
  for (int a = 0; a < kAttrs; ++a)
    if ((g_names[a] = PyUnicode_InternFromString(kAttrNames[a])) == nullptr) return nullptr;
  for (int a = 0; a < kCacheAttrs; ++a)
    if ((g_cache_names[a] = PyUnicode_InternFromString(kCacheAttrNames[a])) == nullptr) return nullptr;
  for (int a = 0; a < kGrads; ++a)
    if ((g_grad_names[a] = PyUnicode_InternFromString(kGradNames[a])) == nullptr) return nullptr;
  if ((g_inv_freq = PyUnicode_InternFromString("inv_freq")) == nullptr || (g_axis = PyUnicode_InternFromString("axis")) == nullptr ||
      (g_interleaved = PyUnicode_InternFromString("interleaved")) == nullptr)
    return nullptr;
  if ((g_cuda_stream = PyUnicode_InternFromString("cuda_stream")) == nullptr ||
      (g_device_index = PyUnicode_InternFromString("device_index")) == nullptr)
    return nullptr;
  return PyModule_Create(&module);
}
