// The calls of a training step's inner loop from Python, in one native step each: argument checks, pointers, the current stream
// and the call.  Through ctypes and the checks in Python a call cost 5.8 us, most of it not the runtime's launch: quantize and
// dequantize of 262 K binary32 elements, whose kernels take 3.4 us each, 11.6 us, now 7.9; a weight gradient of one small tile 6.8 -> 5.4.
//
// Every function takes the arguments of the entry point of its name and returns its status, or None without having done anything where
// an argument is not what the usual call has: then the caller goes on with the general checks, which either raise or make the call.
// Usual are plain tensors (no subclasses, no wrappers of a tracer or of vmap) on a device, contiguous, of the right type and large enough.
#define PY_SSIZE_T_CLEAN
#include <ATen/TensorSubclassLikeUtils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "daf.h"
#include "daf_block.h"

namespace {

struct Library {
  decltype(&daf_quantize_pack) quantize_pack;
  decltype(&daf_quantize_pack_static) quantize_pack_static;
  decltype(&daf_unpack_dequantize) unpack_dequantize;
  decltype(&daf_quantize_pack_metrics) quantize_pack_metrics;
  decltype(&daf_relu_quantize_pack) relu_quantize_pack;
  decltype(&daf_unpack_relu_backward) unpack_relu_backward;
  decltype(&daf_group_minmax) group_minmax;
  decltype(&daf_select_bits) select_bits;
  decltype(&daf_select_bits_from_scale) select_bits_from_scale;
  decltype(&daf_select_bits_workspace_bytes) select_bits_workspace_bytes;
  decltype(&daf_plan_update) plan_update;
  decltype(&daf_linear_quantize_pack) linear_quantize_pack;
  decltype(&daf_unpack_matmul_grad_weight) unpack_matmul_grad_weight;
  decltype(&daf_unpack_matmul_workspace_bytes) unpack_matmul_workspace_bytes;
  decltype(&daf_plan_num_elements) plan_num_elements;
  decltype(&daf_plan_num_groups) plan_num_groups;
  decltype(&daf_plan_packed_words) plan_packed_words;
} lib;
struct BlockLibrary {                                    // daf_block.h
  decltype(&daf_clip_grad_norm) clip_grad_norm;
  decltype(&daf_grad_norm_workspace_bytes) grad_norm_workspace_bytes;
  decltype(&daf_residual_norm) residual_norm;
  decltype(&daf_residual_norm_backward) residual_norm_backward;
  decltype(&daf_residual_norm_backward_workspace_bytes) residual_norm_backward_workspace_bytes;
  decltype(&daf_gated_linear) gated_linear;
  decltype(&daf_gated_linear_workspace_bytes) gated_linear_workspace_bytes;
  decltype(&daf_gated_linear_backward) gated_linear_backward;
  decltype(&daf_gated_linear_backward_workspace_bytes) gated_linear_backward_workspace_bytes;
} block = {};
PyObject* plan_type = nullptr;
PyObject* handle_name = nullptr;
PyObject* stream_name = nullptr;

// What one call's arguments amount to; `ok` stays true as long as all of them are usual.
struct Call {
  bool ok = true;
  daf_plan_t* plan = nullptr;
  int64_t elements = 0, groups = 0;
  void* stream = nullptr;

  void with_plan(PyObject* o) {
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != plan_type) { ok = false; return; }
    PyObject* h = PyObject_GetAttr(o, handle_name);
    plan = h != nullptr && PyLong_CheckExact(h) ? static_cast<daf_plan_t*>(PyLong_AsVoidPtr(h)) : nullptr;
    Py_XDECREF(h);
    if (PyErr_Occurred()) PyErr_Clear();
    if (plan == nullptr) { ok = false; return; }
    elements = lib.plan_num_elements(plan);
    groups = lib.plan_num_groups(plan);
  }
  void with_stream(PyObject* o) {
    if (!ok) return;
    if (o == Py_None) {
      stream = c10::hip::getCurrentHIPStream().stream();
      return;
    }
    PyObject* h = PyObject_GetAttr(o, stream_name);
    if (h == nullptr || !PyLong_CheckExact(h)) ok = false;
    else stream = PyLong_AsVoidPtr(h);
    Py_XDECREF(h);
    if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
  }
  const at::Tensor* tensor(PyObject* o) {
    if (!ok) return nullptr;
    if (THPVariable_CheckExact(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      if (t.defined() && !at::isTensorSubclassLike(t) && t.is_cuda() && t.has_storage() && t.is_contiguous()) return &t;
    }
    ok = false;
    return nullptr;
  }
  void* data(PyObject* o, at::ScalarType type, int64_t least) {
    const at::Tensor* t = tensor(o);
    if (t == nullptr || t->scalar_type() != type || t->numel() < least) { ok = false; return nullptr; }
    return t->data_ptr();
  }
  void* bytes(PyObject* o, int64_t least) {              // of any type
    const at::Tensor* t = tensor(o);
    if (t == nullptr || t->numel() * (int64_t)t->element_size() < least) { ok = false; return nullptr; }
    return t->data_ptr();
  }
  static int dtype_of(at::ScalarType type) {
    return type == at::kFloat ? DAF_F32 : type == at::kHalf ? DAF_F16 : type == at::kBFloat16 ? DAF_BF16 : -1;
  }
  // a tensor of the plan's size in one of the element formats; `dtype` -1: any, and it is told
  void* activation(PyObject* o, int& dtype) {
    const at::Tensor* t = tensor(o);
    const int d = t != nullptr ? dtype_of(t->scalar_type()) : -1;
    if (d < 0 || (dtype >= 0 && d != dtype) || t->numel() != elements) { ok = false; return nullptr; }
    dtype = d;
    return t->data_ptr();
  }
  struct Packed { uint32_t* words; float *min, *scale; };
  Packed packed(PyObject* words, PyObject* min, PyObject* scale) {
    Packed p;
    p.words = static_cast<uint32_t*>(data(words, at::kInt, ok ? lib.plan_packed_words(plan) : 0));
    p.min = static_cast<float*>(data(min, at::kFloat, groups));
    p.scale = static_cast<float*>(data(scale, at::kFloat, groups));
    return p;
  }
  const uint8_t* widths(PyObject* o) {                   // or None
    return o == Py_None ? nullptr : static_cast<const uint8_t*>(data(o, at::kByte, groups));
  }
  uint64_t seed(PyObject* o) {
    if (!PyLong_CheckExact(o)) { ok = false; return 0; }
    return PyLong_AsUnsignedLongLongMask(o);
  }
};

// Runs `make(call)`, which fills in the call and returns what is to be done without the interpreter's lock.
template <class Make>
PyObject* run(Py_ssize_t got, Py_ssize_t wanted, Make make) {
  try {
    Call c;
    if (got != wanted || plan_type == nullptr) c.ok = false;             // (nothing bound yet)
    if (c.ok) {
      auto call = make(c);
      if (c.ok) {
        int rc;
        // (An exception from the library's C functions ends the process, as it did on its way through ctypes: caught below, it would
        // come back to the interpreter without the lock.)
        auto without_the_lock = [&]() noexcept { rc = call(); };
        Py_BEGIN_ALLOW_THREADS
        without_the_lock();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
      }
    }
  } catch (...) {                                        // (a tensor that gives no pointer: the general way says so)
  }
  Py_RETURN_NONE;
}
using Args = PyObject* const*;

template <class F>
PyObject* quantize(F fn, Args a, Py_ssize_t n) {
  return run(n, 7, [&](Call& c) {
    c.with_plan(a[0]);
    int dt = -1;
    const void* x = c.activation(a[1], dt);
    const uint64_t seed = c.seed(a[2]);
    const auto p = c.packed(a[3], a[4], a[5]);
    c.with_stream(a[6]);
    return [=] { return fn(c.plan, x, static_cast<daf_dtype_t>(dt), seed, p.words, p.min, p.scale, c.stream); };
  });
}
PyObject* quantize_pack(PyObject*, Args a, Py_ssize_t n) { return quantize(lib.quantize_pack, a, n); }
PyObject* quantize_pack_static(PyObject*, Args a, Py_ssize_t n) { return quantize(lib.quantize_pack_static, a, n); }

PyObject* unpack_dequantize(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 7, [&](Call& c) {
    c.with_plan(a[0]);
    const auto p = c.packed(a[1], a[2], a[3]);
    int dt = -1;
    void* out = c.activation(a[4], dt);
    const uint8_t* bits = c.widths(a[5]);
    c.with_stream(a[6]);
    return [=] { return lib.unpack_dequantize(c.plan, p.words, p.min, p.scale, bits, out, static_cast<daf_dtype_t>(dt), c.stream); };
  });
}

PyObject* quantize_pack_metrics(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c) {
    c.with_plan(a[0]);
    int dt = -1;
    const void* x = c.activation(a[1], dt);
    const uint64_t seed = c.seed(a[2]);
    const auto p = c.packed(a[3], a[4], a[5]);
    float* metrics = static_cast<float*>(c.data(a[6], at::kFloat, 3 * c.groups));
    c.with_stream(a[7]);
    return [=] { return lib.quantize_pack_metrics(c.plan, x, static_cast<daf_dtype_t>(dt), seed, p.words, p.min, p.scale, metrics, c.stream); };
  });
}

PyObject* relu_quantize_pack(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c) {
    c.with_plan(a[0]);
    int dt = -1;
    const void* z = c.activation(a[1], dt);
    const uint64_t seed = c.seed(a[2]);
    void* y = c.activation(a[3], dt);
    const auto p = c.packed(a[4], a[5], a[6]);
    c.with_stream(a[7]);
    return [=] { return lib.relu_quantize_pack(c.plan, z, static_cast<daf_dtype_t>(dt), seed, y, p.words, p.min, p.scale, c.stream); };
  });
}

PyObject* unpack_relu_backward(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 8, [&](Call& c) {
    c.with_plan(a[0]);
    const auto p = c.packed(a[1], a[2], a[3]);
    int dt = -1;
    const void* grad_y = c.activation(a[4], dt);
    void* grad_z = c.activation(a[5], dt);
    const uint8_t* bits = c.widths(a[6]);
    c.with_stream(a[7]);
    return [=] { return lib.unpack_relu_backward(c.plan, p.words, p.min, p.scale, bits, grad_y, grad_z, static_cast<daf_dtype_t>(dt), c.stream); };
  });
}

PyObject* group_minmax(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 5, [&](Call& c) {
    c.with_plan(a[0]);
    int dt = -1;
    const void* x = c.activation(a[1], dt);
    float* lo = static_cast<float*>(c.data(a[2], at::kFloat, c.groups));
    float* hi = static_cast<float*>(c.data(a[3], at::kFloat, c.groups));
    c.with_stream(a[4]);
    return [=] { return lib.group_minmax(c.plan, x, static_cast<daf_dtype_t>(dt), lo, hi, c.stream); };
  });
}

PyObject* plan_update(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 3, [&](Call& c) {
    c.with_plan(a[0]);
    const uint8_t* bits = static_cast<const uint8_t*>(c.data(a[1], at::kByte, c.groups));
    if (c.ok && THPVariable_Unpack(a[1]).numel() != c.groups) c.ok = false;
    c.with_stream(a[2]);
    return [=] { return lib.plan_update(c.plan, bits, c.stream); };
  });
}

struct Classes {
  uint8_t of[4];
  int32_t n = 0;
};
Classes classes_of(Call& c, PyObject* o) {               // a list or tuple of up to four whole numbers
  Classes k;
  const bool list = PyList_CheckExact(o), tuple = PyTuple_CheckExact(o);
  const Py_ssize_t n = list ? PyList_GET_SIZE(o) : tuple ? PyTuple_GET_SIZE(o) : -1;
  if (n < 1 || n > 4) { c.ok = false; return k; }
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* v = list ? PyList_GET_ITEM(o, i) : PyTuple_GET_ITEM(o, i);
    if (!PyLong_CheckExact(v)) { c.ok = false; return k; }
    k.of[k.n++] = (uint8_t)PyLong_AsUnsignedLongLongMask(v);
  }
  return k;
}

// group_min, group_max (or group_scale, prev_bits), classes, out_bits, workspace, stream
PyObject* select(Args a, Py_ssize_t n, bool from_scale) {
  return run(n, 6, [&](Call& c) {
    const float* first = static_cast<const float*>(c.data(a[0], at::kFloat, 1));
    const int64_t G = c.ok ? THPVariable_Unpack(a[0]).numel() : 0;
    const float* max = nullptr;
    const uint8_t* prev = nullptr;
    int32_t uniform = 0;
    if (from_scale && PyLong_CheckExact(a[1])) {
      const long v = PyLong_AsLong(a[1]);
      if (PyErr_Occurred()) PyErr_Clear();
      if (v < 1 || v > 8) c.ok = false;
      uniform = (int32_t)v;
    } else {
      void* second = c.data(a[1], from_scale ? at::kByte : at::kFloat, G);
      if (c.ok && THPVariable_Unpack(a[1]).numel() != G) c.ok = false;
      if (from_scale) prev = static_cast<const uint8_t*>(second);
      else max = static_cast<const float*>(second);
    }
    const Classes k = classes_of(c, a[2]);
    uint8_t* out = static_cast<uint8_t*>(c.data(a[3], at::kByte, G));
    void* ws = c.data(a[4], at::kByte, c.ok ? lib.select_bits_workspace_bytes(G) : 0);
    c.with_stream(a[5]);
    return [=] {
      return from_scale ? lib.select_bits_from_scale(first, prev, uniform, G, k.of, k.n, out, ws, c.stream)
                        : lib.select_bits(first, max, G, k.of, k.n, out, ws, c.stream);
    };
  });
}
PyObject* select_bits(PyObject*, Args a, Py_ssize_t n) { return select(a, n, false); }
PyObject* select_bits_from_scale(PyObject*, Args a, Py_ssize_t n) { return select(a, n, true); }

// plan, x [M, K], weight [N, K], seed, out_y, out_words, out_min, out_scale, stream
PyObject* linear_quantize_pack(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 9, [&](Call& c) {
    c.with_plan(a[0]);
    const at::Tensor *x = c.tensor(a[1]), *w = c.tensor(a[2]);
    int64_t N = 0, K = 0;
    if (c.ok) {
      if (x->dim() != 2 || w->dim() != 2 || x->size(1) != w->size(1) || x->scalar_type() != w->scalar_type()) c.ok = false;
      else { N = w->size(0); K = x->size(1); }
      if (c.ok && x->size(0) * N != c.elements) c.ok = false;
    }
    int dt = c.ok ? Call::dtype_of(x->scalar_type()) : -1;
    if (dt < 0) c.ok = false;
    const uint64_t seed = c.seed(a[3]);
    void* y = c.activation(a[4], dt);
    const auto p = c.packed(a[5], a[6], a[7]);
    c.with_stream(a[8]);
    const void *px = c.ok ? x->data_ptr() : nullptr, *pw = c.ok ? w->data_ptr() : nullptr;
    return [=] { return lib.linear_quantize_pack(c.plan, px, pw, N, K, static_cast<daf_dtype_t>(dt), seed, y, p.words, p.min, p.scale, c.stream); };
  });
}

// plan, words, min, scale, grad_y [M, N], out_grad_w [N, K], workspace or None, bits or None, stream
PyObject* unpack_matmul_grad_weight(PyObject*, Args a, Py_ssize_t n) {
  return run(n, 9, [&](Call& c) {
    c.with_plan(a[0]);
    const auto p = c.packed(a[1], a[2], a[3]);
    const at::Tensor *gy = c.tensor(a[4]), *gw = c.tensor(a[5]);
    int64_t N = 0, K = 0;
    if (c.ok) {
      if (gy->dim() != 2 || gw->dim() != 2 || gw->scalar_type() != at::kFloat) c.ok = false;
      else { N = gw->size(0); K = gw->size(1); }
      if (c.ok && (gy->size(1) != N || K < 1 || gy->size(0) * K != c.elements)) c.ok = false;
    }
    const int dt = c.ok ? Call::dtype_of(gy->scalar_type()) : -1;
    if (dt < 0) c.ok = false;
    const int64_t need = c.ok ? lib.unpack_matmul_workspace_bytes(c.plan, N, K) : -1;
    if (need < 0) c.ok = false;
    void* ws = a[6] == Py_None ? nullptr : c.bytes(a[6], need);
    const uint8_t* bits = c.widths(a[7]);
    c.with_stream(a[8]);
    const void* pg = c.ok ? gy->data_ptr() : nullptr;
    float* out = c.ok ? static_cast<float*>(gw->data_ptr()) : nullptr;
    return [=] { return lib.unpack_matmul_grad_weight(c.plan, p.words, p.min, p.scale, bits, pg, N, K, static_cast<daf_dtype_t>(dt), out, ws, c.stream); };
  });
}

// ---- the calls of daf_block.h ----
// Tensors of one call: one device, types and sizes told by the first of each sort.  None: null, where the call has that.
struct BlockCall : Call {
  int device = -2;
  const at::Tensor* on_device(PyObject* o) {
    const at::Tensor* t = tensor(o);
    if (t == nullptr) return nullptr;
    if (device == -2) device = t->get_device();
    if (t->get_device() != device) { ok = false; return nullptr; }
    return t;
  }
  // [rows, cols], whatever the leading dimensions are, of one of the element formats
  void* rows_of(PyObject* o, int& dtype, int64_t& rows, int64_t& cols) {
    const at::Tensor* t = on_device(o);
    const int d = t != nullptr ? dtype_of(t->scalar_type()) : -1;
    if (d < 0 || t->dim() < 1 || t->size(-1) < 1) { ok = false; return nullptr; }
    dtype = d;
    cols = t->size(-1);
    rows = t->numel() / cols;
    return t->data_ptr();
  }
  void* like(PyObject* o, const at::Tensor& first, bool optional) {     // the shape and type of another one
    if (optional && o == Py_None) return nullptr;
    const at::Tensor* t = on_device(o);
    if (t == nullptr || t->scalar_type() != first.scalar_type() || t->sizes() != first.sizes()) { ok = false; return nullptr; }
    return t->data_ptr();
  }
  void* matrix(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, bool optional) {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor* t = on_device(o);
    if (t == nullptr || t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) { ok = false; return nullptr; }
    return t->data_ptr();
  }
  void* vector(PyObject* o, at::ScalarType type, int64_t n) {           // or None
    if (o == Py_None) return nullptr;
    const at::Tensor* t = on_device(o);
    if (t == nullptr || t->scalar_type() != type || t->dim() != 1 || t->size(0) != n) { ok = false; return nullptr; }
    return t->data_ptr();
  }
  void* workspace(PyObject* o, int64_t need) {                          // or None where nothing is needed
    if (need < 0) { ok = false; return nullptr; }
    if (o == Py_None) { ok = ok && need == 0; return nullptr; }
    const at::Tensor* t = on_device(o);
    if (t == nullptr || t->numel() * (int64_t)t->element_size() < need) { ok = false; return nullptr; }
    return t->data_ptr();
  }
  int64_t number(PyObject* o) {
    if (!PyLong_CheckExact(o)) { ok = false; return 0; }
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &over);
    if (over != 0) ok = false;
    return v;
  }
  float real(PyObject* o) {
    if (!PyFloat_CheckExact(o)) { ok = false; return 0.0f; }
    return (float)PyFloat_AS_DOUBLE(o);
  }
  bool truth(PyObject* o) {
    if (o != Py_True && o != Py_False) ok = false;
    return o == Py_True;
  }
};
template <class Make>
PyObject* run_block(Py_ssize_t got, Py_ssize_t wanted, Make make) {
  return run(got, wanted, [&](Call& c) {
    BlockCall b;
    b.ok = c.ok && block.clip_grad_norm != nullptr;
    auto call = make(b);
    c.ok = b.ok;
    return call;
  });
}

// address of the items, their number, max_norm (clipping), out_norm, workspace, stream
PyObject* clip_grad_norm(PyObject*, Args a, Py_ssize_t n) {
  return run_block(n, 6, [&](BlockCall& c) {
    const auto* items = reinterpret_cast<const daf_grad_item_t*>(static_cast<intptr_t>(c.number(a[0])));
    const int32_t count = (int32_t)c.number(a[1]);
    const float most = c.real(a[2]);
    const at::Tensor* norm = c.ok ? c.on_device(a[3]) : nullptr;
    if (norm == nullptr || norm->scalar_type() != at::kFloat || norm->numel() != 1) c.ok = false;
    void* ws = c.ok ? c.workspace(a[4], block.grad_norm_workspace_bytes()) : nullptr;
    c.with_stream(a[5]);
    float* out = c.ok ? static_cast<float*>(norm->data_ptr()) : nullptr;
    return [=] { return block.clip_grad_norm(items, count, most, out, ws, c.stream); };
  });
}

// What the norms' two calls have in common, from `a`: kind, eps, scale, post, pre_weight, pre_bias, post_weight, post_bias, gate
daf_residual_norm_t norm_parameters(BlockCall& c, Args a, int dtype, at::ScalarType type, int64_t rows, int64_t cols, bool z) {
  daf_residual_norm_t p = {};
  p.rows = rows;
  p.cols = cols;
  p.dtype = dtype;
  p.kind = (int32_t)c.number(a[0]);
  p.eps = c.real(a[1]);
  p.scale = c.real(a[2]);
  p.post = c.truth(a[3]);
  p.pre_weight = c.vector(a[4], type, cols);
  p.pre_bias = c.vector(a[5], type, cols);
  p.post_weight = c.vector(a[6], type, cols);
  p.post_bias = c.vector(a[7], type, cols);
  p.gate_groups = 1;
  if (a[8] != Py_None) {
    const at::Tensor* g = c.on_device(a[8]);
    if (g == nullptr || g->scalar_type() != type || g->dim() < 1 || g->dim() > 2 || g->size(-1) != cols || g->numel() < 1) c.ok = false;
    if (c.ok) {
      p.gate = g->data_ptr();
      p.gate_groups = g->numel() / cols;
      if (rows % p.gate_groups != 0) c.ok = false;
    }
  }
  if (!z && (p.post || p.gate != nullptr)) c.ok = false;
  if (!p.post && (p.post_weight != nullptr || p.post_bias != nullptr)) c.ok = false;
  return p;
}

// residual, z, out_residual, out_y, out_stats, the nine of norm_parameters, stream
PyObject* residual_norm(PyObject*, Args a, Py_ssize_t n) {
  return run_block(n, 15, [&](BlockCall& c) {
    int dt = -1;
    int64_t rows = 0, cols = 0;
    const void* r = c.ok ? c.rows_of(a[0], dt, rows, cols) : nullptr;
    daf_residual_norm_t p = {};
    void *z = nullptr, *sum = nullptr, *y = nullptr, *stats = nullptr;
    if (c.ok) {
      const at::Tensor& first = THPVariable_Unpack(a[0]);
      z = c.like(a[1], first, true);
      sum = c.like(a[2], first, true);
      y = c.like(a[3], first, true);
      stats = c.matrix(a[4], at::kFloat, rows, 4, true);
      p = norm_parameters(c, a + 5, dt, first.scalar_type(), rows, cols, a[1] != Py_None);
    }
    c.with_stream(a[14]);
    return [=] { return block.residual_norm(&p, r, z, sum, y, static_cast<float*>(stats), c.stream); };
  });
}

// sum, z, stats, grad_y, grad_residual, out_grad_residual, out_grad_z, five gradients of vectors, workspace, the nine of norm_parameters, stream
PyObject* residual_norm_backward(PyObject*, Args a, Py_ssize_t n) {
  return run_block(n, 23, [&](BlockCall& c) {
    int dt = -1;
    int64_t rows = 0, cols = 0;
    void* dr = c.ok ? c.rows_of(a[5], dt, rows, cols) : nullptr;
    daf_residual_norm_t p = {};
    daf_residual_norm_grads_t grads = {};
    const void *sum = nullptr, *z = nullptr, *stats = nullptr, *dy = nullptr, *ds = nullptr;
    void *dz = nullptr, *ws = nullptr;
    if (c.ok) {
      const at::Tensor& first = THPVariable_Unpack(a[5]);
      sum = c.like(a[0], first, true);
      z = c.like(a[1], first, true);
      stats = c.matrix(a[2], at::kFloat, rows, 4, false);
      dy = c.like(a[3], first, true);
      ds = c.like(a[4], first, true);
      dz = c.like(a[6], first, true);
      p = norm_parameters(c, a + 13, dt, first.scalar_type(), rows, cols, a[1] != Py_None);
      grads.pre_weight = static_cast<float*>(c.vector(a[7], at::kFloat, cols));
      grads.pre_bias = static_cast<float*>(c.vector(a[8], at::kFloat, cols));
      grads.post_weight = static_cast<float*>(c.vector(a[9], at::kFloat, cols));
      grads.post_bias = static_cast<float*>(c.vector(a[10], at::kFloat, cols));
      if (a[11] != Py_None && c.ok) {
        const at::Tensor* g = c.on_device(a[11]);
        const bool as_gate = a[21] != Py_None;
        if (g == nullptr || g->scalar_type() != at::kFloat ||
            (as_gate ? g->sizes() != THPVariable_Unpack(a[21]).sizes() : g->dim() != 1 || g->size(0) != cols))
          c.ok = false;
        else
          grads.gate = static_cast<float*>(g->data_ptr());
      }
      const bool wanted = grads.pre_weight || grads.pre_bias || grads.post_weight || grads.post_bias || grads.gate;
      if (c.ok && (wanted || a[12] != Py_None))
        ws = c.workspace(a[12], wanted ? block.residual_norm_backward_workspace_bytes(rows, cols, p.gate_groups) : 0);
    }
    c.with_stream(a[22]);
    return [=] { return block.residual_norm_backward(&p, sum, z, static_cast<const float*>(stats), dy, ds, dr, dz, &grads, ws, c.stream); };
  });
}

struct GatedOperands {
  int dtype = -1;
  int64_t m = 0, n = 0, k = 0;
  const void *x = nullptr, *w_gate = nullptr, *w_up = nullptr;
  at::ScalarType type = at::kHalf;
};
GatedOperands gated_operands(BlockCall& c, PyObject* x, PyObject* w_gate, PyObject* w_up) {
  GatedOperands o;
  const at::Tensor *tx = c.on_device(x), *tg = c.on_device(w_gate);
  if (!c.ok || tx->dim() != 2 || tg->dim() != 2 || tx->size(1) != tg->size(1) || tg->numel() < 1 || tg->scalar_type() != tx->scalar_type()) {
    c.ok = false;
    return o;
  }
  o.type = tx->scalar_type();
  o.dtype = Call::dtype_of(o.type);
  if (o.dtype != DAF_F16 && o.dtype != DAF_BF16) c.ok = false;
  o.m = tx->size(0);
  o.k = tx->size(1);
  o.n = tg->size(0);
  o.x = tx->data_ptr();
  o.w_gate = tg->data_ptr();
  o.w_up = c.matrix(w_up, o.type, o.n, o.k, false);
  return o;
}

// x, w_gate, w_up, activation, out_h, workspace, out_gate, out_up, stream
PyObject* gated_linear(PyObject*, Args a, Py_ssize_t n) {
  return run_block(n, 9, [&](BlockCall& c) {
    const GatedOperands o = gated_operands(c, a[0], a[1], a[2]);
    const int act = (int)c.number(a[3]);
    void* h = c.matrix(a[4], o.type, o.m, o.n, false);
    void *gate = c.matrix(a[6], o.type, o.m, o.n, true), *up = c.matrix(a[7], o.type, o.m, o.n, true);
    if ((a[6] == Py_None) != (a[7] == Py_None)) c.ok = false;
    const auto dtype = static_cast<daf_dtype_t>(o.dtype);
    void* ws = c.ok ? c.workspace(a[5], block.gated_linear_workspace_bytes(o.m, o.n, o.k, dtype)) : nullptr;
    c.with_stream(a[8]);
    return [=] { return block.gated_linear(o.x, o.w_gate, o.w_up, o.m, o.n, o.k, dtype, act, h, gate, up, ws, c.stream); };
  });
}

// x, w_gate, w_up, grad_h, activation, out_grad_x, out_grad_w_gate, out_grad_w_up, workspace, gate, up, out_h, stream
PyObject* gated_linear_backward(PyObject*, Args a, Py_ssize_t n) {
  return run_block(n, 13, [&](BlockCall& c) {
    const GatedOperands o = gated_operands(c, a[0], a[1], a[2]);
    const void* gh = c.matrix(a[3], o.type, o.m, o.n, false);
    const int act = (int)c.number(a[4]);
    void* dx = c.matrix(a[5], o.type, o.m, o.k, true);
    void *dwg = c.matrix(a[6], o.type, o.n, o.k, true), *dwu = c.matrix(a[7], o.type, o.n, o.k, true);
    const void *gate = c.matrix(a[9], o.type, o.m, o.n, true), *up = c.matrix(a[10], o.type, o.m, o.n, true);
    void* h = c.matrix(a[11], o.type, o.m, o.n, true);
    if ((a[6] == Py_None) != (a[7] == Py_None) || (a[9] == Py_None) != (a[10] == Py_None) || (a[9] != Py_None && a[11] != Py_None)) c.ok = false;
    const auto dtype = static_cast<daf_dtype_t>(o.dtype);
    void* ws = c.ok ? c.workspace(a[8], block.gated_linear_backward_workspace_bytes(o.m, o.n, o.k, dtype)) : nullptr;
    c.with_stream(a[12]);
    return [=] {
      return block.gated_linear_backward(o.x, o.w_gate, o.w_up, gate, up, gh, o.m, o.n, o.k, dtype, act, dx, dwg, dwu, h, ws, c.stream);
    };
  });
}

struct Slot {
  const char* name;
  void* at;
};
// Fills the slots from {name: address}; false, with an exception set, where a name is missing.
bool fill(PyObject* table, const Slot* slots, size_t count) {
  for (size_t i = 0; i < count; ++i) {
    PyObject* v = PyDict_GetItemString(table, slots[i].name);
    void* address = v != nullptr ? PyLong_AsVoidPtr(v) : nullptr;
    if (address == nullptr) {
      if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "no address for %s", slots[i].name);
      return false;
    }
    *static_cast<void**>(slots[i].at) = address;
  }
  return true;
}

// bind_block({name: address}): where the functions of daf_block.h are.
PyObject* bind_block(PyObject*, PyObject* args) {
  PyObject* table;
  if (!PyArg_ParseTuple(args, "O!", &PyDict_Type, &table)) return nullptr;
  BlockLibrary found;
  const Slot slots[] = {
      {"daf_clip_grad_norm", &found.clip_grad_norm},
      {"daf_grad_norm_workspace_bytes", &found.grad_norm_workspace_bytes}, {"daf_residual_norm", &found.residual_norm},
      {"daf_residual_norm_backward", &found.residual_norm_backward},
      {"daf_residual_norm_backward_workspace_bytes", &found.residual_norm_backward_workspace_bytes}, {"daf_gated_linear", &found.gated_linear},
      {"daf_gated_linear_workspace_bytes", &found.gated_linear_workspace_bytes}, {"daf_gated_linear_backward", &found.gated_linear_backward},
      {"daf_gated_linear_backward_workspace_bytes", &found.gated_linear_backward_workspace_bytes}};
  if (!fill(table, slots, sizeof(slots) / sizeof(slots[0]))) return nullptr;
  block = found;
  Py_RETURN_NONE;
}

// bind({name: address}, Plan): where the library's functions are.
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *table, *type;
  if (!PyArg_ParseTuple(args, "O!O", &PyDict_Type, &table, &type)) return nullptr;
  Library found;
  const Slot slots[] = {
      {"daf_quantize_pack", &found.quantize_pack}, {"daf_quantize_pack_static", &found.quantize_pack_static},
      {"daf_unpack_dequantize", &found.unpack_dequantize}, {"daf_quantize_pack_metrics", &found.quantize_pack_metrics},
      {"daf_relu_quantize_pack", &found.relu_quantize_pack}, {"daf_unpack_relu_backward", &found.unpack_relu_backward},
      {"daf_group_minmax", &found.group_minmax}, {"daf_select_bits", &found.select_bits},
      {"daf_select_bits_from_scale", &found.select_bits_from_scale},
      {"daf_select_bits_workspace_bytes", &found.select_bits_workspace_bytes}, {"daf_plan_update", &found.plan_update},
      {"daf_linear_quantize_pack", &found.linear_quantize_pack},
      {"daf_unpack_matmul_grad_weight", &found.unpack_matmul_grad_weight},
      {"daf_unpack_matmul_workspace_bytes", &found.unpack_matmul_workspace_bytes},
      {"daf_plan_num_elements", &found.plan_num_elements}, {"daf_plan_num_groups", &found.plan_num_groups},
      {"daf_plan_packed_words", &found.plan_packed_words}};
  if (!fill(table, slots, sizeof(slots) / sizeof(slots[0]))) return nullptr;
  lib = found;
  Py_INCREF(type);
  Py_XSETREF(plan_type, type);
  Py_RETURN_NONE;
}

#define DAF_FAST(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {DAF_FAST(quantize_pack), DAF_FAST(quantize_pack_static), DAF_FAST(unpack_dequantize),
                         DAF_FAST(quantize_pack_metrics), DAF_FAST(relu_quantize_pack), DAF_FAST(unpack_relu_backward),
                         DAF_FAST(group_minmax), DAF_FAST(plan_update), DAF_FAST(select_bits), DAF_FAST(select_bits_from_scale),
                         DAF_FAST(linear_quantize_pack), DAF_FAST(unpack_matmul_grad_weight),
                         DAF_FAST(clip_grad_norm), DAF_FAST(residual_norm), DAF_FAST(residual_norm_backward), DAF_FAST(gated_linear),
                         DAF_FAST(gated_linear_backward), {"bind", bind, METH_VARARGS, nullptr}, {"bind_block", bind_block, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast_calls() {
  handle_name = PyUnicode_InternFromString("_h");
  stream_name = PyUnicode_InternFromString("cuda_stream");
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", DAF_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
