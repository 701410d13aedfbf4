// The operator calls that a decode step makes of its own, marshalled from torch tensors to
// the C ABI: checks, outputs from torch's allocator, one call.  Through ctypes a router call
// of 64 tokens spends 17 us in the interpreter for 5.6 us of kernel; nothing else is here.
// The library's functions come from the handle that binding.py loaded (bind()).
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <optional>

#include "tuna.h"

namespace {

#define TUNA_CALLS(X)                                                                                       \
  X(tuna_moe_route_workspace_bytes) X(tuna_moe_route) X(tuna_moe_route_backward) X(tuna_fp8_quantize) \
  X(tuna_fp8_matmul) X(tuna_moe_few)
#define X(f) decltype(&f) p_##f = nullptr;
TUNA_CALLS(X)
#undef X
PyObject *raise_status = nullptr;  // moe._check: turns a status into a TunaError

using at::Tensor;

struct Refused {};  // a Python error is set

[[noreturn]] void refuse(const char *format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(PyExc_ValueError, format, args);
  va_end(args);
  throw Refused();
}

int dtype_of(const Tensor &t) {
  switch (t.scalar_type()) {
    case at::kFloat: return TUNA_DTYPE_F32;
    case at::kBFloat16: return TUNA_DTYPE_BF16;
    case at::kFloat8_e4m3fn: return TUNA_DTYPE_E4M3;
    default: return -1;
  }
}

const Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) refuse("%s: a tensor is wanted", name);
  const Tensor &t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse("%s: a CUDA tensor is wanted", name);
  return t;
}

// A matrix whose rows are contiguous and do not overlap; its row pitch.
int64_t matrix(const Tensor &t, const char *name, bool f32, bool bf16, bool e4m3) {
  const int d = dtype_of(t);
  if (t.dim() != 2 || !((f32 && d == TUNA_DTYPE_F32) || (bf16 && d == TUNA_DTYPE_BF16) || (e4m3 && d == TUNA_DTYPE_E4M3)))
    refuse("%s: a CUDA matrix of%s%s%s is wanted", name, f32 ? " float32" : "", bf16 ? " bfloat16" : "", e4m3 ? " float8_e4m3fn" : "");
  const int64_t rows = t.size(0), cols = t.size(1);
  if ((cols > 1 && t.stride(1) != 1) || (rows > 1 && t.stride(0) < cols))
    refuse("%s: rows must be contiguous and must not overlap (strides %lld, %lld)", name, (long long)t.stride(0), (long long)t.stride(1));
  return rows > 1 ? t.stride(0) : std::max<int64_t>(cols, 1);
}

void dense(const Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape, const Tensor &with) {
  if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous()) {
    std::string s;
    for (const int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
    refuse("%s: a contiguous CUDA tensor of %s, shape (%s), is wanted", name, c10::toString(type), s.c_str());
  }
  if (t.device() != with.device()) refuse("%s: on another device than its fellow", name);
}

Tensor make(at::IntArrayRef shape, at::ScalarType type, const Tensor &like) {
  return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}

// Where a call runs: on the device of its tensors and on torch's current stream, or on the stream that was given,
// which is torch's current one until the call returns.  Workspaces, copies and outputs then belong to the stream that
// the kernels run on: what is freed at the end is taken again behind them, and no copy runs beside them.
class Place {
 public:
  Place(PyObject *o, const Tensor &t) : device_(t.device()), before_(c10::cuda::getCurrentCUDAStream(t.device().index())), at_(before_) {
    if (o == Py_None) return;
    cudaStream_t raw = (cudaStream_t)handle(o);
    if (raw == cudaStreamLegacy) raw = nullptr;  // torch's name of the same stream
    if (raw == before_.stream()) return;
    at_ = c10::cuda::getStreamFromExternal(raw, t.device().index());
    guard_.emplace(at_);
  }
  void *stream() const { return at_.stream(); }
  // An output on its way to the caller, who may use and free it on the stream that was current before.
  const Tensor &out(const Tensor &t) const {
    if (guard_) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), before_);
    return t;
  }

 private:
  static void *handle(PyObject *o) {
    PyObject *s = PyLong_Check(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, "cuda_stream");
    if (!s) throw Refused();
    void *p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) throw Refused();
    return p;
  }
  c10::cuda::CUDAGuard device_;
  c10::cuda::CUDAStream before_, at_;
  std::optional<c10::cuda::CUDAStreamGuard> guard_;
};

int64_t integer(PyObject *o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int small(PyObject *o) {  // what does not fit an int is beyond every limit of the library: let it say so
  return (int)std::min<int64_t>(std::max<int64_t>(integer(o), INT32_MIN), INT32_MAX);
}
double number(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused();
  return v;
}
bool truth(PyObject *o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused();
  return v != 0;
}

void check(int rc, const char *what) {
  if (rc == TUNA_OK) return;
  PyObject *r = raise_status ? PyObject_CallFunction(raise_status, "is", rc, what) : nullptr;
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_Format(PyExc_RuntimeError, "%s: status %d", what, rc);
  throw Refused();
}

void *at_of(const Tensor &t) { return t.data_ptr(); }
int clip(int64_t n) { return (int)std::min<int64_t>(n, INT32_MAX); }

template <typename... T>
PyObject *pack(const T &...t) {
  PyObject *r = PyTuple_New(sizeof...(T));
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  (PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t)), ...);
  return r;
}

// Runs f; turns its refusals and C++ exceptions into Python's.
template <typename F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F f) {
  if (have != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, got %zd", want, have);
    return nullptr;
  }
  try {
    return f();
  } catch (const Refused &) {
    return nullptr;
  } catch (const c10::OutOfMemoryError &e) {
    PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    return nullptr;
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// route(logits, k, scoring, renormalize, scale, ranks, stream)
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const Tensor &z = tensor(a[0], "logits");
    const int64_t ld = matrix(z, "logits", true, true, false), t = z.size(0), e = z.size(1), k = integer(a[1]), ranks = integer(a[5]);
    if (ranks < 1 || t % ranks) refuse("%lld tokens do not divide over %lld ranks", (long long)t, (long long)ranks);
    size_t need = 0;
    const Place place(a[6], z);
    check(p_tuna_moe_route_workspace_bytes(t, clip(e), clip(k), clip(ranks), &need), "tuna_moe_route_workspace_bytes");
    Tensor ws;
    if (need) ws = make({(int64_t)need}, at::kByte, z);
    const Tensor ids = make({t, k}, at::kInt, z), weights = make({t, k}, at::kFloat, z), counts = make({ranks, e}, at::kLong, z),
                 offsets = make({ranks * e + 1}, at::kLong, z), rows = make({t * k}, at::kLong, z), pos = make({t, k}, at::kLong, z);
    check(p_tuna_moe_route(at_of(z), dtype_of(z), t, clip(e), ld, clip(k), clip(ranks), small(a[2]), truth(a[3]), (float)number(a[4]),
                           (int32_t *)at_of(ids), (float *)at_of(weights), (int64_t *)at_of(counts), (int64_t *)at_of(offsets),
                           (int64_t *)at_of(rows), (int64_t *)at_of(pos), need ? at_of(ws) : nullptr, need, place.stream()),
          "tuna_moe_route");
    return pack(place.out(ids), place.out(weights), place.out(counts), place.out(offsets), place.out(rows), place.out(pos));
  });
}

// route_backward(logits, ids, dweights, scoring, renormalize, scale, stream)
PyObject *route_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const Tensor &z = tensor(a[0], "logits"), &ids = tensor(a[1], "ids"), &dw = tensor(a[2], "dweights");
    const int64_t ld = matrix(z, "logits", true, true, false), t = z.size(0), e = z.size(1);
    if (ids.dim() != 2) refuse("ids: [tokens, k] is wanted");
    const int64_t k = ids.size(1);
    dense(ids, "ids", at::kInt, {t, k}, z);
    dense(dw, "dweights", at::kFloat, {t, k}, z);
    const Place place(a[6], z);
    const Tensor d = make({t, e}, z.scalar_type(), z);
    check(p_tuna_moe_route_backward(at_of(z), dtype_of(z), t, clip(e), ld, clip(k), small(a[3]), truth(a[4]), (float)number(a[5]),
                                    (const int32_t *)at_of(ids), (const float *)at_of(dw), at_of(d), e, place.stream()),
          "tuna_moe_route_backward");
    return THPVariable_Wrap(place.out(d));
  });
}

// fp8_quantize(x, layout, stream)
PyObject *fp8_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 3, [&] {
    const Tensor &x = tensor(a[0], "x");
    const int64_t ld = matrix(x, "x", true, true, false), rows = x.size(0), cols = x.size(1);
    const int layout = small(a[1]);
    const bool turned = layout == TUNA_FP8_COLUMNS || layout == TUNA_FP8_TILES_T, tiles = layout >= TUNA_FP8_TILES;
    const int64_t out_rows = turned ? cols : rows, out_cols = turned ? rows : cols, pitch = (out_cols + 15) / 16 * 16;
    const int64_t blocks = (out_cols + 127) / 128;
    const Place place(a[2], x);
    Tensor q = make({out_rows, pitch}, at::kFloat8_e4m3fn, x);
    const Tensor scale = tiles ? make({(out_rows + 127) / 128, blocks}, at::kFloat, x) : make({blocks, out_rows}, at::kFloat, x);
    check(p_tuna_fp8_quantize(at_of(x), dtype_of(x), rows, clip(cols), ld, layout, at_of(q), std::max<int64_t>(pitch, 16),
                              (float *)at_of(scale), place.stream()),
          "tuna_fp8_quantize");
    place.out(q), place.out(scale);
    return pack(pitch == out_cols ? q : q.narrow(1, 0, out_cols), scale);
  });
}

// An e4m3 operand whose rows start on 16-byte boundaries: the tensor itself, or a copy.
Tensor operand(const Tensor &q, const char *name, int64_t &ld) {
  ld = matrix(q, name, false, false, true);
  if (q.size(0) <= 1) ld = (q.size(1) + 15) / 16 * 16;  // the pitch of a single row is free
  if (ld % 16 == 0 && (uintptr_t)q.data_ptr() % 16 == 0) {
    ld = std::max<int64_t>(ld, 16);
    return q;
  }
  ld = std::max<int64_t>((q.size(1) + 15) / 16 * 16, 16);
  Tensor p = make({q.size(0), ld}, at::kByte, q).zero_();
  p.narrow(1, 0, q.size(1)).copy_(q.view(at::kByte));
  return p;
}

// fp8_matmul(a, a_scale, b, b_scale, offsets, b_layout, out_dtype, stream)
PyObject *fp8_matmul(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const Tensor &left = tensor(a[0], "a"), &sa = tensor(a[1], "a_scale"), &right = tensor(a[2], "b"), &sb = tensor(a[3], "b_scale");
    if (right.device() != left.device()) refuse("b: on another device than its fellow");
    const Place place(a[7], left);
    int64_t lda = 0, ldb = 0, groups = 1, cols, kb;
    const Tensor x = operand(left, "a", lda);
    const int64_t m = left.size(0), k = left.size(1), blocks = (k + 127) / 128;
    const int layout = small(a[5]), out = small(a[6]);
    const int64_t *offsets = nullptr;
    Tensor w;
    if (a[4] != Py_None) {
      if (right.dim() != 3 || !right.is_contiguous() || layout != TUNA_FP8_TILES)
        refuse("b: contiguous matrices [groups, n, k] with tile scales go with offsets");
      groups = right.size(0), cols = right.size(1), kb = right.size(2);
      if (kb != k) refuse("a has %lld columns, b %lld", (long long)k, (long long)kb);
      const Tensor &o = tensor(a[4], "offsets");
      dense(o, "offsets", at::kLong, {groups + 1}, left);
      offsets = (const int64_t *)at_of(o);
      w = operand(right.view({groups * cols, kb}), "b", ldb);
      dense(sb, "b_scale", at::kFloat, {groups, (cols + 127) / 128, blocks}, left);
    } else {
      w = operand(right, "b", ldb);
      cols = right.size(0), kb = right.size(1);
      if (kb != k) refuse("a has %lld columns, b %lld", (long long)k, (long long)kb);
      if (layout == TUNA_FP8_TILES)
        dense(sb, "b_scale", at::kFloat, {(cols + 127) / 128, blocks}, left);
      else
        dense(sb, "b_scale", at::kFloat, {blocks, cols}, left);
    }
    dense(sa, "a_scale", at::kFloat, {blocks, m}, left);
    const Tensor y = make({m, cols}, out == TUNA_DTYPE_F32 ? at::kFloat : at::kBFloat16, left);
    check(p_tuna_fp8_matmul(at_of(x), (const float *)at_of(sa), m, lda, at_of(w), (const float *)at_of(sb), layout, clip(cols), ldb, clip(k),
                            clip(groups), offsets, at_of(y), out, std::max<int64_t>(cols, 1), place.stream()),
          "tuna_fp8_matmul");
    return THPVariable_Wrap(place.out(y));
  });
}

// few(x, router, k, w13, w2, s13, s2, scoring, renormalize, scale, ids, weights, workspace, stream)
PyObject *few(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 14, [&] {
    const Tensor &given = tensor(a[0], "x"), &router = tensor(a[1], "router"), &w13 = tensor(a[3], "w13"), &w2 = tensor(a[4], "w2");
    int64_t ld = matrix(given, "x", false, true, false);
    const int64_t t = given.size(0), d = given.size(1), k = integer(a[2]);
    if (router.dim() != 2) refuse("router: [experts, hidden] is wanted");
    const int64_t e = router.size(0);
    dense(router, "router", at::kBFloat16, {e, d}, given);
    if (w13.dim() != 4) refuse("w13: [experts, 2, inter, hidden] is wanted");
    const int64_t i = w13.size(2), bi = (i + 127) / 128, bd = (d + 127) / 128;
    const bool fp8 = w13.scalar_type() == at::kFloat8_e4m3fn;
    const at::ScalarType type = fp8 ? at::kFloat8_e4m3fn : at::kBFloat16;
    dense(w13, "w13", type, {e, 2, i, d}, given);
    dense(w2, "w2", type, {e, d, i}, given);
    const float *s13 = nullptr, *s2 = nullptr;
    if (fp8) {
      if (a[5] == Py_None || a[6] == Py_None) refuse("8-bit weights need s13 and s2");
      const Tensor &p = tensor(a[5], "s13"), &q = tensor(a[6], "s2");
      dense(p, "s13", at::kFloat, {e, 2, bi, bd}, given);
      dense(q, "s2", at::kFloat, {e, bd, bi}, given);
      s13 = (const float *)at_of(p), s2 = (const float *)at_of(q);
    }
    int32_t *ids = nullptr;
    float *weights = nullptr;
    if (a[10] != Py_None) {
      const Tensor &o = tensor(a[10], "ids");
      dense(o, "ids", at::kInt, {t, k}, given);
      ids = (int32_t *)at_of(o);
    }
    if (a[11] != Py_None) {
      const Tensor &o = tensor(a[11], "weights");
      dense(o, "weights", at::kFloat, {t, k}, given);
      weights = (float *)at_of(o);
    }
    const Tensor &ws = tensor(a[12], "workspace");
    if (!ws.is_contiguous()) refuse("workspace: a contiguous tensor is wanted");
    if (ws.device() != given.device()) refuse("workspace: on another device than its fellow");
    const Place place(a[13], given);
    Tensor x = given;
    if (ld % 8 || (uintptr_t)given.data_ptr() % 16) x = given.clone(at::MemoryFormat::Contiguous), ld = d;
    const Tensor out = make({t, d}, at::kBFloat16, given);
    check(p_tuna_moe_few(at_of(x), ld, clip(t), at_of(router), clip(e), clip(k), small(a[7]), truth(a[8]), (float)number(a[9]), clip(d), clip(i),
                         fp8 ? TUNA_DTYPE_E4M3 : TUNA_DTYPE_BF16, at_of(w13), s13, at_of(w2), s2, at_of(out), std::max<int64_t>(d, 1), ids, weights,
                         at_of(ws), (size_t)ws.nbytes(), place.stream()),
          "tuna_moe_few");
    return THPVariable_Wrap(place.out(out));
  });
}

// bind(handle of the loaded library, raise_status)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 2, [&]() -> PyObject * {
    void *handle = PyLong_AsVoidPtr(a[0]);
    if (PyErr_Occurred()) throw Refused();
#define X(f)                                                  \
  p_##f = (decltype(&f))dlsym(handle, #f);                    \
  if (!p_##f) {                                               \
    PyErr_SetString(PyExc_RuntimeError, "no " #f " in the library"); \
    throw Refused();                                          \
  }
    TUNA_CALLS(X)
#undef X
    Py_XSETREF(raise_status, Py_NewRef(a[1]));
    Py_RETURN_NONE;
  });
}

#define F(f) {#f, (PyCFunction)(void (*)())f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {F(route), F(route_backward), F(fp8_quantize), F(fp8_matmul), F(few), F(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tuna_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit_tuna_torch() { return PyModule_Create(&module); }
