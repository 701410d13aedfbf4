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
#include <torch/version.h>

#include <algorithm>
#include <optional>
#include <utility>

#include "tuna.h"

namespace {

#define TUNA_CALLS(X)                                                                                       \
  X(tuna_moe_route_workspace_bytes) X(tuna_moe_route) X(tuna_moe_route_backward) X(tuna_fp8_quantize) \
  X(tuna_fp8_matmul) X(tuna_moe_few) X(tuna_moe_balance_workspace_bytes) X(tuna_moe_balance) X(tuna_moe_balance_backward)  \
  X(tuna_fp4_quantize) X(tuna_fp4_dequantize) X(tuna_fp4_align) X(tuna_fp4_matmul) X(tuna_fp4_expert_rows_workspace_bytes) X(tuna_fp4_expert_rows) \
  X(tuna_fp4_experts_workspace_bytes) X(tuna_fp4_experts)
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
int clip(int64_t n) { return (int)std::min<int64_t>(std::max<int64_t>(n, INT32_MIN), INT32_MAX); }
int small(PyObject *o) {  // what does not fit an int is beyond every limit of the library: let it say so
  return clip(integer(o));
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

// The segments' bounds: int64 [segments + 1], or None for one segment.
const int64_t *segments_of(PyObject *o, const Tensor &with, int64_t &segments) {
  segments = 1;
  if (o == Py_None) return nullptr;
  const Tensor &t = tensor(o, "offsets");
  if (t.dim() != 1 || t.size(0) < 2) refuse("offsets: [segments + 1] is wanted");
  segments = t.size(0) - 1;
  dense(t, "offsets", at::kLong, {segments + 1}, with);
  return (const int64_t *)at_of(t);
}

// balance(logits, ids, scoring, offsets, stream)
PyObject *balance(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const Tensor &z = tensor(a[0], "logits"), &ids = tensor(a[1], "ids");
    const int64_t ld = matrix(z, "logits", true, true, false), t = z.size(0), e = z.size(1);
    if (ids.dim() != 2) refuse("ids: [tokens, k] is wanted");
    const int64_t k = ids.size(1);
    dense(ids, "ids", at::kInt, {t, k}, z);
    int64_t segments;
    const int64_t *offsets = segments_of(a[3], z, segments);
    const Place place(a[4], z);
    size_t need = 0;
    check(p_tuna_moe_balance_workspace_bytes(t, clip(e), clip(segments), &need), "tuna_moe_balance_workspace_bytes");
    Tensor ws;
    if (need) ws = make({(int64_t)need}, at::kByte, z);
    const Tensor loss = make({segments}, at::kFloat, z), squares = make({segments}, at::kFloat, z), counts = make({segments, e}, at::kLong, z),
                 mass = make({segments, e}, at::kFloat, z), live = make({segments}, at::kLong, z);
    check(p_tuna_moe_balance(at_of(z), dtype_of(z), t, clip(e), ld, (const int32_t *)at_of(ids), clip(k), small(a[2]), clip(segments), offsets,
                             (float *)at_of(loss), (float *)at_of(squares), (int64_t *)at_of(counts), (float *)at_of(mass), (int64_t *)at_of(live),
                             need ? at_of(ws) : nullptr, need, place.stream()),
          "tuna_moe_balance");
    return pack(place.out(loss), place.out(squares), place.out(counts), place.out(mass), place.out(live));
  });
}

// balance_backward(logits, counts, tokens, k, dloss, dz, scoring, offsets, stream)
PyObject *balance_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const Tensor &z = tensor(a[0], "logits"), &counts = tensor(a[1], "counts"), &live = tensor(a[2], "tokens"), &dloss = tensor(a[4], "dloss");
    const int64_t ld = matrix(z, "logits", true, true, false), t = z.size(0), e = z.size(1), k = integer(a[3]);
    int64_t segments;
    const int64_t *offsets = segments_of(a[7], z, segments);
    dense(counts, "counts", at::kLong, {segments, e}, z);
    dense(live, "tokens", at::kLong, {segments}, z);
    dense(dloss, "dloss", at::kFloat, {segments}, z);
    const float *dz = nullptr;
    if (a[5] != Py_None) {
      const Tensor &o = tensor(a[5], "dz");
      dense(o, "dz", at::kFloat, {segments}, z);
      dz = (const float *)at_of(o);
    }
    const Place place(a[8], z);
    const Tensor d = make({t, e}, z.scalar_type(), z);
    check(p_tuna_moe_balance_backward(at_of(z), dtype_of(z), t, clip(e), ld, clip(k), small(a[6]), clip(segments), offsets, (const int64_t *)at_of(counts),
                                      (const int64_t *)at_of(live), (const float *)at_of(dloss), dz, at_of(d), std::max<int64_t>(e, 1), place.stream()),
          "tuna_moe_balance_backward");
    return THPVariable_Wrap(place.out(d));
  });
}

// A torch without the types of 4-bit operands (before 2.8) has the other operators all the same.
#ifndef TUNA_TORCH_FP4
#define TUNA_TORCH_FP4 (TORCH_VERSION_MAJOR > 2 || (TORCH_VERSION_MAJOR == 2 && TORCH_VERSION_MINOR >= 8))
#endif
#if TUNA_TORCH_FP4
constexpr at::ScalarType kFp4 = at::ScalarType::Float4_e2m1fn_x2, kPower = at::ScalarType::Float8_e8m0fnu;
#else
constexpr at::ScalarType kFp4 = at::ScalarType::Undefined, kPower = at::ScalarType::Undefined;
#endif

// The groups' bounds: int64 [groups + 1], or None (0 groups).
const int64_t *groups_of(PyObject *o, const Tensor &with, int64_t &groups) {
  groups = 0;
  if (o == Py_None) return nullptr;
  const Tensor &t = tensor(o, "offsets");
  if (t.dim() != 1 || t.size(0) < 2) refuse("offsets: [groups + 1] is wanted");
  groups = t.size(0) - 1;
  dense(t, "offsets", at::kLong, {groups + 1}, with);
  return (const int64_t *)at_of(t);
}
int64_t scale_tiles(int64_t rows, int64_t groups) { return groups ? rows / 128 + groups : (rows + 127) / 128; }

// A matrix of 4-bit values, two a byte; its pitch in bytes.
int64_t matrix4(const Tensor &t, const char *name) {
  if (t.dim() != 2 || t.scalar_type() != kFp4) refuse("%s: a CUDA matrix of float4_e2m1fn_x2 is wanted", name);
  const int64_t rows = t.size(0), cols = t.size(1);
  if ((cols > 1 && t.stride(1) != 1) || (rows > 1 && t.stride(0) < cols))
    refuse("%s: rows must be contiguous and must not overlap (strides %lld, %lld)", name, (long long)t.stride(0), (long long)t.stride(1));
  return rows > 1 ? t.stride(0) : std::max<int64_t>(cols, 1);
}
// The same for a product: rows on 16-byte boundaries, the tensor itself or a copy.
Tensor operand4(const Tensor &q, const char *name, int64_t &ld, void *stream) {
  ld = matrix4(q, name);
  if (q.size(0) <= 1) ld = (q.size(1) + 15) / 16 * 16;  // the pitch of a single row is free
  if (ld % 16 == 0 && (uintptr_t)q.data_ptr() % 16 == 0) {
    ld = std::max<int64_t>(ld, 16);
    return q;
  }
  const int64_t pitch = ld;
  ld = std::max<int64_t>((q.size(1) + 15) / 16 * 16, 16);
  Tensor p = make({q.size(0), ld}, at::kByte, q);  // (what stands behind the rows is not read)
  check(p_tuna_fp4_align(at_of(q), pitch, q.size(0), q.size(1), at_of(p), ld, stream), "tuna_fp4_align");
  return p;
}

// fp4_quantize(x, layout, offsets, stream)
PyObject *fp4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    if (kFp4 == at::ScalarType::Undefined) refuse("this torch has no float4_e2m1fn_x2");
    const Tensor &x = tensor(a[0], "x");
    const int64_t ld = matrix(x, "x", true, true, false), rows = x.size(0), cols = x.size(1);
    const int layout = small(a[1]);
    const bool turned = layout == TUNA_FP4_COLUMNS;
    if (turned && a[2] != Py_None) refuse("offsets go with the layout rows");
    int64_t groups;
    const int64_t *offsets = groups_of(a[2], x, groups);
    const int64_t out_rows = turned ? cols : rows, out_cols = turned ? rows : cols, bytes = (out_cols + 1) / 2, pitch = (bytes + 15) / 16 * 16;
    const Place place(a[3], x);
    const Tensor q = make({out_rows, pitch}, kFp4, x), scale = make({scale_tiles(out_rows, groups), (out_cols + 127) / 128, 32, 4, 4}, kPower, x);
    check(p_tuna_fp4_quantize(at_of(x), dtype_of(x), rows, clip(cols), ld, layout, clip(groups), offsets, at_of(q), pitch, at_of(scale),
                              place.stream()),
          "tuna_fp4_quantize");
    place.out(q), place.out(scale);
    return pack(pitch == bytes ? q : q.narrow(1, 0, bytes), scale);
  });
}

// fp4_dequantize(q, scale, offsets, out_dtype, stream)
PyObject *fp4_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const Tensor &q = tensor(a[0], "q"), &scale = tensor(a[1], "scale");
    const int64_t ld = matrix4(q, "q"), rows = q.size(0), cols = 2 * q.size(1);
    int64_t groups;
    const int64_t *offsets = groups_of(a[2], q, groups);
    dense(scale, "scale", kPower, {scale_tiles(rows, groups), (cols + 127) / 128, 32, 4, 4}, q);
    const int out = small(a[3]);
    const Place place(a[4], q);
    const Tensor y = make({rows, cols}, out == TUNA_DTYPE_F32 ? at::kFloat : at::kBFloat16, q);
    check(p_tuna_fp4_dequantize(at_of(q), ld, at_of(scale), rows, clip(cols), clip(groups), offsets, at_of(y), out, std::max<int64_t>(cols, 1),
                                place.stream()),
          "tuna_fp4_dequantize");
    return THPVariable_Wrap(place.out(y));
  });
}

// fp4_matmul(a, a_scale, b, b_scale, offsets, out_dtype, stream)
PyObject *fp4_matmul(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const Tensor &left = tensor(a[0], "a"), &sa = tensor(a[1], "a_scale"), &right = tensor(a[2], "b"), &sb = tensor(a[3], "b_scale");
    if (right.device() != left.device()) refuse("b: on another device than its fellow");
    int64_t groups;
    const int64_t *offsets = groups_of(a[4], left, groups);
    const int out = small(a[5]);
    const Place place(a[6], left);
    int64_t lda = 0, ldb = 0, cols, kb;
    const Tensor x = operand4(left, "a", lda, place.stream());
    const int64_t m = left.size(0), k = 2 * left.size(1), runs = (k + 127) / 128;
    Tensor w;
    if (offsets) {
      if (right.dim() != 3 || !right.is_contiguous() || right.size(0) != groups) refuse("b: contiguous matrices [%lld, n, k / 2] go with these offsets", (long long)groups);
      cols = right.size(1), kb = 2 * right.size(2);
      w = operand4(right.view({groups * cols, right.size(2)}), "b", ldb, place.stream());
      dense(sb, "b_scale", kPower, {groups, (cols + 127) / 128, runs, 32, 4, 4}, left);
    } else {
      w = operand4(right, "b", ldb, place.stream());
      cols = right.size(0), kb = 2 * right.size(1);
      dense(sb, "b_scale", kPower, {(cols + 127) / 128, runs, 32, 4, 4}, left);
    }
    if (kb != k) refuse("a has %lld columns, b %lld", (long long)k, (long long)kb);
    dense(sa, "a_scale", kPower, {scale_tiles(m, groups), runs, 32, 4, 4}, left);
    const Tensor y = make({m, cols}, out == TUNA_DTYPE_F32 ? at::kFloat : at::kBFloat16, left);
    check(p_tuna_fp4_matmul(at_of(x), at_of(sa), m, lda, at_of(w), at_of(sb), clip(cols), ldb, clip(k), clip(groups), offsets, at_of(y), out,
                            std::max<int64_t>(cols, 1), place.stream()),
          "tuna_fp4_matmul");
    return THPVariable_Wrap(place.out(y));
  });
}

// Checked 4-bit expert weights; (experts, inter) of them.
std::pair<int64_t, int64_t> weights4(PyObject *const *w, int64_t hidden, const Tensor &with) {
  const Tensor &w13 = tensor(w[0], "w13"), &s13 = tensor(w[1], "s13"), &w2 = tensor(w[2], "w2"), &s2 = tensor(w[3], "s2");
  if (w13.dim() != 4) refuse("w13: [experts, 2, inter, hidden / 2] is wanted");
  if (hidden % 2) refuse("x: an even number of columns is wanted");
  const int64_t e = w13.size(0), i = w13.size(2), bi = (i + 127) / 128, bd = (hidden + 127) / 128;
  dense(w13, "w13", kFp4, {e, 2, i, hidden / 2}, with);
  dense(s13, "s13", kPower, {e, 2, bi, bd, 32, 4, 4}, with);
  dense(w2, "w2", kFp4, {e, hidden, i / 2}, with);
  dense(s2, "s2", kPower, {e, bd, bi, 32, 4, 4}, with);
  return {e, i};
}
// A workspace: the caller's, or one of the call's own.
Tensor space(PyObject *given, size_t need, const Tensor &with) {
  if (given == Py_None) return make({(int64_t)std::max<size_t>(need, 256)}, at::kByte, with);
  const Tensor &t = tensor(given, "workspace");
  if (!t.is_contiguous()) refuse("workspace: a contiguous tensor is wanted");
  if (t.device() != with.device()) refuse("workspace: on another device than its fellow");
  return t;
}

// fp4_expert_rows(x, offsets, w13, s13, w2, s2, workspace, stream)
PyObject *fp4_expert_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const Tensor &x = tensor(a[0], "x"), &offsets = tensor(a[1], "offsets");
    const int64_t ld = matrix(x, "x", false, true, false), rows = x.size(0), d = x.size(1);
    const auto [e, i] = weights4(a + 2, d, x);
    dense(offsets, "offsets", at::kLong, {e + 1}, x);
    size_t need = 0;
    const Place place(a[7], x);
    check(p_tuna_fp4_expert_rows_workspace_bytes(rows, clip(e), clip(d), clip(i), &need), "tuna_fp4_expert_rows_workspace_bytes");
    const Tensor ws = space(a[6], need, x), y = make({rows, d}, at::kBFloat16, x);
    check(p_tuna_fp4_expert_rows(at_of(x), ld, rows, clip(e), (const int64_t *)at_of(offsets), clip(d), clip(i), at_of(tensor(a[2], "w13")),
                                 at_of(tensor(a[3], "s13")), at_of(tensor(a[4], "w2")), at_of(tensor(a[5], "s2")), at_of(y), std::max<int64_t>(d, 1),
                                 at_of(ws), ws.nbytes(), place.stream()),
          "tuna_fp4_expert_rows");
    return THPVariable_Wrap(place.out(y));
  });
}

// fp4_experts(x, ids, weights, w13, s13, w2, s2, workspace, stream)
PyObject *fp4_experts(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const Tensor &x = tensor(a[0], "x"), &ids = tensor(a[1], "ids"), &weights = tensor(a[2], "weights");
    const int64_t ld = matrix(x, "x", false, true, false), t = x.size(0), d = x.size(1);
    if (ids.dim() != 2) refuse("ids: [tokens, k] is wanted");
    const int64_t k = ids.size(1);
    dense(ids, "ids", at::kInt, {t, k}, x);
    dense(weights, "weights", at::kFloat, {t, k}, x);
    const auto [e, i] = weights4(a + 3, d, x);
    size_t need = 0;
    const Place place(a[8], x);
    check(p_tuna_fp4_experts_workspace_bytes(t, clip(e), clip(k), clip(d), clip(i), &need), "tuna_fp4_experts_workspace_bytes");
    const Tensor ws = space(a[7], need, x), out = make({t, d}, at::kBFloat16, x);
    check(p_tuna_fp4_experts(at_of(x), ld, t, (const int32_t *)at_of(ids), (const float *)at_of(weights), clip(k), clip(e), clip(d), clip(i),
                             at_of(tensor(a[3], "w13")), at_of(tensor(a[4], "s13")), at_of(tensor(a[5], "w2")), at_of(tensor(a[6], "s2")), at_of(out),
                             std::max<int64_t>(d, 1), at_of(ws), ws.nbytes(), place.stream()),
          "tuna_fp4_experts");
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
PyMethodDef methods[] = {F(route), F(route_backward), F(fp8_quantize), F(fp8_matmul), F(few), F(balance), F(balance_backward), F(fp4_quantize),
                         F(fp4_dequantize), F(fp4_matmul), F(fp4_expert_rows), F(fp4_experts), F(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tuna_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyObject *PyInit_tuna_torch() { return PyModule_Create(&module); }
