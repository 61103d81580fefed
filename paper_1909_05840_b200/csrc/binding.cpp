// _qbert: the Python entry to libqbert's C ABI for the calls that a model makes on every pass.
//
// A quantized linear at a few dozen tokens keeps the GPU busy for about ten microseconds; through ctypes,
// torch.empty and torch.cuda.current_stream the same two calls took the host more than thirty (an output
// allocated from Python 2.5 us each, the stream 3.2 us, seventeen converted arguments 1.5 us).  Here the
// tensors are read, the outputs allocated and the stream looked up in C++, so that a call costs the host
// little more than its launches.  Marshalling only: no arithmetic, no state, no fallback.  The interpreter's lock is
// released while outputs are allocated and the library runs: both can block (a full launch queue, an allocation that has to
// free first), and other threads go on meanwhile.
//
// Every function takes its arguments by position (the wrappers in __init__.py give them names and
// defaults) and raises what the wrapper's own checks would: AssertionError for a tensor of the wrong kind,
// QbertError (through the function set by set_raise) for a status.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <utility>
#include <vector>

#include "qbert.h"

namespace {

PyObject* g_raise = nullptr;  // __init__._raise(status, what)

struct Failed {};  // a Python error is set

[[noreturn]] void fail(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Failed{};
}
void need(bool ok, const char* text) {
  if (!ok) fail(PyExc_AssertionError, text);
}
void check(qb_status st, const char* what) {
  if (st == QB_OK) return;
  PyObject* r = PyObject_CallFunction(g_raise, "is", (int)st, what);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, what);
  throw Failed{};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a torch.Tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor& input(PyObject* o, at::ScalarType type, const char* what) {
  const at::Tensor& t = tensor(o);
  need(t.is_cuda() && t.scalar_type() == type && t.is_contiguous(), what);
  return t;
}
void* ptr(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Failed{};
  return v;
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Other Python threads run while one of these lives; no Python object may be touched.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// An output: the caller's tensor, or a new one that `make` allocates (a caller's tensor stays).  `get` hands over a new
// reference.
struct Out {
  PyObject* obj = nullptr;
  void* data = nullptr;
  at::Tensor made;
  explicit Out(PyObject* given) {
    if (given == Py_None) return;
    data = tensor(given).data_ptr();
    obj = Py_NewRef(given);
  }
  Out(const Out&) = delete;
  ~Out() { Py_XDECREF(obj); }
  void make(at::IntArrayRef shape, at::ScalarType type, at::Device device) {
    if (obj) return;
    made = at::Tensor(at::detail::empty_cuda(shape, type, device, std::nullopt));
    data = made.data_ptr();
  }
  // The same as a part of `base` (contiguous bytes), which lives as long as one of its parts: an allocation costs the host
  // 0.9 us, a part of one 0.1.
  void make_in(const at::Tensor& base, int64_t offset, at::IntArrayRef shape, at::ScalarType type) {
    if (obj) return;
    made = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                    c10::scalarTypeToTypeMeta(type));
    c10::TensorImpl* const impl = made.unsafeGetTensorImpl();
    impl->set_storage_offset(offset / (int64_t)c10::elementSize(type));
    impl->set_sizes_contiguous(shape);
    data = made.data_ptr();
  }
  void wrap() {
    if (!obj) obj = THPVariable_Wrap(std::move(made));
    if (!obj) throw Failed{};
  }
  PyObject* get() {
    wrap();
    return std::exchange(obj, nullptr);
  }
};
PyObject* triple(Out& a, Out& b, Out& c) {
  a.wrap();
  b.wrap();
  c.wrap();
  PyObject* r = PyTuple_New(3);
  if (!r) throw Failed{};
  PyTuple_SET_ITEM(r, 0, a.get());
  PyTuple_SET_ITEM(r, 1, b.get());
  PyTuple_SET_ITEM(r, 2, c.get());
  return r;
}

struct Workspace {
  void* data;
  size_t bytes;
  explicit Workspace(PyObject* o) {
    const at::Tensor& t = tensor(o);
    data = t.data_ptr();
    bytes = (size_t)t.numel();
  }
};

// A ctypes array of descriptors.
struct Descs {
  Py_buffer b;
  explicit Descs(PyObject* o) {
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Failed{};
  }
  Descs(const Descs&) = delete;
  ~Descs() { PyBuffer_Release(&b); }
  template <class T>
  const T* as(int32_t* count) const {
    *count = (int32_t)(b.len / (Py_ssize_t)sizeof(T));
    return static_cast<const T*>(b.buf);
  }
};

typedef PyObject* const* Args;

// quantize_act(x, ws, xq, act_scale, rowsum) -> (xq, act_scale, rowsum)
PyObject* quantize_act(Args a) {
  const at::Tensor& x = input(a[0], at::kFloat, "x: a contiguous fp32 CUDA tensor of two dimensions");
  need(x.dim() == 2, "x: a contiguous fp32 CUDA tensor of two dimensions");
  const int64_t M = x.size(0), K = x.size(1);
  const at::Device device = x.device();
  const float* const x_data = x.const_data_ptr<float>();
  const Workspace ws(a[1]);
  Out xq(a[2]), scale(a[3]), rowsum(a[4]);
  qb_status st;
  {
    const Unlocked unlocked;
    xq.make({M, K}, at::kChar, device);
    scale.make({1}, at::kFloat, device);
    rowsum.make({M}, at::kInt, device);
    st = qb_quantize_act(x_data, M, K, static_cast<int8_t*>(xq.data), static_cast<float*>(scale.data),
                         static_cast<int32_t*>(rowsum.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_quantize_act");
  return triple(xq, scale, rowsum);
}

// gemm(kind, xq, act_scale, rowsum, packed, delta, q0, bias, N, bits, groups, ws, y, acc_out | out_scale)
// kind 0: fp32 (last argument: int32 accumulators or None), 1: bfloat16 (None), 2: int8 (the output scale)
PyObject* gemm(Args a) {
  const int64_t kind = integer(a[0]);
  const at::Tensor& xq = input(a[1], at::kChar, "xq: a contiguous int8 CUDA tensor");
  need(xq.dim() == 2, "xq: two dimensions");
  const int64_t M = xq.size(0), K = xq.size(1), N = integer(a[8]);
  const at::Device device = xq.device();
  const int bits = (int)integer(a[9]), groups = (int)integer(a[10]);
  const Workspace ws(a[11]);
  if (kind == 1 && a[12] != Py_None)
    need(tensor(a[12]).scalar_type() == at::kBFloat16 && tensor(a[12]).is_contiguous(), "y: a contiguous bfloat16 tensor");
  if (kind == 2) need(tensor(a[13]).is_cuda() && tensor(a[13]).scalar_type() == at::kFloat, "out_scale: an fp32 CUDA tensor");
  Out y(a[12]);
  const int8_t* x = xq.const_data_ptr<int8_t>();
  const float* scale = static_cast<const float*>(ptr(a[2]));
  const int32_t* rowsum = static_cast<const int32_t*>(ptr(a[3]));
  const uint32_t* packed = static_cast<const uint32_t*>(ptr(a[4]));
  const float* delta = static_cast<const float*>(ptr(a[5]));
  const float* q0 = static_cast<const float*>(ptr(a[6]));
  const float* bias = static_cast<const float*>(ptr(a[7]));
  void* const last = ptr(a[13]);
  qb_status st;
  {
    const Unlocked unlocked;
    y.make({M, N}, kind == 0 ? at::kFloat : (kind == 1 ? at::kBFloat16 : at::kChar), device);
    if (kind == 0)
      st = qb_gemm(x, scale, rowsum, packed, delta, q0, bias, M, N, K, bits, groups, static_cast<float*>(y.data),
                   static_cast<int32_t*>(last), ws.data, ws.bytes, stream());
    else if (kind == 1)
      st = qb_gemm_bf16(x, scale, rowsum, packed, delta, q0, bias, M, N, K, bits, groups, static_cast<uint16_t*>(y.data),
                        ws.data, ws.bytes, stream());
    else
      st = qb_gemm_i8(x, scale, rowsum, packed, delta, q0, bias, M, N, K, bits, groups, static_cast<const float*>(last),
                      static_cast<int8_t*>(y.data), ws.data, ws.bytes, stream());
  }
  check(st, kind == 0 ? "qb_gemm" : (kind == 1 ? "qb_gemm_bf16" : "qb_gemm_i8"));
  return y.get();
}

// rowsum_i8(xq, rowsum) -> rowsum
PyObject* rowsum_i8(Args a) {
  const at::Tensor& xq = input(a[0], at::kChar, "xq: a contiguous int8 CUDA tensor of two dimensions");
  need(xq.dim() == 2, "xq: a contiguous int8 CUDA tensor of two dimensions");
  const int64_t M = xq.size(0), K = xq.size(1);
  const at::Device device = xq.device();
  const int8_t* const x = xq.const_data_ptr<int8_t>();
  Out rowsum(a[1]);
  qb_status st;
  {
    const Unlocked unlocked;
    rowsum.make({M}, at::kInt, device);
    st = qb_rowsum_i8(x, M, K, static_cast<int32_t*>(rowsum.data), stream());
  }
  check(st, "qb_rowsum_i8");
  return rowsum.get();
}

// quantize_pack_weights(w, bits, groups, ws, range_lo, range_hi, packed, delta, q0) -> (packed, delta, q0)
PyObject* quantize_pack_weights(Args a) {
  const at::Tensor& w = input(a[0], at::kFloat, "w: a contiguous fp32 CUDA tensor of two dimensions");
  need(w.dim() == 2, "w: a contiguous fp32 CUDA tensor of two dimensions");
  const int64_t N = w.size(0), K = w.size(1), bits = integer(a[1]), groups = integer(a[2]);
  const at::Device device = w.device();
  const float* const w_data = w.const_data_ptr<float>();
  const Workspace ws(a[3]);
  const float* const lo = static_cast<const float*>(ptr(a[4]));
  const float* const hi = static_cast<const float*>(ptr(a[5]));
  Out packed(a[6]), delta(a[7]), q0(a[8]);
  qb_status st;
  {
    const Unlocked unlocked;
    packed.make({N, std::max<int64_t>(1, K * bits / 32)}, at::kInt, device);
    delta.make({std::max<int64_t>(groups, 1)}, at::kFloat, device);
    q0.make({std::max<int64_t>(groups, 1)}, at::kFloat, device);
    st = qb_quantize_pack_weights(w_data, N, K, (int)bits, (int)groups, lo, hi, static_cast<uint32_t*>(packed.data),
                                  static_cast<float*>(delta.data), static_cast<float*>(q0.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_quantize_pack_weights");
  return triple(packed, delta, q0);
}

// fake_quantize_weights(w, bits, groups, ws, range_lo, range_hi, wq) -> (wq, delta, q0)
PyObject* fake_quantize_weights(Args a) {
  const at::Tensor& w = input(a[0], at::kFloat, "w: a contiguous fp32 CUDA tensor of two dimensions");
  need(w.dim() == 2, "w: a contiguous fp32 CUDA tensor of two dimensions");
  const int64_t N = w.size(0), K = w.size(1), bits = integer(a[1]), groups = integer(a[2]);
  const at::Device device = w.device();
  const float* const w_data = w.const_data_ptr<float>();
  const Workspace ws(a[3]);
  const float* const lo = static_cast<const float*>(ptr(a[4]));
  const float* const hi = static_cast<const float*>(ptr(a[5]));
  Out wq(a[6]), delta(Py_None), q0(Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    wq.make({N, K}, at::kFloat, device);
    delta.make({std::max<int64_t>(groups, 0)}, at::kFloat, device);
    q0.make({std::max<int64_t>(groups, 0)}, at::kFloat, device);
    st = qb_fake_quantize_weights(w_data, N, K, (int)bits, (int)groups, lo, hi, static_cast<float*>(wq.data),
                                  static_cast<float*>(delta.data), static_cast<float*>(q0.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_fake_quantize_weights");
  return triple(wq, delta, q0);
}

// ste_backward(grad_wq, w, groups, range_lo, range_hi, grad_w) -> grad_w
PyObject* ste_backward(Args a) {
  const at::Tensor& g = input(a[0], at::kFloat, "grad_wq: a contiguous fp32 CUDA tensor of the shape of w");
  const at::Tensor& w = tensor(a[1]);
  need(g.dim() == 2 && g.sizes() == w.sizes(), "grad_wq: a contiguous fp32 CUDA tensor of the shape of w");
  const int64_t N = w.size(0), K = w.size(1), groups = integer(a[2]);
  const at::Device device = w.device();
  const float* const g_data = g.const_data_ptr<float>();
  const float* const w_data = static_cast<const float*>(w.const_data_ptr());
  const float* const lo = static_cast<const float*>(ptr(a[3]));
  const float* const hi = static_cast<const float*>(ptr(a[4]));
  Out grad_w(a[5]);
  qb_status st;
  {
    const Unlocked unlocked;
    grad_w.make({N, K}, at::kFloat, device);
    st = qb_ste_backward(g_data, w_data, N, K, (int)groups, lo, hi, static_cast<float*>(grad_w.data), stream());
  }
  check(st, "qb_ste_backward");
  return grad_w.get();
}

// quantize_embedding(table, bits, groups, ws, packed) -> (packed, delta, q0)
PyObject* quantize_embedding(Args a) {
  const at::Tensor& t = input(a[0], at::kFloat, "table: a contiguous fp32 CUDA tensor of two dimensions");
  need(t.dim() == 2, "table: a contiguous fp32 CUDA tensor of two dimensions");
  const int64_t V = t.size(0), D = t.size(1), bits = integer(a[1]), groups = integer(a[2]);
  const at::Device device = t.device();
  const float* const table = t.const_data_ptr<float>();
  const Workspace ws(a[3]);
  Out packed(a[4]), delta(Py_None), q0(Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    packed.make({V, D * bits / 32}, at::kInt, device);
    delta.make({std::max<int64_t>(groups, 0)}, at::kFloat, device);
    q0.make({std::max<int64_t>(groups, 0)}, at::kFloat, device);
    st = qb_quantize_embedding(table, V, D, (int)bits, (int)groups, static_cast<uint32_t*>(packed.data),
                               static_cast<float*>(delta.data), static_cast<float*>(q0.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_quantize_embedding");
  return triple(packed, delta, q0);
}

// embedding_lookup(ids, packed, delta, q0, D, bits, groups, ws, out, accumulate) -> out
PyObject* embedding_lookup(Args a) {
  const at::Tensor& ids = input(a[0], at::kInt, "ids: a contiguous int32 CUDA tensor");
  const at::Tensor& packed = tensor(a[1]);
  const int64_t T = ids.numel(), V = packed.size(0), D = integer(a[4]), bits = integer(a[5]), groups = integer(a[6]);
  const at::Device device = ids.device();
  const int32_t* const id_data = ids.const_data_ptr<int32_t>();
  const uint32_t* const codes = static_cast<const uint32_t*>(packed.const_data_ptr());
  const float* const delta = static_cast<const float*>(ptr(a[2]));
  const float* const q0 = static_cast<const float*>(ptr(a[3]));
  const Workspace ws(a[7]);
  const int accumulate = PyObject_IsTrue(a[9]);
  if (accumulate < 0) throw Failed{};
  if (a[8] == Py_None) need(!accumulate, "accumulate needs `out`");
  Out out(a[8]);
  qb_status st;
  {
    const Unlocked unlocked;
    out.make({T, D}, at::kFloat, device);
    st = qb_embedding_lookup(id_data, T, codes, delta, q0, V, D, (int)bits, (int)groups, accumulate ? 1 : 0,
                             static_cast<float*>(out.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_embedding_lookup");
  return out.get();
}

// ---- 8-bit floating point, dropout -----------------------------------------------------------------------------------
// These calls take tensors of the current device alone: its current stream is what they are enqueued on.
const at::Tensor& here(PyObject* o, const char* what) {
  const at::Tensor& t = tensor(o);
  need(t.is_cuda() && t.is_contiguous() && t.device().index() == c10::cuda::current_device(), what);
  return t;
}
// A caller's output has to have the type and the size of what is written.
void fits(PyObject* o, at::ScalarType type, int64_t count, const char* what) {
  if (o == Py_None) return;
  const at::Tensor& t = here(o, what);
  need(t.scalar_type() == type && t.numel() == count, what);
}
// A matrix has to have its shape too: the elements of [N][M] are as many as those of [M][N].
void fits(PyObject* o, at::ScalarType type, int64_t rows, int64_t cols, const char* what) {
  if (o == Py_None) return;
  const at::Tensor& t = here(o, what);
  need(t.scalar_type() == type && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols, what);
}
int element_type(const at::Tensor& t, const char* what) {
  switch (t.scalar_type()) {
    case at::kFloat: return QB_F32;
    case at::kBFloat16: return QB_BF16;
    case at::kHalf: return QB_F16;
    default: fail(PyExc_AssertionError, what);
  }
}
int fp8_format(const at::Tensor& t, const char* what) {
  switch (t.scalar_type()) {
    case at::kFloat8_e4m3fn: return QB_E4M3;
    case at::kFloat8_e5m2: return QB_E5M2;
    default: fail(PyExc_AssertionError, what);
  }
}
Workspace workspace_here(PyObject* o) {
  const at::Tensor& t = here(o, "ws: a contiguous CUDA tensor of bytes on the current device");
  need(t.scalar_type() == at::kByte, "ws: a contiguous CUDA tensor of bytes on the current device");
  return Workspace(o);
}

// dropout(x, p, rng, call, residual, out) -> out
PyObject* dropout(Args a) {
  const char* const what = "x: a contiguous fp32, bfloat16 or fp16 CUDA tensor on the current device";
  const at::Tensor& x = here(a[0], what);
  const int type = element_type(x, what);
  const double p = PyFloat_AsDouble(a[1]);
  if (p == -1.0 && PyErr_Occurred()) throw Failed{};
  const at::Tensor& rng = here(a[2], "rng: int64 [2] on the current device (seed, offset)");
  need(rng.scalar_type() == at::kLong && rng.numel() == 2, "rng: int64 [2] on the current device (seed, offset)");
  const uint64_t call = PyLong_AsUnsignedLongLong(a[3]);
  if (call == (uint64_t)-1 && PyErr_Occurred()) throw Failed{};
  const int64_t n = x.numel();
  fits(a[4], x.scalar_type(), n, "residual: contiguous, of the type and size of x");
  fits(a[5], x.scalar_type(), n, "out: contiguous, of the type and size of x");
  const at::Device device = x.device();
  const std::vector<int64_t> shape = x.sizes().vec();
  const at::ScalarType scalar = x.scalar_type();
  const void* const x_data = x.const_data_ptr();
  const uint64_t* const rng_data = static_cast<const uint64_t*>(rng.const_data_ptr());
  const void* const residual = ptr(a[4]);
  Out out(a[5]);
  qb_status st;
  {
    const Unlocked unlocked;
    out.make(shape, scalar, device);
    st = qb_dropout(x_data, type, n, p, rng_data, call, residual, out.data, stream());
  }
  check(st, "qb_dropout");
  return out.get();
}

// Codes [rows][cols] and their scales, in one allocation where both are new.
void codes_and_scales(Out& q, Out& s, int64_t rows, int64_t cols, at::ScalarType code, at::Device device) {
  const int64_t shape[5] = {(rows + 127) / 128, (cols + 511) / 512, 32, 4, 4};
  if (q.obj || s.obj) {
    q.make({rows, cols}, code, device);
    s.make(shape, at::kByte, device);
    return;
  }
  const int64_t bytes = (rows * cols + 511) / 512 * 512;
  const at::Tensor both(at::detail::empty_cuda({bytes + shape[0] * shape[1] * 512}, at::kByte, device, std::nullopt));
  q.make_in(both, 0, {rows, cols}, code);
  s.make_in(both, bytes, shape, at::kByte);
}

// quantize_fp8(x, ws, format, transposed, weights, codes, scales, codes_t, scales_t, want_sums, sums)
//   -> (codes, scales[, codes_t, scales_t][, sums])
PyObject* quantize_fp8(Args a) {
  const char* const what = "x: a contiguous fp32, bfloat16 or fp16 CUDA tensor of two dimensions on the current device";
  const at::Tensor& x = here(a[0], what);
  need(x.dim() == 2, what);
  const int type = element_type(x, what), format = (int)integer(a[2]);
  const Workspace ws = workspace_here(a[1]);
  const bool transposed = integer(a[3]) != 0, weights = integer(a[4]) != 0;
  const int64_t M = x.size(0), K = x.size(1), Kp = (K + 127) / 128 * 128, Mp = (M + 127) / 128 * 128;
  const at::ScalarType code = format == QB_E4M3 ? at::kFloat8_e4m3fn : at::kFloat8_e5m2;
  fits(a[5], code, M, Kp, "codes: contiguous, of the asked format, [M][K up to 128]");
  fits(a[6], at::kByte, (int64_t)qb_fp8_scale_bytes(M, K), "scales: contiguous bytes, fp8_scale_bytes(M, K) of them");
  if (transposed) {
    fits(a[7], code, K, Mp, "codes_t: contiguous, of the asked format, [K][M up to 128]");
    fits(a[8], at::kByte, (int64_t)qb_fp8_scale_bytes(K, M), "scales_t: contiguous bytes, fp8_scale_bytes(K, M) of them");
  }
  const bool want_sums = transposed && !weights && integer(a[9]) != 0;
  if (want_sums) fits(a[10], at::kFloat, K, "sums: contiguous fp32 [K] on the current device");
  const at::Device device = x.device();
  const void* const x_data = x.const_data_ptr();
  Out q(a[5]), s(a[6]), qt(transposed ? a[7] : Py_None), s_t(transposed ? a[8] : Py_None), sums(want_sums ? a[10] : Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    codes_and_scales(q, s, M, Kp, code, device);
    if (transposed) codes_and_scales(qt, s_t, K, Mp, code, device);
    if (want_sums) sums.make({K}, at::kFloat, device);
    uint8_t *const qd = static_cast<uint8_t*>(q.data), *const sd = static_cast<uint8_t*>(s.data);
    uint8_t *const qtd = static_cast<uint8_t*>(qt.data), *const st_data = static_cast<uint8_t*>(s_t.data);
    if (weights) st = qb_quantize_fp8_weights(x_data, type, M, K, format, qd, sd, qtd, st_data, ws.data, ws.bytes, stream());
    else st = qb_quantize_fp8(x_data, type, M, K, format, qd, sd, qtd, st_data, static_cast<float*>(sums.data), ws.data, ws.bytes, stream());
  }
  check(st, weights ? "qb_quantize_fp8_weights" : "qb_quantize_fp8");
  Out* const outs[5] = {&q, &s, &qt, &s_t, &sums};
  const int count = transposed ? (want_sums ? 5 : 4) : 2;
  for (int i = 0; i < count; ++i) outs[i]->wrap();
  PyObject* r = PyTuple_New(count);
  if (!r) throw Failed{};
  for (int i = 0; i < count; ++i) PyTuple_SET_ITEM(r, i, outs[i]->get());
  return r;
}

// gemm_fp8(a, a_scale, b, b_scale, bias, ws, out_type, y) -> y
PyObject* gemm_fp8(Args g) {
  const char* const what_a = "a: contiguous e4m3 or e5m2 codes of two dimensions on the current device";
  const char* const what_b = "b: contiguous e4m3 or e5m2 codes of two dimensions on the current device, rows as long as a's";
  const at::Tensor& a = here(g[0], what_a);
  const at::Tensor& b = here(g[2], what_b);
  need(a.dim() == 2, what_a);
  need(b.dim() == 2 && b.size(1) == a.size(1), what_b);
  const int fa = fp8_format(a, what_a), fb = fp8_format(b, what_b), out_type = (int)integer(g[6]);
  const int64_t M = a.size(0), N = b.size(0), K = a.size(1);
  const auto scales = [](PyObject* o, int64_t rows, int64_t k, const char* what) {
    const at::Tensor& t = here(o, what);
    need(t.scalar_type() == at::kByte && t.numel() == (int64_t)qb_fp8_scale_bytes(rows, k), what);
    return static_cast<const uint8_t*>(t.const_data_ptr());
  };
  const uint8_t* const sa = scales(g[1], M, K, "a_scale: the bytes that came with a");
  const uint8_t* const sb = scales(g[3], N, K, "b_scale: the bytes that came with b");
  fits(g[4], at::kFloat, N, "bias: contiguous fp32 [N] on the current device");
  const Workspace ws = workspace_here(g[5]);
  const at::ScalarType type = out_type == QB_F32 ? at::kFloat : at::kBFloat16;
  fits(g[7], type, M, N, "y: contiguous [M][N] of the asked type on the current device");
  const at::Device device = a.device();
  const uint8_t* const a_data = static_cast<const uint8_t*>(a.const_data_ptr());
  const uint8_t* const b_data = static_cast<const uint8_t*>(b.const_data_ptr());
  const float* const bias = static_cast<const float*>(ptr(g[4]));
  Out y(g[7]);
  qb_status st;
  {
    const Unlocked unlocked;
    y.make({M, N}, type, device);
    st = qb_gemm_fp8(a_data, sa, fa, b_data, sb, fb, bias, M, N, K, out_type, y.data, ws.data, ws.bytes, stream());
  }
  check(st, "qb_gemm_fp8");
  return y.get();
}

// ---- vocabulary loss ---------------------------------------------------------------------------------------------------
struct VocabInputs {
  int64_t T, V, D;
  const uint16_t *h, *w;
  const float* bias;
  const int32_t* targets;
  at::Device device;
  static const at::Tensor& matrix(PyObject* o, const char* what) {
    const at::Tensor& t = here(o, what);
    need(t.dim() == 2 && t.scalar_type() == at::kBFloat16, what);
    return t;
  }
  VocabInputs(PyObject* ho, PyObject* wo, PyObject* bo, PyObject* to) : device(at::kCUDA) {
    const at::Tensor& ht = matrix(ho, "h: contiguous bfloat16 [T][D] on the current device");
    const at::Tensor& wt = matrix(wo, "w: contiguous bfloat16 [V][D] on the current device");
    T = ht.size(0);
    D = ht.size(1);
    V = wt.size(0);
    need(wt.size(1) == D, "w: contiguous bfloat16 [V][D] on the current device");
    fits(bo, at::kFloat, V, "bias: contiguous fp32 [V] on the current device");
    need(to != Py_None, "targets: contiguous int32 [T] on the current device");
    fits(to, at::kInt, T, "targets: contiguous int32 [T] on the current device");
    h = static_cast<const uint16_t*>(ht.const_data_ptr());
    w = static_cast<const uint16_t*>(wt.const_data_ptr());
    bias = static_cast<const float*>(ptr(bo));
    targets = static_cast<const int32_t*>(ptr(to));
    device = ht.device();
  }
};

// vocab_loss(h, w, bias, targets, ws, loss, lse) -> (loss, lse)
PyObject* vocab_loss(Args a) {
  const VocabInputs in(a[0], a[1], a[2], a[3]);
  const Workspace ws = workspace_here(a[4]);
  fits(a[5], at::kFloat, in.T, "loss: contiguous fp32 [T] on the current device");
  fits(a[6], at::kFloat, in.T, "lse: contiguous fp32 [T] on the current device");
  Out loss(a[5]), lse(a[6]);
  qb_status st;
  {
    const Unlocked unlocked;
    if (loss.obj || lse.obj) {
      loss.make({in.T}, at::kFloat, in.device);
      lse.make({in.T}, at::kFloat, in.device);
    } else {
      const int64_t bytes = (in.T * 4 + 511) / 512 * 512;
      const at::Tensor both(at::detail::empty_cuda({2 * bytes}, at::kByte, in.device, std::nullopt));
      loss.make_in(both, 0, {in.T}, at::kFloat);
      lse.make_in(both, bytes, {in.T}, at::kFloat);
    }
    st = qb_vocab_loss(in.h, in.w, in.bias, in.targets, in.T, in.V, in.D, static_cast<float*>(loss.data), static_cast<float*>(lse.data),
                       ws.data, ws.bytes, stream());
  }
  check(st, "qb_vocab_loss");
  loss.wrap();
  lse.wrap();
  PyObject* r = PyTuple_New(2);
  if (!r) throw Failed{};
  PyTuple_SET_ITEM(r, 0, loss.get());
  PyTuple_SET_ITEM(r, 1, lse.get());
  return r;
}

// vocab_loss_backward(h, w, bias, targets, lse, grad_loss, ws, grad_h, grad_w, grad_bias, need_h, need_w, need_bias) -> three gradients
PyObject* vocab_loss_backward(Args a) {
  const VocabInputs in(a[0], a[1], a[2], a[3]);
  need(a[4] != Py_None, "lse: contiguous fp32 [T] on the current device");
  fits(a[4], at::kFloat, in.T, "lse: contiguous fp32 [T] on the current device");
  need(a[5] != Py_None, "grad_loss: contiguous fp32 [T] on the current device");
  fits(a[5], at::kFloat, in.T, "grad_loss: contiguous fp32 [T] on the current device");
  const Workspace ws = workspace_here(a[6]);
  fits(a[7], at::kBFloat16, in.T, in.D, "grad_h: contiguous bfloat16 [T][D] on the current device");
  fits(a[8], at::kBFloat16, in.V, in.D, "grad_w: contiguous bfloat16 [V][D] on the current device");
  fits(a[9], at::kFloat, in.V, "grad_bias: contiguous fp32 [V] on the current device");
  const bool want[3] = {integer(a[10]) != 0, integer(a[11]) != 0, integer(a[12]) != 0 && (in.bias || a[9] != Py_None)};
  Out gh(want[0] ? a[7] : Py_None), gw(want[1] ? a[8] : Py_None), gb(want[2] ? a[9] : Py_None);
  const float* const lse = static_cast<const float*>(ptr(a[4]));
  const float* const grad_loss = static_cast<const float*>(ptr(a[5]));
  qb_status st;
  {
    const Unlocked unlocked;
    if (want[0]) gh.make({in.T, in.D}, at::kBFloat16, in.device);
    if (want[1]) gw.make({in.V, in.D}, at::kBFloat16, in.device);
    if (want[2]) gb.make({in.V}, at::kFloat, in.device);
    st = qb_vocab_loss_backward(in.h, in.w, in.bias, in.targets, lse, grad_loss, in.T, in.V, in.D, static_cast<uint16_t*>(gh.data),
                                static_cast<uint16_t*>(gw.data), static_cast<float*>(gb.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_vocab_loss_backward");
  Out* const outs[3] = {&gh, &gw, &gb};
  for (int i = 0; i < 3; ++i)
    if (want[i]) outs[i]->wrap();
  PyObject* r = PyTuple_New(3);
  if (!r) throw Failed{};
  for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(r, i, want[i] ? outs[i]->get() : Py_NewRef(Py_None));
  return r;
}

// ---- an encoder block's other operators -----------------------------------------------------------------------------------
PyObject* tuple_of(std::initializer_list<Out*> outs) {
  for (Out* o : outs) o->wrap();
  PyObject* r = PyTuple_New((Py_ssize_t)outs.size());
  if (!r) throw Failed{};
  Py_ssize_t i = 0;
  for (Out* o : outs) PyTuple_SET_ITEM(r, i++, o->get());
  return r;
}
const at::Tensor& matrix_here(PyObject* o, const char* what) {
  const at::Tensor& t = here(o, what);
  need(t.dim() == 2, what);
  return t;
}

// layer_norm(x, gamma, beta, eps, want_stats, y, mean, rstd) -> y or (y, mean, rstd)
PyObject* layer_norm(Args a) {
  const char* const what = "x: a contiguous fp32, bfloat16 or fp16 CUDA tensor of two dimensions on the current device";
  const at::Tensor& x = matrix_here(a[0], what);
  const int type = element_type(x, what);
  const int64_t M = x.size(0), D = x.size(1);
  fits(a[1], at::kFloat, D, "gamma: contiguous fp32 [D] on the current device");
  fits(a[2], at::kFloat, D, "beta: contiguous fp32 [D] on the current device");
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) throw Failed{};
  const bool stats = integer(a[4]) != 0;
  fits(a[5], x.scalar_type(), M, D, "y: contiguous, of the type and shape of x");
  fits(a[6], at::kFloat, M, "mean: contiguous fp32 [M] on the current device");
  fits(a[7], at::kFloat, M, "rstd: contiguous fp32 [M] on the current device");
  const at::Device device = x.device();
  const at::ScalarType scalar = x.scalar_type();
  const void* const x_data = x.const_data_ptr();
  const float *const gamma = static_cast<const float*>(ptr(a[1])), *const beta = static_cast<const float*>(ptr(a[2]));
  Out y(a[5]), mean(stats ? a[6] : Py_None), rstd(stats ? a[7] : Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    y.make({M, D}, scalar, device);
    if (stats) {
      if (mean.obj || rstd.obj) {
        mean.make({M}, at::kFloat, device);
        rstd.make({M}, at::kFloat, device);
      } else {
        const int64_t bytes = (M * 4 + 511) / 512 * 512;
        const at::Tensor both(at::detail::empty_cuda({2 * bytes}, at::kByte, device, std::nullopt));
        mean.make_in(both, 0, {M}, at::kFloat);
        rstd.make_in(both, bytes, {M}, at::kFloat);
      }
    }
    st = qb_layer_norm(x_data, type, gamma, beta, eps, M, D, y.data, static_cast<float*>(mean.data), static_cast<float*>(rstd.data), stream());
  }
  check(st, "qb_layer_norm");
  if (!stats) return y.get();
  return tuple_of({&y, &mean, &rstd});
}

// layer_norm_backward(grad_y, x, gamma, mean, rstd, ws, grad_x, grad_gamma, grad_beta, need_weights) -> (grad_x, grad_gamma, grad_beta)
PyObject* layer_norm_backward(Args a) {
  const char* const what = "grad_y: a contiguous fp32, bfloat16 or fp16 CUDA tensor of two dimensions on the current device";
  const at::Tensor& gy = matrix_here(a[0], what);
  const int type = element_type(gy, what);
  const int64_t M = gy.size(0), D = gy.size(1);
  need(a[1] != Py_None, "x: contiguous, of the type and shape of grad_y");
  fits(a[1], gy.scalar_type(), M, D, "x: contiguous, of the type and shape of grad_y");
  fits(a[2], at::kFloat, D, "gamma: contiguous fp32 [D] on the current device");
  need(a[3] != Py_None && a[4] != Py_None, "mean, rstd: contiguous fp32 [M] on the current device");
  fits(a[3], at::kFloat, M, "mean: contiguous fp32 [M] on the current device");
  fits(a[4], at::kFloat, M, "rstd: contiguous fp32 [M] on the current device");
  const bool weights = integer(a[9]) != 0;
  fits(a[6], gy.scalar_type(), M, D, "grad_x: contiguous, of the type and shape of grad_y");
  fits(a[7], at::kFloat, D, "grad_gamma: contiguous fp32 [D] on the current device");
  fits(a[8], at::kFloat, D, "grad_beta: contiguous fp32 [D] on the current device");
  const Workspace ws = workspace_here(a[5]);
  const at::Device device = gy.device();
  const at::ScalarType scalar = gy.scalar_type();
  const void *const gy_data = gy.const_data_ptr(), *const x_data = ptr(a[1]);
  const float *const gamma = static_cast<const float*>(ptr(a[2])), *const mean = static_cast<const float*>(ptr(a[3])), *const rstd = static_cast<const float*>(ptr(a[4]));
  Out gx(a[6]), gg(weights ? a[7] : Py_None), gb(weights ? a[8] : Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    gx.make({M, D}, scalar, device);
    if (weights) {
      if (gg.obj || gb.obj) {
        gg.make({D}, at::kFloat, device);
        gb.make({D}, at::kFloat, device);
      } else {
        const int64_t bytes = (D * 4 + 511) / 512 * 512;
        const at::Tensor both(at::detail::empty_cuda({2 * bytes}, at::kByte, device, std::nullopt));
        gg.make_in(both, 0, {D}, at::kFloat);
        gb.make_in(both, bytes, {D}, at::kFloat);
      }
    }
    st = qb_layer_norm_backward(gy_data, x_data, type, gamma, mean, rstd, M, D, gx.data, static_cast<float*>(gg.data), static_cast<float*>(gb.data), ws.data, ws.bytes,
                                stream());
  }
  check(st, "qb_layer_norm_backward");
  if (weights) return tuple_of({&gx, &gg, &gb});
  gx.wrap();
  return Py_BuildValue("(NOO)", gx.get(), Py_None, Py_None);
}

// Codes [M][K] and scales [M][blocks of K], both the caller's or both new.
const char* const kCodesWhat = "codes: contiguous int8 [M][K] on the current device";
const char* const kScalesWhat = "scales: contiguous fp32 [M][blocks of 64 of K] on the current device";
void fit_codes(PyObject* codes, PyObject* scales, int64_t M, int64_t K) {
  fits(codes, at::kChar, M, K, kCodesWhat);
  fits(scales, at::kFloat, M, (K + QB_CHECKPOINT_BLOCK - 1) / QB_CHECKPOINT_BLOCK, kScalesWhat);
}
void make_codes(Out& codes, Out& scales, int64_t M, int64_t K, at::Device device) {
  const int64_t blocks = (K + QB_CHECKPOINT_BLOCK - 1) / QB_CHECKPOINT_BLOCK;
  if (codes.obj || scales.obj) {
    codes.make({M, K}, at::kChar, device);
    scales.make({M, blocks}, at::kFloat, device);
    return;
  }
  const int64_t bytes = (M * K + 511) / 512 * 512;
  const at::Tensor both(at::detail::empty_cuda({bytes + M * blocks * 4}, at::kByte, device, std::nullopt));
  codes.make_in(both, 0, {M, K}, at::kChar);
  scales.make_in(both, bytes, {M, blocks}, at::kFloat);
}

// checkpoint(x, codes, scales) -> (codes, scales)
PyObject* checkpoint(Args a) {
  const char* const what = "x: a contiguous fp32, bfloat16 or fp16 CUDA tensor of two dimensions on the current device";
  const at::Tensor& x = matrix_here(a[0], what);
  const int type = element_type(x, what);
  const int64_t M = x.size(0), K = x.size(1);
  fit_codes(a[1], a[2], M, K);
  const at::Device device = x.device();
  const void* const x_data = x.const_data_ptr();
  Out codes(a[1]), scales(a[2]);
  qb_status st;
  {
    const Unlocked unlocked;
    make_codes(codes, scales, M, K, device);
    st = qb_checkpoint(x_data, type, M, K, static_cast<int8_t*>(codes.data), static_cast<float*>(scales.data), stream());
  }
  check(st, "qb_checkpoint");
  return tuple_of({&codes, &scales});
}

// restore(codes, scales, activation, type, y) -> y
PyObject* restore(Args a) {
  const at::Tensor& codes = matrix_here(a[0], kCodesWhat);
  const int64_t M = codes.size(0), K = codes.size(1);
  need(a[1] != Py_None, kScalesWhat);
  fit_codes(a[0], a[1], M, K);
  const int activation = (int)integer(a[2]), type = (int)integer(a[3]);
  const at::ScalarType scalar = type == QB_F32 ? at::kFloat : (type == QB_BF16 ? at::kBFloat16 : at::kHalf);
  fits(a[4], scalar, M, K, "y: contiguous [M][K] of the asked type on the current device");
  const at::Device device = codes.device();
  const int8_t* const code_data = codes.const_data_ptr<int8_t>();
  const float* const scales = static_cast<const float*>(ptr(a[1]));
  Out y(a[4]);
  qb_status st;
  {
    const Unlocked unlocked;
    y.make({M, K}, scalar, device);
    st = qb_restore(code_data, scales, M, K, activation, type, y.data, stream());
  }
  check(st, "qb_restore");
  return y.get();
}

// A pre-activation [M][K]: in `scalar`'s type, or as codes and scales, or none.
struct Pre {
  const void* pre;
  const int8_t* codes;
  const float* scales;
  Pre(PyObject* p, PyObject* c, PyObject* s, at::ScalarType scalar, int64_t M, int64_t K) {
    fits(p, scalar, M, K, "pre: contiguous, of the gradient's type, a value for each of the output's");
    fit_codes(c, s, M, K);
    pre = ptr(p);
    codes = static_cast<const int8_t*>(ptr(c));
    scales = static_cast<const float*>(ptr(s));
  }
};

// gelu_backward(grad_y, pre, codes, scales, grad_x) -> grad_x
PyObject* gelu_backward(Args a) {
  const char* const what = "grad_y: a contiguous fp32, bfloat16 or fp16 CUDA tensor of two dimensions on the current device";
  const at::Tensor& gy = matrix_here(a[0], what);
  const int type = element_type(gy, what);
  const int64_t M = gy.size(0), K = gy.size(1);
  const Pre p(a[1], a[2], a[3], gy.scalar_type(), M, K);
  fits(a[4], gy.scalar_type(), M, K, "grad_x: contiguous, of the type and shape of grad_y");
  const at::Device device = gy.device();
  const at::ScalarType scalar = gy.scalar_type();
  const void* const gy_data = gy.const_data_ptr();
  Out gx(a[4]);
  qb_status st;
  {
    const Unlocked unlocked;
    gx.make({M, K}, scalar, device);
    st = qb_gelu_backward(gy_data, type, p.pre, p.codes, p.scales, M, K, gx.data, stream());
  }
  check(st, "qb_gelu_backward");
  return gx.get();
}

int linear_type(const at::Tensor& t, const char* what) {
  need(t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf, what);
  return t.scalar_type() == at::kHalf ? QB_F16 : QB_BF16;
}

// linear(x, w, bias, ws, activation, residual, out32, save, y, pre, codes, scales) -> y, (y, pre) or (y, codes, scales); save 0: nothing, 1: pre, 2: codes
PyObject* linear(Args a) {
  const char* const what = "x: a contiguous bfloat16 or fp16 CUDA tensor [M][K] on the current device";
  const char* const what_w = "w: contiguous [N][K] of x's type on the current device";
  const at::Tensor& x = matrix_here(a[0], what);
  const int type = linear_type(x, what);
  const at::Tensor& w = matrix_here(a[1], what_w);
  need(w.scalar_type() == x.scalar_type() && w.size(1) == x.size(1), what_w);
  const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
  fits(a[2], at::kFloat, N, "bias: contiguous fp32 [N] on the current device");
  const Workspace ws = workspace_here(a[3]);
  const int activation = (int)integer(a[4]);
  const bool out32 = integer(a[6]) != 0;
  const int64_t save = integer(a[7]);
  const at::ScalarType scalar = x.scalar_type(), out_scalar = out32 ? at::kFloat : scalar;
  fits(a[5], out_scalar, M, N, "residual: contiguous [M][N] of the output's type on the current device");
  fits(a[8], out_scalar, M, N, "y: contiguous [M][N] of the asked type on the current device");
  fits(a[9], scalar, M, N, "pre: contiguous [M][N] of x's type on the current device");
  fit_codes(a[10], a[11], M, N);
  const at::Device device = x.device();
  const void *const x_data = x.const_data_ptr(), *const w_data = w.const_data_ptr(), *const residual = ptr(a[5]);
  const float* const bias = static_cast<const float*>(ptr(a[2]));
  Out y(a[8]), pre(save == 1 ? a[9] : Py_None), codes(save == 2 ? a[10] : Py_None), scales(save == 2 ? a[11] : Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    y.make({M, N}, out_scalar, device);
    if (save == 1) pre.make({M, N}, scalar, device);
    if (save == 2) make_codes(codes, scales, M, N, device);
    st = qb_linear(x_data, w_data, type, bias, activation, residual, M, N, K, out32 ? QB_F32 : type, y.data, pre.data, static_cast<int8_t*>(codes.data),
                   static_cast<float*>(scales.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_linear");
  if (save == 1) return tuple_of({&y, &pre});
  if (save == 2) return tuple_of({&y, &codes, &scales});
  return y.get();
}

// linear_grad_x(grad_y, w, ws, pre, codes, scales, residual, grad_x) -> grad_x
PyObject* linear_grad_x(Args a) {
  const char* const what = "grad_y: a contiguous bfloat16 or fp16 CUDA tensor [M][N] on the current device";
  const char* const what_w = "w: contiguous [N][K] of grad_y's type on the current device";
  const at::Tensor& gy = matrix_here(a[0], what);
  const int type = linear_type(gy, what);
  const at::Tensor& w = matrix_here(a[1], what_w);
  need(w.scalar_type() == gy.scalar_type() && w.size(0) == gy.size(1), what_w);
  const int64_t M = gy.size(0), N = gy.size(1), K = w.size(1);
  const Workspace ws = workspace_here(a[2]);
  const at::ScalarType scalar = gy.scalar_type();
  const Pre p(a[3], a[4], a[5], scalar, M, K);
  fits(a[6], scalar, M, K, "residual: contiguous [M][K] of grad_y's type on the current device");
  fits(a[7], scalar, M, K, "grad_x: contiguous [M][K] of grad_y's type on the current device");
  const at::Device device = gy.device();
  const void *const gy_data = gy.const_data_ptr(), *const w_data = w.const_data_ptr(), *const residual = ptr(a[6]);
  Out gx(a[7]);
  qb_status st;
  {
    const Unlocked unlocked;
    gx.make({M, K}, scalar, device);
    st = qb_linear_grad_x(gy_data, w_data, type, p.pre, p.codes, p.scales, residual, M, N, K, gx.data, ws.data, ws.bytes, stream());
  }
  check(st, "qb_linear_grad_x");
  return gx.get();
}

// linear_grad_w(grad_y, x, ws, out32, grad_w, grad_bias, need_w, need_bias) -> (grad_w, grad_bias)
PyObject* linear_grad_w(Args a) {
  const char* const what = "grad_y: a contiguous bfloat16 or fp16 CUDA tensor [M][N] on the current device";
  const char* const what_x = "x: contiguous [M][K] of grad_y's type on the current device";
  const at::Tensor& gy = matrix_here(a[0], what);
  const int type = linear_type(gy, what);
  const at::Tensor& x = matrix_here(a[1], what_x);
  need(x.scalar_type() == gy.scalar_type() && x.size(0) == gy.size(0), what_x);
  const int64_t M = gy.size(0), N = gy.size(1), K = x.size(1);
  const Workspace ws = workspace_here(a[2]);
  const bool out32 = integer(a[3]) != 0, want_w = integer(a[6]) != 0, want_b = integer(a[7]) != 0;
  const at::ScalarType scalar = out32 ? at::kFloat : gy.scalar_type();
  fits(a[4], scalar, N, K, "grad_w: contiguous [N][K] of the asked type on the current device");
  fits(a[5], at::kFloat, N, "grad_bias: contiguous fp32 [N] on the current device");
  const at::Device device = gy.device();
  const void *const gy_data = gy.const_data_ptr(), *const x_data = x.const_data_ptr();
  Out gw(want_w ? a[4] : Py_None), gb(want_b ? a[5] : Py_None);
  qb_status st;
  {
    const Unlocked unlocked;
    if (want_w) gw.make({N, K}, scalar, device);
    if (want_b) gb.make({N}, at::kFloat, device);
    st = qb_linear_grad_w(gy_data, x_data, type, M, N, K, out32 ? QB_F32 : type, gw.data, static_cast<float*>(gb.data), ws.data, ws.bytes, stream());
  }
  check(st, "qb_linear_grad_w");
  if (want_w) gw.wrap();
  if (want_b) gb.wrap();
  return Py_BuildValue("(NN)", want_w ? gw.get() : Py_NewRef(Py_None), want_b ? gb.get() : Py_NewRef(Py_None));
}

// The calls over an array of descriptors: (array, ws)
template <class T, qb_status (*F)(const T*, int32_t, void*, size_t, void*)>
PyObject* over_descs(Args a, const char* what) {
  const Descs d(a[0]);
  const Workspace ws(a[1]);
  int32_t count = 0;
  const T* p = d.as<T>(&count);
  qb_status st;
  {
    const Unlocked unlocked;
    st = F(p, count, ws.data, ws.bytes, stream());
  }
  check(st, what);
  Py_RETURN_NONE;
}
PyObject* quantize_act_batch(Args a) { return over_descs<qb_act_desc, qb_quantize_act_batch>(a, "qb_quantize_act_batch"); }
PyObject* quantize_pack_weights_batch(Args a) {
  return over_descs<qb_weight_desc, qb_quantize_pack_weights_batch>(a, "qb_quantize_pack_weights_batch");
}
PyObject* fake_quantize_weights_batch(Args a) {
  return over_descs<qb_weight_desc, qb_fake_quantize_weights_batch>(a, "qb_fake_quantize_weights_batch");
}
PyObject* layer_linears(Args a) { return over_descs<qb_linear_desc, qb_layer_linears>(a, "qb_layer_linears"); }
PyObject* layer_linears_bf16(Args a) { return over_descs<qb_linear_desc, qb_layer_linears_bf16>(a, "qb_layer_linears_bf16"); }

PyObject* set_raise(Args a) {
  Py_XSETREF(g_raise, Py_NewRef(a[0]));
  Py_RETURN_NONE;
}

template <PyObject* (*F)(Args), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
    return nullptr;
  }
  HANDLE_TH_ERRORS  // what torch throws (out of memory, no device) becomes the exception torch raises for it
  try {
    return F(args);
  } catch (const Failed&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
#define QB_ENTRY(f, n) {#f, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {QB_ENTRY(quantize_act, 5),
                           QB_ENTRY(gemm, 14),
                           QB_ENTRY(rowsum_i8, 2),
                           QB_ENTRY(quantize_pack_weights, 9),
                           QB_ENTRY(fake_quantize_weights, 7),
                           QB_ENTRY(ste_backward, 6),
                           QB_ENTRY(quantize_embedding, 5),
                           QB_ENTRY(embedding_lookup, 10),
                           QB_ENTRY(dropout, 6),
                           QB_ENTRY(quantize_fp8, 11),
                           QB_ENTRY(gemm_fp8, 8),
                           QB_ENTRY(vocab_loss, 7),
                           QB_ENTRY(vocab_loss_backward, 13),
                           QB_ENTRY(layer_norm, 8),
                           QB_ENTRY(layer_norm_backward, 10),
                           QB_ENTRY(checkpoint, 3),
                           QB_ENTRY(restore, 5),
                           QB_ENTRY(gelu_backward, 5),
                           QB_ENTRY(linear, 12),
                           QB_ENTRY(linear_grad_x, 8),
                           QB_ENTRY(linear_grad_w, 8),
                           QB_ENTRY(quantize_act_batch, 2),
                           QB_ENTRY(quantize_pack_weights_batch, 2),
                           QB_ENTRY(fake_quantize_weights_batch, 2),
                           QB_ENTRY(layer_linears, 2),
                           QB_ENTRY(layer_linears_bf16, 2),
                           QB_ENTRY(set_raise, 1),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_qbert", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qbert(void) { return PyModule_Create(&g_module); }
