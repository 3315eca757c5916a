// The marshalling half of jq_block.py: tensors checked and turned into the
// pointers of include/jq_block.h, missing outputs and workspaces allocated, the
// current stream looked up.  It computes nothing.  The calls of a decoding step
// are a few microseconds of GPU work each; the same checks in Python took 10 to
// 15 us a call (and ctypes 3 of them for 27 arguments), which is what bound
// such a step.
//
// Functions take positional arguments, a fixed number each (jq_block.py is the
// public interface, with names, defaults and documentation), and return their
// outputs, or the status as an int where the library refused.

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/python_headers.h>

#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>

#include <optional>

#include "jq_block.h"

namespace {

using at::Tensor;

// One call's tensors: all on the device of the first one seen.
class Call {
 public:
  // For the call, the current device becomes that of this tensor, and the
  // current stream the one that the caller gave (None: as it is): what the call
  // allocates then belongs to that stream, so a workspace that it lets go at the
  // end is not handed to another stream's work while the kernels still use it.
  Call(PyObject* o, const char* name, PyObject* stream) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a torch.Tensor");
    const Tensor& t = THPVariable_Unpack(o);
    TORCH_CHECK_VALUE(t.is_cuda(), name, " must be on the GPU, got ", t.device());
    device_ = t.device();
    guard_.reset_device(device_);
    if (stream != Py_None) {
      void* given = PyLong_AsVoidPtr(stream);
      if (given == nullptr && PyErr_Occurred()) throw python_error();
      stream_.reset_stream(c10::hip::getStreamFromExternal(static_cast<hipStream_t>(given), device_.index()));
    }
  }

  const Tensor& tensor(PyObject* o, const char* name, at::ScalarType type) const {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a torch.Tensor");
    const Tensor& t = THPVariable_Unpack(o);
    TORCH_CHECK_VALUE(t.is_cuda(), name, " must be on the GPU, got ", t.device());
    TORCH_CHECK_VALUE(t.device() == device_, "all tensors must be on one device, got ", device_, " and ", t.device(),
                      " for ", name);
    TORCH_CHECK_TYPE(t.scalar_type() == type, name, " must be ", type, ", got ", t.scalar_type());
    return t;
  }
  // A contiguous tensor; of this shape, if one is given.
  const Tensor& dense(PyObject* o, const char* name, at::ScalarType type) const {
    const Tensor& t = tensor(o, name, type);
    TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
    return t;
  }
  const Tensor& dense(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    const Tensor& t = dense(o, name, type);
    TORCH_CHECK_VALUE(t.sizes() == shape, name, " must have shape ", shape, ", got ", t.sizes());
    return t;
  }
  // The same, or a new one where the caller gave None.
  Tensor out(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    return o == Py_None ? make(type, shape) : dense(o, name, type, shape);
  }
  Tensor make(at::ScalarType type, at::IntArrayRef shape) const {
    // torch's allocator without its dispatcher, half the time of at::empty
    return Tensor(at::detail::empty_cuda(shape, type, device_, std::nullopt));
  }
  // A tensor whose rows (all but the first dimension) are contiguous; the elements between them.
  const Tensor& rows(PyObject* o, const char* name, at::IntArrayRef shape, int64_t* stride) const {
    const Tensor& t = tensor(o, name, at::kBFloat16);
    TORCH_CHECK_VALUE(t.sizes() == shape, name, " must have shape ", shape, ", got ", t.sizes());
    int64_t need = 1;
    for (int64_t d = t.dim() - 1; d >= 1; --d) {
      TORCH_CHECK_VALUE(t.size(d) == 1 || t.stride(d) == need, name, ": the elements of a row must be contiguous");
      need *= t.size(d);
    }
    *stride = t.size(0) > 1 ? t.stride(0) : need;
    return t;
  }
  void* stream() const { return c10::hip::getCurrentHIPStream(device_.index()).stream(); }

 private:
  at::Device device_{at::kCPU};
  c10::OptionalDeviceGuard guard_;
  c10::hip::OptionalHIPStreamGuard stream_;
};

void* ptr(const Tensor& t) { return t.data_ptr(); }
float* f32(const Tensor& t) { return static_cast<float*>(t.data_ptr()); }
int64_t blocks(int64_t n) { return (n + 127) / 128; }

int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v != 0;
}

PyObject* wrap(const Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrap(const Tensor& a, const Tensor& b) {
  PyObject* r = PyTuple_New(2);
  if (r == nullptr) throw python_error();
  PyTuple_SET_ITEM(r, 0, wrap(a));
  PyTuple_SET_ITEM(r, 1, wrap(b));
  return r;
}
PyObject* refused(jq_status st) { return PyLong_FromLong(st); }

void count(Py_ssize_t got, Py_ssize_t want) { TORCH_CHECK_TYPE(got == want, want, " arguments expected, got ", got); }

const Tensor& matrix(const Tensor& t, const char* name) {
  TORCH_CHECK_VALUE(t.dim() == 2, name, " must be a matrix, got shape ", t.sizes());
  return t;
}

constexpr at::ScalarType kBf16 = at::kBFloat16, kFp8 = at::kFloat8_e4m3fn, kF32 = at::kFloat;

// x, weight, eps, residual, out, y, scale, residual_out, stream
PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 9);
  TORCH_CHECK_VALUE(a[3] != Py_None || a[7] == Py_None, "residual_out without a residual");
  Call c(a[0], "x", a[8]);
  const Tensor& x = matrix(c.tensor(a[0], "x", kBf16), "x");
  const int64_t M = x.size(0), D = x.size(1), out = integer(a[4]);
  int64_t xs = 0, rs = 0, ros = 0;
  c.rows(a[0], "x", x.sizes(), &xs);
  const Tensor& w = c.dense(a[1], "weight", kBf16, {D});
  Tensor y = c.out(a[5], "y", out == JQ_NORM_BF16 ? kBf16 : out == JQ_NORM_FP8 ? kFp8 : at::kByte,
                   {M, out == JQ_NORM_INT4 ? D / 2 : D});
  Tensor scale, res_out;
  if (out == JQ_NORM_FP8) scale = c.out(a[6], "scale", kF32, {M, blocks(D)});
  else if (out == JQ_NORM_INT4) scale = c.out(a[6], "scale", kF32, {M});
  else TORCH_CHECK_VALUE(a[6] == Py_None, "a bf16 output has no scale");
  const bool res = a[3] != Py_None;
  const void* rp = nullptr;
  if (res) {
    rp = ptr(c.rows(a[3], "residual", x.sizes(), &rs));
    res_out = a[7] == Py_None ? c.make(kBf16, x.sizes()) : c.rows(a[7], "residual_out", x.sizes(), &ros);
    if (a[7] == Py_None) ros = D;
  }
  const jq_status st = jq_rmsnorm(ptr(x), xs, rp, rs, ptr(w), M, D, static_cast<float>(number(a[2])),
                                  static_cast<jq_norm_out>(out), ptr(y), scale.defined() ? f32(scale) : nullptr,
                                  res ? ptr(res_out) : nullptr, ros, c.stream());
  if (st != JQ_OK) return refused(st);
  PyObject* r = PyTuple_New(1 + scale.defined() + res);
  if (r == nullptr) throw python_error();
  Py_ssize_t i = 0;
  PyTuple_SET_ITEM(r, i++, wrap(y));
  if (scale.defined()) PyTuple_SET_ITEM(r, i++, wrap(scale));
  if (res) PyTuple_SET_ITEM(r, i++, wrap(res_out));
  return r;
  END_HANDLE_TH_ERRORS
}

// x, q, scale, stream
PyObject* quantize_act_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 4);
  Call c(a[0], "x", a[3]);
  const Tensor& x = matrix(c.tensor(a[0], "x", kBf16), "x");
  const int64_t M = x.size(0), K = x.size(1);
  int64_t xs = 0;
  c.rows(a[0], "x", x.sizes(), &xs);
  Tensor q = c.out(a[1], "q", kFp8, {M, K}), s = c.out(a[2], "scale", kF32, {M, blocks(K)});
  const jq_status st = jq_quantize_act_fp8(ptr(x), xs, M, K, ptr(q), f32(s), c.stream());
  return st == JQ_OK ? wrap(q, s) : refused(st);
  END_HANDLE_TH_ERRORS
}

// w, wq, w_scale, stream
PyObject* pack_weight_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 4);
  Call c(a[0], "w", a[3]);
  const Tensor& w = matrix(c.dense(a[0], "w", kBf16), "w");
  const int64_t N = w.size(0), K = w.size(1);
  Tensor q = c.out(a[1], "wq", kFp8, {N, K}), s = c.out(a[2], "w_scale", kF32, {blocks(N), blocks(K)});
  const jq_status st = jq_pack_weight_fp8(ptr(w), N, K, ptr(q), f32(s), c.stream());
  return st == JQ_OK ? wrap(q, s) : refused(st);
  END_HANDLE_TH_ERRORS
}

struct Weight {
  const Tensor& q;
  const Tensor& s;
  const void* bias;
  int64_t N;
};
Weight weight(const Call& c, PyObject* wq, PyObject* ws, PyObject* bias, int64_t K) {
  const Tensor& q = matrix(c.dense(wq, "wq", kFp8), "wq");
  const int64_t N = q.size(0);
  TORCH_CHECK_VALUE(q.size(1) == K, "wq must have ", K, " columns, got shape ", q.sizes());
  const Tensor& s = c.dense(ws, "w_scale", kF32, {blocks(N), blocks(K)});
  return {q, s, bias == Py_None ? nullptr : ptr(c.dense(bias, "bias", kBf16, {N})), N};
}

// q, scale, wq, w_scale, bias, y, stream
PyObject* fp8_gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 7);
  Call c(a[0], "q", a[6]);
  const Tensor& q = matrix(c.dense(a[0], "q", kFp8), "q");
  const int64_t M = q.size(0), K = q.size(1);
  const Tensor& s = c.dense(a[1], "scale", kF32, {M, blocks(K)});
  const Weight w = weight(c, a[2], a[3], a[4], K);
  Tensor y = c.out(a[5], "y", kBf16, {M, w.N});
  const jq_status st = jq_fp8_gemm(ptr(q), f32(s), M, K, ptr(w.q), f32(w.s), w.N, w.bias, ptr(y), c.stream());
  return st == JQ_OK ? wrap(y) : refused(st);
  END_HANDLE_TH_ERRORS
}

// x, wq, w_scale, bias, y, workspace, stream
PyObject* fp8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 7);
  Call c(a[0], "x", a[6]);
  const Tensor& x = matrix(c.tensor(a[0], "x", kBf16), "x");
  const int64_t M = x.size(0), K = x.size(1);
  int64_t xs = 0;
  c.rows(a[0], "x", x.sizes(), &xs);
  const Weight w = weight(c, a[1], a[2], a[3], K);
  Tensor y = c.out(a[4], "y", kBf16, {M, w.N});
  Tensor ws = a[5] == Py_None ? c.make(at::kByte, {static_cast<int64_t>(jq_fp8_workspace_bytes(M, K))})
                              : c.dense(a[5], "workspace", at::kByte);
  const jq_status st = jq_fp8_linear(ptr(x), xs, M, K, ptr(w.q), f32(w.s), w.N, w.bias, ptr(y), ptr(ws), ws.numel(),
                                     c.stream());
  return st == JQ_OK ? wrap(y) : refused(st);
  END_HANDLE_TH_ERRORS
}

struct Cache {
  const Tensor& k;
  const Tensor& v;
  float *ks, *vs;
  int64_t pages, Hk, page, D;
  jq_cache_type type;
};
// What a cache's type asks of its scales; the type.
at::ScalarType cache_type(PyObject* ko, PyObject* kso, PyObject* vso) {
  TORCH_CHECK_TYPE(THPVariable_Check(ko), "k_cache must be a torch.Tensor");
  const at::ScalarType type = THPVariable_Unpack(ko).scalar_type();
  TORCH_CHECK_TYPE(type == kBf16 || type == kFp8, "k_cache must be ", kBf16, " or ", kFp8, ", got ", type);
  if (type == kBf16) {
    TORCH_CHECK_VALUE(kso == Py_None && vso == Py_None, "a bf16 cache has no scales");
    return kBf16;
  }
  TORCH_CHECK_VALUE(kso != Py_None && vso != Py_None, "an 8-bit cache needs k_scale and v_scale");
  return kFp8;
}
Cache cache(const Call& c, at::ScalarType type, PyObject* ko, PyObject* vo, PyObject* kso, PyObject* vso) {
  const Tensor& k = c.dense(ko, "k_cache", type);
  TORCH_CHECK_VALUE(k.dim() == 4, "a cache is [pages, Hk, page_size, D], got shape ", k.sizes());
  const Tensor& v = c.dense(vo, "v_cache", type, k.sizes());
  float *ks = nullptr, *vs = nullptr;
  if (type == kFp8) {
    ks = f32(c.dense(kso, "k_scale", kF32, k.sizes().slice(0, 3)));
    vs = f32(c.dense(vso, "v_scale", kF32, k.sizes().slice(0, 3)));
  }
  return {k, v, ks, vs, k.size(0), k.size(1), k.size(2), k.size(3), type == kBf16 ? JQ_CACHE_BF16 : JQ_CACHE_FP8};
}

// q, k, v, positions, cos, sin, slots, k_cache, v_cache, k_scale, v_scale, interleaved, q_out, stream
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 14);
  const at::ScalarType type = cache_type(a[7], a[9], a[10]);
  Call c(a[1], "k", a[13]);
  const Cache kv = cache(c, type, a[7], a[8], a[9], a[10]);
  const Tensor& k = c.tensor(a[1], "k", kBf16);
  TORCH_CHECK_VALUE(k.dim() == 3, "k must be [T, Hk, D], got shape ", k.sizes());
  const int64_t T = k.size(0);
  int64_t ks = 0, vs = 0, qs = 0, qos = 0, Hq = 0, P = 0, R = 0;
  c.rows(a[1], "k", {T, kv.Hk, kv.D}, &ks);
  const Tensor& v = c.rows(a[2], "v", {T, kv.Hk, kv.D}, &vs);
  const void* qp = nullptr;
  Tensor q_out;
  if (a[0] != Py_None) {
    const Tensor& q = c.tensor(a[0], "q", kBf16);
    TORCH_CHECK_VALUE(q.dim() == 3 && q.size(1) > 0, "q must be [T, Hq, D], got shape ", q.sizes());
    Hq = q.size(1);
    qp = ptr(c.rows(a[0], "q", {T, Hq, kv.D}, &qs));
    q_out = a[12] == Py_None ? c.make(kBf16, {T, Hq, kv.D}) : c.rows(a[12], "q_out", {T, Hq, kv.D}, &qos);
    if (a[12] == Py_None) qos = Hq * kv.D;
  } else {
    TORCH_CHECK_VALUE(a[12] == Py_None, "q_out without q");
  }
  const float *cos = nullptr, *sin = nullptr;
  if (a[4] != Py_None) {
    const Tensor& t = matrix(c.dense(a[4], "cos", kF32), "cos");
    P = t.size(0), R = 2 * t.size(1);
    cos = f32(t), sin = f32(c.dense(a[5], "sin", kF32, t.sizes()));
  } else {
    TORCH_CHECK_VALUE(a[5] == Py_None, "sin without cos");
  }
  const Tensor& pos = c.dense(a[3], "positions", at::kInt, {T});
  const Tensor& slots = c.dense(a[6], "slots", at::kLong, {T});
  const jq_status st = jq_rope_append(
      qp, qs, ptr(k), ks, ptr(v), vs, T, Hq, kv.Hk, kv.D, static_cast<const int32_t*>(ptr(pos)), cos, sin, P, R,
      truth(a[11]), static_cast<const int64_t*>(ptr(slots)), q_out.defined() ? ptr(q_out) : nullptr, qos, ptr(kv.k),
      ptr(kv.v), kv.ks, kv.vs, kv.pages, kv.page, kv.type, c.stream());
  if (st != JQ_OK) return refused(st);
  if (q_out.defined()) return wrap(q_out);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// q, k_cache, v_cache, page_table, lens, k_scale, v_scale, max_len, sm_scale, causal, out, lse, workspace, stream
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  count(n, 14);
  const at::ScalarType type = cache_type(a[1], a[5], a[6]);
  Call c(a[0], "q", a[13]);
  const Cache kv = cache(c, type, a[1], a[2], a[5], a[6]);
  const Tensor& q = c.dense(a[0], "q", kBf16);
  TORCH_CHECK_VALUE(q.dim() == 4, "q must be [B, Tq, Hq, D], got shape ", q.sizes());
  const int64_t B = q.size(0), Tq = q.size(1), Hq = q.size(2), D = q.size(3);
  TORCH_CHECK_VALUE(D == kv.D, "q has heads of ", D, ", the cache of ", kv.D);
  const Tensor& table = c.dense(a[3], "page_table", at::kInt);
  TORCH_CHECK_VALUE(table.dim() == 2 && table.size(0) == B, "page_table must be [", B, ", columns], got shape ", table.sizes());
  const Tensor& lens = c.dense(a[4], "lens", at::kInt, {B});
  const int64_t max_len = a[7] == Py_None ? table.size(1) * kv.page : integer(a[7]);
  const double scale = a[8] == Py_None ? 1.0 / std::sqrt(static_cast<double>(D)) : number(a[8]);
  Tensor out = c.out(a[10], "out", kBf16, q.sizes());
  float* lse = a[11] == Py_None ? nullptr : f32(c.dense(a[11], "lse", kF32, {B, Tq, Hq}));
  Tensor ws;
  if (a[12] != Py_None) {
    ws = c.dense(a[12], "workspace", at::kByte);
  } else if (const size_t need = jq_paged_attention_workspace_bytes(B, Tq, Hq, kv.Hk, D, max_len)) {
    ws = c.make(at::kByte, {static_cast<int64_t>(need)});
  }
  const jq_status st = jq_paged_attention(
      ptr(q), ptr(kv.k), ptr(kv.v), kv.ks, kv.vs, static_cast<const int32_t*>(ptr(table)), table.size(1),
      static_cast<const int32_t*>(ptr(lens)), B, Tq, Hq, kv.Hk, D, kv.pages, kv.page, max_len,
      static_cast<float>(scale), truth(a[9]), kv.type, ptr(out), lse, ws.defined() ? ptr(ws) : nullptr,
      ws.defined() ? ws.numel() : 0, c.stream());
  return st == JQ_OK ? wrap(out) : refused(st);
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<rmsnorm>("rmsnorm"),
                         method<quantize_act_fp8>("quantize_act_fp8"),
                         method<pack_weight_fp8>("pack_weight_fp8"),
                         method<fp8_gemm>("fp8_gemm"),
                         method<fp8_linear>("fp8_linear"),
                         method<rope_append>("rope_append"),
                         method<paged_attention>("paged_attention"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_jq_block", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__jq_block() { return PyModule_Create(&module); }
