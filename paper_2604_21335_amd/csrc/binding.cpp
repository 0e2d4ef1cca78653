// Python's way into the C ABI: checks and unpacks torch tensors in native code.  A call takes up to 12
// of them, and looking at one through the interpreter costs 0.45 us, as much as a launch costs for
// five; here it is 0.01 us.  Nothing is computed here and nothing is kept between calls.
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/stc.h"

namespace {

PyObject* g_error;       // StcError(status, where)
PyObject* g_shape;       // stc_shape_t
PyObject* g_device;      // torch._C._cuda_getDevice
PyObject* g_raw_stream;  // torch._C._cuda_getCurrentRawStream, which takes the device
PyObject* g_any_stream;  // the package's own way, for builds of torch without these two

struct PythonError {};  // the interpreter's error is set

constexpr at::ScalarType kBf16 = at::kBFloat16, kF32 = at::kFloat, kU8 = at::kByte, kF64 = at::kDouble;

// The arguments of one call, in order.
class Args {
 public:
  Args(const char* where, PyObject* const* args, Py_ssize_t n, Py_ssize_t want)
      : where_(where), args_(args) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, not %zd", where, want, n);
      throw PythonError();
    }
  }

  const stc_shape_t* shape() {
    PyObject* o = next();
    const int is = PyObject_IsInstance(o, g_shape);
    if (is == 0) PyErr_Format(PyExc_TypeError, "%s: shape must be a stc_shape_t", where_);
    Py_buffer b;
    if (is != 1 || PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw PythonError();
    memcpy(&shape_, b.buf, sizeof shape_);  // a subclass can only be larger
    PyBuffer_Release(&b);
    return &shape_;
  }

  // Device pointer of a contiguous tensor (None: nullptr) of one of the given types.
  template <class... T>
  void* tensor(const char* name, T... types) {
    PyObject* o = next();
    bytes_ = 0;
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) {
      PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
      throw PythonError();
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
      throw PythonError();
    }
    if (sizeof...(T) > 0 && !((t.scalar_type() == types) || ...)) {
      PyObject* dtype = PyObject_GetAttrString(o, "dtype");
      if (dtype) PyErr_Format(PyExc_TypeError, "%s has dtype %S", name, dtype);
      Py_XDECREF(dtype);
      throw PythonError();
    }
    on_device(name, t);
    bytes_ = (size_t)t.numel() * t.element_size();
    return t.data_ptr();
  }
  void* bf16(const char* name) { return tensor(name, kBf16); }
  float* f32(const char* name) { return (float*)tensor(name, kF32); }
  uint8_t* u8(const char* name) { return (uint8_t*)tensor(name, kU8); }
  uint16_t* u16(const char* name) { return (uint16_t*)tensor(name, at::kShort, at::kUInt16); }
  uint32_t* u32(const char* name) { return (uint32_t*)tensor(name, at::kInt, at::kUInt32); }
  int32_t* i32(const char* name) { return (int32_t*)tensor(name, at::kInt); }
  void* ws() { return tensor("ws"); }
  size_t bytes() const { return bytes_; }  // of the tensor taken last

  // From here on: the call's tensors lie on one device, the current one.
  void one_device() { one_device_ = true; }

  void need(bool ok, const char* name, const char* what) {
    if (ok) return;
    PyErr_Format(PyExc_ValueError, "%s: %s %s", where_, name, what);
    throw PythonError();
  }

  // A contiguous tensor of exactly n elements (None: nullptr).
  template <class... T>
  void* sized(const char* name, int64_t n, T... types) {
    PyObject* o = args_[at_];
    void* p = tensor(name, types...);
    if (o != Py_None) need(THPVariable_Unpack(o).numel() == n, name, "has another size");
    return p;
  }

  // A bf16 tensor of `dims` dimensions whose last one is contiguous.
  struct Rows {
    void* p;
    int64_t size[4], stride[4];  // stride 0 where there is nothing to step over
  };
  Rows rows(const char* name, int dims) {
    PyObject* o = next();
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) {
      PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
      throw PythonError();
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    on_device(name, t);
    if (t.scalar_type() != kBf16) {
      PyErr_Format(PyExc_TypeError, "%s must be bfloat16", name);
      throw PythonError();
    }
    need(t.dim() == dims, name, "has another number of dimensions");
    Rows r{t.data_ptr(), {}, {}};
    for (int i = 0; i < dims; ++i) r.size[i] = t.size(i), r.stride[i] = t.size(i) > 1 ? t.stride(i) : 0;
    need(r.size[dims - 1] > 1 && r.size[dims - 1] <= INT32_MAX && r.stride[dims - 1] == 1, name, "must be contiguous in its last dimension");
    need(t.numel() > 0 && t.numel() / r.size[dims - 1] <= INT32_MAX, name, "is empty or too large");
    return r;
  }

  // The next argument stands for the number of layers' tensors: a list or tuple of them, of at least one.
  // (They stay where this object is, which outlives the call.)
  struct Many {
    static constexpr int kMost = 1024;
    void* p[kMost];
    int n;
  };
  Many tails[4];
  template <class... T>
  void many(Many& m, const char* name, int64_t numel, T... types) {
    PyObject* o = next();
    if (!PyList_Check(o) && !PyTuple_Check(o)) {
      PyErr_Format(PyExc_TypeError, "%s must be a list or tuple of tensors", name);
      throw PythonError();
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
    need(n >= 1 && n <= Many::kMost, name, "must have 1 to 1024 tensors");
    m.n = (int)n;
    PyObject* const* const args = args_;
    const Py_ssize_t at = at_;
    args_ = PySequence_Fast_ITEMS(o), at_ = 0;
    for (Py_ssize_t i = 0; i < n; ++i) m.p[i] = sized(name, numel, types...);
    args_ = args, at_ = at;
  }

  float real() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return (float)v;
  }

  // What int() takes; index(): whole numbers only.
  int integer() { return number(PyNumber_Long); }
  int index() { return number(PyNumber_Index); }

  // The current stream of the current device.
  void* stream() {
    PyObject* s = nullptr;
    if (g_device && g_raw_stream) {
      PyObject* dev = PyObject_CallNoArgs(g_device);
      if (dev && one_device_ && device_ >= 0 && PyLong_AsLong(dev) != device_) {
        PyErr_Format(PyExc_ValueError, "%s: the tensors are not on the current device", where_);
        Py_DECREF(dev);
        throw PythonError();
      }
      if (dev) s = PyObject_CallOneArg(g_raw_stream, dev);
      Py_XDECREF(dev);
    } else {
      s = PyObject_CallNoArgs(g_any_stream);
    }
    if (!s) throw PythonError();
    void* p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw PythonError();
    return p;
  }

 private:
  PyObject* next() { return args_[at_++]; }
  void on_device(const char* name, const at::Tensor& t) {
    if (!one_device_) return;
    if (device_ < 0) device_ = t.get_device();
    need(t.get_device() == device_, name, "is on another device than the tensors before it");
  }
  int number(PyObject* (*convert)(PyObject*)) {
    PyObject* o = next();
    PyObject* i = PyLong_CheckExact(o) ? Py_NewRef(o) : convert(o);
    if (!i) throw PythonError();
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(i);
    Py_DECREF(i);
    if (v == ~0ull && PyErr_Occurred()) throw PythonError();
    return (int)v;
  }
  const char* where_;
  PyObject* const* args_;
  Py_ssize_t at_ = 0;
  stc_shape_t shape_;
  size_t bytes_ = 0;
  bool one_device_ = false;
  int device_ = -1;
};

// Runs `body`, which takes the arguments in order and returns the call to make; the call runs without
// the interpreter's lock.  A status other than STC_OK raises StcError.
template <class Body>
PyObject* run(const char* where, PyObject* const* args, Py_ssize_t n, Py_ssize_t want, Body body) {
  try {
    Args a(where, args, n, want);
    auto call = body(a);
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    if (status != STC_OK) {
      PyObject* e = PyObject_CallFunction(g_error, "is", status, where);
      if (e) PyErr_SetObject(g_error, e);
      Py_XDECREF(e);
      return nullptr;
    }
    Py_RETURN_NONE;
  } catch (const PythonError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define STC_PY(name, want, ...)                                                           \
  PyObject* name(PyObject*, PyObject* const* args, Py_ssize_t n) {                        \
    return run("stc_" #name, args, n, want, [](Args& a) { __VA_ARGS__ });                 \
  }

STC_PY(build_page_bounds, 3,
  auto s = *a.shape(); auto K = a.bf16("K"); auto bounds = a.bf16("bounds"); auto st = a.stream();
  return [=] { return stc_build_page_bounds(&s, K, bounds, st); };)

STC_PY(route_and_pack_values, 12,
  auto s = *a.shape(); auto mode = a.index(); auto V = a.bf16("V"); auto logits = a.f32("logits");
  auto kcount = a.u8("kcount"); auto fixed_k = a.integer(); auto mask_in = a.u16("mask_in");
  auto mask = a.u16("mask"); auto off = a.u32("tok_off"); auto vpacked = a.bf16("vpacked");
  auto status = a.i32("dev_status"); auto ws = a.ws(); auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_route_and_pack_values(&s, mode, V, logits, kcount, fixed_k, mask_in, mask, off, vpacked, status, ws, nws, st); };)

#define STC_PY_SELECT(name)                                                                        \
  STC_PY(name, 7,                                                                                  \
    auto s = *a.shape(); auto q = a.bf16("q"); auto bounds = a.bf16("bounds"); auto k = a.integer(); \
    auto idx = a.i32("page_idx"); auto score = a.f32("page_score"); auto ws = a.ws();              \
    auto nws = a.bytes(); auto st = a.stream();                                                    \
    return [=] { return stc_##name(&s, q, bounds, k, idx, score, ws, nws, st); };)
STC_PY_SELECT(select_pages)
STC_PY_SELECT(select_pages_per_head)

STC_PY(score_pages, 4,
  auto s = *a.shape(); auto q = a.bf16("q"); auto bounds = a.bf16("bounds");
  auto score = a.f32("page_score"); auto st = a.stream();
  return [=] { return stc_score_pages(&s, q, bounds, score, st); };)

#define STC_PY_ATTENTION(name)                                                                     \
  STC_PY(name, 10,                                                                                 \
    auto s = *a.shape(); auto q = a.bf16("q"); auto K = a.bf16("K"); auto v = a.bf16("vpacked");   \
    auto mask = a.u16("mask"); auto off = a.u32("tok_off"); auto idx = a.i32("page_idx");          \
    auto k = a.integer(); auto out = a.f32("out"); auto ws = a.ws(); auto nws = a.bytes();         \
    auto st = a.stream();                                                                          \
    return [=] { return stc_##name(&s, q, K, v, mask, off, idx, k, out, ws, nws, st); };)
STC_PY_ATTENTION(decode_attention)
STC_PY_ATTENTION(decode_attention_per_head)

STC_PY(decode_attention_tail, 14,
  auto s = *a.shape(); auto q = a.bf16("q"); auto K = a.bf16("K"); auto v = a.bf16("vpacked");
  auto mask = a.u16("mask"); auto off = a.u32("tok_off"); auto idx = a.i32("page_idx");
  auto k = a.integer(); auto Kt = a.bf16("K_tail"); auto Vt = a.bf16("V_tail");
  auto n_tail = a.integer(); auto cap = a.integer(); auto out = a.f32("out"); auto ws = a.ws();
  auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_decode_attention_tail(&s, q, K, v, mask, off, idx, k, Kt, Vt, n_tail, cap, out, ws, nws, st); };)

STC_PY(decode_attention_union, 11,
  auto s = *a.shape(); auto q = a.bf16("q"); auto K = a.bf16("K"); auto v = a.bf16("vpacked");
  auto mask = a.u16("mask"); auto off = a.u32("tok_off"); auto idx = a.i32("union_idx");
  auto heads = a.u16("union_heads"); auto cap = a.integer(); auto out = a.f32("out");
  auto ws = a.ws(); auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_decode_attention_union(&s, q, K, v, mask, off, idx, heads, cap, out, ws, nws, st); };)

STC_PY(union_pages, 6,
  auto s = *a.shape(); auto lists = a.i32("page_idx_per_head"); auto k = a.integer();
  auto idx = a.i32("union_idx"); auto heads = a.u16("union_heads"); auto cap = a.integer();
  auto st = a.stream();
  return [=] { return stc_union_pages(&s, lists, k, idx, heads, cap, st); };)

STC_PY(decode_step, 11,
  auto s = *a.shape(); auto q = a.bf16("q"); auto bounds = a.bf16("bounds"); auto K = a.bf16("K");
  auto v = a.bf16("vpacked"); auto mask = a.u16("mask"); auto off = a.u32("tok_off");
  auto k = a.integer(); auto idx = a.i32("page_idx"); auto out = a.f32("out"); auto ws = a.ws();
  auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_decode_step(&s, q, bounds, K, v, mask, off, k, idx, out, ws, nws, st); };)

STC_PY(decode_step_static, 10,
  auto s = *a.shape(); auto q = a.bf16("q"); auto bounds = a.bf16("bounds"); auto K = a.bf16("K");
  auto v = a.bf16("vpacked"); auto mask = a.u16("mask"); auto off = a.u32("tok_off");
  auto k = a.integer(); auto idx = a.i32("page_idx"); auto out = a.f32("out"); auto st = a.stream();
  return [=] { return stc_decode_step_static(&s, q, bounds, K, v, mask, off, k, idx, out, st); };)

STC_PY(decode_step_tail, 15,
  auto s = *a.shape(); auto q = a.bf16("q"); auto bounds = a.bf16("bounds"); auto K = a.bf16("K");
  auto v = a.bf16("vpacked"); auto mask = a.u16("mask"); auto off = a.u32("tok_off");
  auto k = a.integer(); auto Kt = a.bf16("K_tail"); auto Vt = a.bf16("V_tail");
  auto n_tail = a.integer(); auto cap = a.integer(); auto idx = a.i32("page_idx");
  auto out = a.f32("out"); auto ws = a.ws(); auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_decode_step_tail(&s, q, bounds, K, v, mask, off, k, Kt, Vt, n_tail, cap, idx, out, ws, nws, st); };)

STC_PY(flush_tail, 17,
  auto s = *a.shape(); auto Kt = a.bf16("K_tail"); auto Vt = a.bf16("V_tail"); auto nf = a.integer();
  auto n_tail = a.integer(); auto cap = a.integer(); auto mode = a.integer();
  auto logits = a.f32("logits"); auto kcount = a.u8("kcount"); auto fixed_k = a.integer();
  auto mask_in = a.u16("mask_in"); auto K = a.bf16("K"); auto bounds = a.bf16("bounds");
  auto mask = a.u16("mask"); auto off = a.u32("tok_off"); auto v = a.bf16("vpacked");
  auto status = a.i32("dev_status"); auto st = a.stream();
  return [=] { return stc_flush_tail(&s, Kt, Vt, nf, n_tail, cap, mode, logits, kcount, fixed_k, mask_in, K, bounds, mask, off, v, status, st); };)

STC_PY(append_tail, 7,
  auto s = *a.shape(); auto k = a.bf16("k_new"); auto v = a.bf16("v_new"); auto Kt = a.bf16("K_tail");
  auto Vt = a.bf16("V_tail"); auto n_tail = a.integer(); auto cap = a.integer(); auto st = a.stream();
  return [=] { return stc_append_tail(&s, k, v, Kt, Vt, n_tail, cap, st); };)

STC_PY(router_logits, 10,
  auto B = a.index(); auto Hkv = a.index(); auto N = a.index(); auto dm = a.index();
  auto G = a.index(); auto h = a.bf16("h"); auto W = a.bf16("W"); auto bias = a.f32("bias");
  auto per = a.integer(); auto logits = a.f32("logits"); auto st = a.stream();
  return [=] { return stc_router_logits(B, Hkv, N, dm, G, h, W, bias, per, logits, st); };)

STC_PY(compact_tokens, 9,
  auto src = a.bf16("src"); auto idx = a.i32("token_idx"); auto dst = a.bf16("dst");
  auto B = a.index(); auto Hkv = a.index(); auto N = a.index(); auto keep = a.index();
  auto D = a.index(); auto status = a.i32("dev_status"); auto st = a.stream();
  return [=] { return stc_compact_tokens(src, idx, dst, B, Hkv, N, keep, D, status, st); };)

STC_PY(rotary, 8,
  a.one_device(); auto x = a.rows("x", 4); auto y = a.rows("y", 4);
  for (int i = 0; i < 4; ++i) a.need(x.size[i] == y.size[i], "y", "has another shape than x");
  auto turns = (double*)a.tensor("turns", kF64); auto nturns = a.bytes() / 8; auto rot = a.integer();
  a.need(!turns || (int64_t)nturns * 2 == rot, "turns", "must have rot_dim/2 elements");
  auto layout = a.integer(); auto pos = (int32_t*)a.sized("pos", x.size[0] * x.size[2], at::kInt);
  auto pos0 = a.integer(); auto amp = a.real(); auto st = a.stream();
  return [=] { return stc_rotary(x.size[0], x.size[1], x.size[2], x.size[3], rot, layout, turns, amp, pos, pos0, x.p, x.stride, y.p, y.stride, st); };)

STC_PY(rotary_append, 17,
  auto s = *a.shape(); a.one_device();
  auto q = a.rows("q", 3); auto k = a.rows("k_new", 3); auto v = a.rows("v_new", 3);
  const auto heads = [&](const Args::Rows& r, const char* name, int32_t H) {
    a.need(r.size[0] == s.B && r.size[1] == H && r.size[2] == s.D, name, "has another shape");
    a.need(H == 1 || r.stride[1] == s.D, name, "must have contiguous heads");
  };
  heads(q, "q", s.Hq); heads(k, "k_new", s.Hkv); heads(v, "v_new", s.Hkv);
  const int64_t streams = (int64_t)s.B * s.Hkv * s.D;
  auto qo = a.sized("q_out", (int64_t)s.B * s.Hq * s.D, kBf16);
  auto Kt = a.bf16("K_tail"); auto nk = a.bytes(); auto Vt = a.bf16("V_tail"); auto nv = a.bytes();
  auto n = (int32_t*)a.sized("n_tail", s.B, at::kInt); auto cap = a.integer();
  a.need(nk == (size_t)streams * cap * 2 && nv == nk, "K_tail, V_tail", "must be [B, Hkv, tail_cap, D]");
  auto turns = (double*)a.tensor("turns", kF64); auto nturns = a.bytes() / 8; auto rot = a.integer();
  a.need(!turns || (int64_t)nturns * 2 == rot, "turns", "must have rot_dim/2 elements");
  auto layout = a.integer(); auto amp = a.real(); auto pos = (int32_t*)a.sized("pos", s.B, at::kInt);
  auto pos0 = a.integer(); auto n_out = (int32_t*)a.sized("n_out", s.B, at::kInt);
  auto status = a.i32("dev_status"); auto st = a.stream();
  const int64_t qs = s.B > 1 ? q.stride[0] : (int64_t)s.Hq * s.D;
  return [=] { return stc_rotary_append(&s, q.p, qs, k.p, k.stride[0], v.p, v.stride[0], qo, Kt, Vt, n, n_out, cap, rot, layout, turns, amp, pos, pos0, status, st); };)

STC_PY(decode_attention_shared, 14,
  auto s = *a.shape(); a.one_device();
  const int64_t Nc = s.N_cap ? s.N_cap : s.N; const int64_t gd = s.G > 0 ? s.D / s.G : 0;
  const int64_t n_q = (int64_t)s.B * s.Hq * s.D;
  auto q = a.sized("q", n_q, kBf16); auto K = a.sized("K", s.Hkv * Nc * s.D, kBf16);
  auto v = a.sized("vpacked", s.Hkv * s.v_cap_groups * gd, kBf16);
  auto mask = (uint16_t*)a.sized("mask", s.Hkv * Nc, at::kShort, at::kUInt16);
  auto off = (uint32_t*)a.sized("tok_off", s.Hkv * (Nc + 1), at::kInt, at::kUInt32);
  auto idx = a.i32("page_idx"); auto nidx = a.bytes() / 4; auto k = a.integer();
  a.need(!idx || (int64_t)nidx == (int64_t)s.Hkv * k, "page_idx", "must be [Hkv, k_pages]");
  auto Kt = a.bf16("K_tail"); auto nk = a.bytes(); auto Vt = a.bf16("V_tail"); auto nv = a.bytes();
  auto n = (int32_t*)a.sized("n_tail", s.B, at::kInt); auto cap = a.integer();
  const size_t tails = cap > 0 ? (size_t)s.B * s.Hkv * cap * s.D * 2 : 0;
  a.need(cap <= 0 || ((!Kt || nk == tails) && (!Vt || nv == tails)), "K_tail, V_tail", "must be [B, Hkv, tail_cap, D]");
  auto out = a.sized("out", n_q, kF32, kBf16);
  auto type = out && a.bytes() == (size_t)n_q * 2 ? STC_OUT_BF16 : STC_OUT_F32;
  auto ws = a.ws(); auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_decode_attention_shared(&s, q, K, v, mask, off, idx, k, Kt, Vt, n, cap, type, out, ws, nws, st); };)

// Sets of visible nodes: [B, T], or [T] for all sequences.
struct Tree {
  const uint64_t* p;
  int per_batch;
};
static Tree tree_of(Args& a, int32_t B, int64_t T) {
  const auto p = (const uint64_t*)a.tensor("tree", at::kLong, at::kUInt64);
  const int64_t n = a.bytes() / 8;
  a.need(!p || n == T || n == (int64_t)B * T, "tree", "must be [T] or [B, T]");
  return {p, p && n != T};
}

STC_PY(rotary_append_tree, 19,
  auto s = *a.shape(); a.one_device();
  auto q = a.rows("q", 4); auto k = a.rows("k_new", 4); auto v = a.rows("v_new", 4);
  const int64_t T = q.size[1];
  const auto heads = [&](const Args::Rows& r, const char* name, int32_t H) {
    a.need(r.size[0] == s.B && r.size[1] == T && r.size[2] == H && r.size[3] == s.D, name, "has another shape");
    a.need(H == 1 || r.stride[2] == s.D, name, "must have contiguous heads");
  };
  heads(q, "q", s.Hq); heads(k, "k_new", s.Hkv); heads(v, "v_new", s.Hkv);
  const int64_t streams = (int64_t)s.B * s.Hkv * s.D;
  auto qo = a.sized("q_out", (int64_t)s.B * T * s.Hq * s.D, kBf16);
  auto Kt = a.bf16("K_tail"); auto nk = a.bytes(); auto Vt = a.bf16("V_tail"); auto nv = a.bytes();
  auto n = (int32_t*)a.sized("n_tail", s.B, at::kInt); auto cap = a.integer();
  a.need(nk == (size_t)streams * cap * 2 && nv == nk, "K_tail, V_tail", "must be [B, Hkv, tail_cap, D]");
  auto turns = (double*)a.tensor("turns", kF64); auto nturns = a.bytes() / 8; auto rot = a.integer();
  a.need(!turns || (int64_t)nturns * 2 == rot, "turns", "must have rot_dim/2 elements");
  auto layout = a.integer(); auto tree = tree_of(a, s.B, T);
  auto nd = (int32_t*)a.sized("n_draft", s.B, at::kInt); auto amp = a.real();
  auto pos = (int32_t*)a.sized("pos", s.B * T, at::kInt); auto pos0 = a.integer();
  auto have = (int32_t*)a.sized("n_have", s.B, at::kInt);
  auto status = (int32_t*)a.sized("dev_status", 1, at::kInt); auto st = a.stream();
  // strides of dimensions of one element: as if rows followed each other
  if (T == 1) q.stride[1] = (int64_t)s.Hq * s.D;
  if (s.B == 1) q.stride[0] = T * s.Hq * s.D;
  return [=] { return stc_rotary_append_drafts(&s, (int)T, q.p, q.stride, k.p, k.stride, v.p, v.stride, qo, Kt, Vt, n, nd, cap, tree.p, tree.per_batch, rot, layout, turns, amp, pos, pos0, have, status, st); };)

STC_PY(decode_attention_tree, 18,
  auto s = *a.shape(); a.one_device(); auto P = a.integer(); auto T = a.integer();
  const int64_t Nc = s.N_cap ? s.N_cap : s.N; const int64_t gd = s.G > 0 ? s.D / s.G : 0;
  const int64_t n_q = (int64_t)s.B * T * s.Hq * s.D; const int64_t heads = (int64_t)P * s.Hkv;
  a.need(T >= 1 && T <= 64, "q", "must have 1 to 64 nodes");
  a.need(P == 1 || P == s.B, "n_prefix", "must be 1 or B");
  auto q = a.sized("q", n_q, kBf16); auto K = a.sized("K", heads * Nc * s.D, kBf16);
  auto v = a.sized("vpacked", heads * s.v_cap_groups * gd, kBf16);
  auto mask = (uint16_t*)a.sized("mask", heads * Nc, at::kShort, at::kUInt16);
  auto off = (uint32_t*)a.sized("tok_off", heads * (Nc + 1), at::kInt, at::kUInt32);
  auto idx = a.i32("page_idx"); auto nidx = a.bytes() / 4; auto k = a.integer();
  a.need(!idx || (int64_t)nidx == heads * k, "page_idx", "must be [n_prefix, Hkv, k_pages]");
  auto Kt = a.bf16("K_tail"); auto nk = a.bytes(); auto Vt = a.bf16("V_tail"); auto nv = a.bytes();
  auto n = (int32_t*)a.sized("n_tail", s.B, at::kInt); auto cap = a.integer();
  a.need(nk == (size_t)s.B * s.Hkv * cap * s.D * 2 && nv == nk, "K_tail, V_tail", "must be [B, Hkv, tail_cap, D]");
  auto tree = tree_of(a, s.B, T); auto nd = (int32_t*)a.sized("n_draft", s.B, at::kInt);
  auto out = a.sized("out", n_q, kF32, kBf16);
  auto type = out && a.bytes() == (size_t)n_q * 2 ? STC_OUT_BF16 : STC_OUT_F32;
  auto ws = a.ws(); auto nws = a.bytes(); auto st = a.stream();
  return [=] { return stc_decode_attention_tree(&s, T, P, q, K, v, mask, off, idx, k, Kt, Vt, n, nd, cap, tree.p, tree.per_batch, type, out, ws, nws, st); };)

// The tails of all layers: K_tails, V_tails, n_tails, n_outs
struct LayerTails {
  int n;
  void **K, **V;
  const int32_t* const* len;
  int32_t* const* out;
};
static LayerTails layer_tails(Args& a, const stc_shape_t& s, int cap) {
  const int64_t rows = (int64_t)s.B * s.Hkv * cap * s.D;
  auto& t = a.tails;
  a.many(t[0], "K_tails", rows, kBf16); a.many(t[1], "V_tails", rows, kBf16);
  a.many(t[2], "n_tails", s.B, at::kInt); a.many(t[3], "n_outs", s.B, at::kInt);
  a.need(t[1].n == t[0].n && t[2].n == t[0].n && t[3].n == t[0].n, "K_tails, V_tails, n_tails, n_outs", "must be as many");
  return {t[0].n, t[0].p, t[1].p, (const int32_t* const*)t[2].p, (int32_t* const*)t[3].p};
}

STC_PY(accept_tail, 9,
  auto s = *a.shape(); a.one_device(); auto T = a.integer(); auto cap = a.integer();
  auto t = layer_tails(a, s, cap);
  auto keep = (const uint64_t*)a.sized("keep", s.B, at::kLong, at::kUInt64);
  auto nd = (const int32_t*)a.sized("n_draft", s.B, at::kInt); auto st = a.stream();
  return [=] { return stc_accept_drafts(&s, T, t.n, t.K, t.V, t.len, t.out, cap, keep, nd, st); };)

STC_PY(fork_tail, 9,
  auto s = *a.shape(); a.one_device(); auto cap = a.integer();
  auto t = layer_tails(a, s, cap);
  auto src = (const int32_t*)a.sized("src", s.B, at::kInt); auto keep = (const int32_t*)a.sized("n_keep", s.B, at::kInt);
  auto status = (int32_t*)a.sized("dev_status", 1, at::kInt); auto st = a.stream();
  return [=] { return stc_fork_tail(&s, t.n, t.K, t.V, t.len, t.out, cap, src, keep, status, st); };)

PyMethodDef methods[] = {
#define STC_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
    STC_METHOD(build_page_bounds), STC_METHOD(route_and_pack_values), STC_METHOD(select_pages),
    STC_METHOD(select_pages_per_head), STC_METHOD(score_pages), STC_METHOD(decode_attention),
    STC_METHOD(decode_attention_per_head), STC_METHOD(decode_attention_tail),
    STC_METHOD(decode_attention_union), STC_METHOD(union_pages), STC_METHOD(decode_step),
    STC_METHOD(decode_step_static), STC_METHOD(decode_step_tail), STC_METHOD(flush_tail),
    STC_METHOD(append_tail), STC_METHOD(router_logits), STC_METHOD(compact_tokens),
    STC_METHOD(rotary), STC_METHOD(rotary_append), STC_METHOD(decode_attention_shared),
    STC_METHOD(rotary_append_tree), STC_METHOD(decode_attention_tree), STC_METHOD(accept_tail),
    STC_METHOD(fork_tail),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The module takes what it needs of Python from its package when it is loaded.
PyMODINIT_FUNC PyInit__binding() {
  PyObject* torch_c = PyImport_ImportModule("torch._C");
  PyObject* pkg = PyImport_ImportModule("paper_2604_21335_amd");
  if (torch_c && pkg) {
    g_error = PyObject_GetAttrString(pkg, "StcError");
    g_shape = PyObject_GetAttrString(pkg, "stc_shape_t");
    g_any_stream = PyObject_GetAttrString(pkg, "_current_stream");
    if (g_error && g_shape && g_any_stream) {
      g_device = PyObject_GetAttrString(torch_c, "_cuda_getDevice");
      if (g_device) g_raw_stream = PyObject_GetAttrString(torch_c, "_cuda_getCurrentRawStream");
      PyErr_Clear();
    }
  }
  Py_XDECREF(torch_c);
  Py_XDECREF(pkg);
  return g_error && g_shape && g_any_stream ? PyModule_Create(&module_def) : nullptr;
}
