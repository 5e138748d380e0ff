// The common case of the Python entry points around training and serving, without the interpreter:
// every tensor an ordinary one of the right kind, outputs and workspace allocated here, the current
// stream.  Each function checks its tensors, allocates, calls the C ABI and returns the outputs as a
// tuple; or None, having done nothing, where anything is not as the common case has it -- the caller's
// Python code then does the call or names what is wrong; or the status, an int, where the C call
// refuses.  Tensors are looked at and made through torch's C++ interface: GB300 host, us a call, by their
// Python attributes / here: backward of 128 rows 16.5 / 9, norm and rotation 11.6 / 5.4, into a
// cache 9.1 / 3.8, its gradients 17.0 / 8.
// It does not link against the library: set_up() gets the C functions' addresses.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <initializer_list>

#include "../../include/loom_attn.h"

namespace {

struct Functions {
  decltype(&loom_attn_bwd) attn_bwd;
  decltype(&loom_attn_bwd_workspace_bytes) attn_bwd_bytes;
  decltype(&loom_attn_bwd_varlen) attn_bwd_varlen;
  decltype(&loom_attn_bwd_varlen_workspace_bytes) attn_bwd_varlen_bytes;
  decltype(&loom_qkv_norm_rope) norm_rope;
  decltype(&loom_qkv_norm_rope_cache) norm_rope_cache;
  decltype(&loom_qkv_norm_rope_bwd) norm_rope_bwd;
  decltype(&loom_qkv_norm_rope_bwd_workspace_bytes) norm_rope_bwd_bytes;
  decltype(&loom_qkv_norm_rope_axes) norm_rope_axes;
  decltype(&loom_qkv_norm_rope_axes_cache) norm_rope_axes_cache;
  decltype(&loom_qkv_norm_rope_axes_bwd) norm_rope_axes_bwd;
  decltype(&loom_attn_chunk_paged) chunk;
  decltype(&loom_attn_chunk_paged_workspace_bytes) chunk_bytes;
  decltype(&loom_paged_plan) plan;
} F = {};

struct Ref {  // owned
  PyObject* p = nullptr;
  explicit Ref(PyObject* q = nullptr) : p(q) {}
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
  ~Ref() { Py_XDECREF(p); }
  PyObject* release() {
    PyObject* q = p;
    p = nullptr;
    return q;
  }
};

constexpr at::ScalarType kBf16 = at::kBFloat16, kF32 = at::kFloat, kI32 = at::kInt;

struct Tensor {
  const at::Tensor* t = nullptr;
  PyObject* obj = nullptr;
  void* ptr = nullptr;
  long long size[4] = {};
  int dims = 0;
};

// t as a CUDA tensor of this type with at most four dimensions, contiguous or (strided) with contiguous
// rows; false if it is anything else.
bool view(PyObject* obj, at::ScalarType type, Tensor* out, bool strided = false) {
  if (!THPVariable_CheckExact(obj)) return false;  // torch.Tensor or Parameter: no subclass
  const at::Tensor& t = THPVariable_Unpack(obj);
  if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != type || t.dim() > 4 || !t.has_storage() ||
      (!strided && !t.is_contiguous()))
    return false;
  out->dims = static_cast<int>(t.dim());
  for (int i = 0; i < out->dims; ++i) out->size[i] = t.size(i);
  out->ptr = t.data_ptr();
  out->t = &t;
  out->obj = obj;
  return true;
}
bool same(const Tensor& a, const Tensor& b) {
  if (a.dims != b.dims) return false;
  for (int i = 0; i < a.dims; ++i)
    if (a.size[i] != b.size[i]) return false;
  return true;
}
// Every size of the call fits the C ABI's ints.
bool small(const Tensor& a) {
  for (int i = 0; i < a.dims; ++i)
    if (a.size[i] < 0 || a.size[i] > 0x7fffffffLL) return false;
  return true;
}

// The others (those that there are) are on the first's device.
bool together(const Tensor& first, std::initializer_list<const Tensor*> others) {
  for (const Tensor* t : others)
    if (t->t && t->t->get_device() != first.t->get_device()) return false;
  return true;
}

// The device whose current stream the call takes, where outputs may be allocated without torch's
// dispatcher: no mode that would miss them, no deterministic fill, the current device.  -1 otherwise.
long long device_of(const Tensor& t) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(t.obj)) != THPVariableClass) return -1;
  if (c10::impl::TorchDispatchModeTLS::stack_len() != 0 || at::impl::PythonTorchFunctionTLS::stack_len() != 0 ||
      at::globalContext().deterministicAlgorithms())
    return -1;
  const long long d = t.t->get_device();
  return d == c10::cuda::current_device() ? d : -1;
}
void* stream_of(long long device) {
  return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
}

// A new contiguous tensor (c10::Error: out of memory).
PyObject* make(long long device, int dims, const long long* size, at::ScalarType type, void** ptr) {
  int64_t n[4];
  for (int i = 0; i < dims; ++i) n[i] = size[i];
  const at::Device cuda(at::kCUDA, static_cast<c10::DeviceIndex>(device));
  at::Tensor t(at::detail::empty_cuda(at::IntArrayRef(n, static_cast<size_t>(dims)), type, cuda, std::nullopt));
  *ptr = t.data_ptr();
  return THPVariable_Wrap(std::move(t));
}
PyObject* make_like(long long device, const Tensor& t, at::ScalarType type, void** ptr) {
  return make(device, t.dims, t.size, type, ptr);
}
// Scratch on the current device for a call on its current stream (no tensor: nobody sees it).
c10::DataPtr scratch(size_t bytes) { return c10::cuda::CUDACachingAllocator::get()->allocate(bytes < 16 ? 16 : bytes); }

PyObject* status(loom_status st) { return PyLong_FromLong(st); }

bool as_float(PyObject* o, float* out) {
  const double d = PyFloat_AsDouble(o);
  if (d == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *out = static_cast<float>(d);
  return true;
}
bool as_int(PyObject* o, long long* out) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *out = PyLong_AsLongLongAndOverflow(o, &over);
  return !over && *out >= 0 && *out <= 0x7fffffffLL;
}

// attn_bwd(do, q, k, v, o, lse, dlse, causal, scale)
// attn_bwd_varlen(do, q, k, v, o, lse, dlse, causal, scale, cu_seqlens_q, cu_seqlens_k, max_q, max_k)
PyObject* bwd(PyObject* const* a, bool varlen) {
  Tensor d, q, k, v, o, lse, dlse, cq, ck;
  const int dims = varlen ? 3 : 4, hd = 1, sd = varlen ? 0 : 2;  // the axes of heads and of rows
  constexpr at::ScalarType bf16 = kBf16;
  if (!view(a[1], bf16, &q) || q.dims != dims || !view(a[0], bf16, &d) || !same(d, q) || !view(a[4], bf16, &o) || !same(o, q) ||
      !view(a[2], bf16, &k) || k.dims != dims || !view(a[3], bf16, &v) || !same(v, k) || !small(q) || !small(k))
    Py_RETURN_NONE;
  const long long D = q.size[dims - 1], Hq = q.size[hd], Hkv = k.size[hd], Sq = q.size[sd], Skv = k.size[sd];
  long long B = varlen ? 0 : q.size[0], max_q = 0, max_k = 0;
  if (k.size[dims - 1] != D || (!varlen && k.size[0] != B)) Py_RETURN_NONE;
  if (!view(a[5], kF32, &lse)) Py_RETURN_NONE;
  if (varlen ? lse.dims != 2 || lse.size[0] != Hq || lse.size[1] != Sq
             : lse.dims != 3 || lse.size[0] != B || lse.size[1] != Hq || lse.size[2] != Sq)
    Py_RETURN_NONE;
  if (a[6] != Py_None && (!view(a[6], kF32, &dlse) || !same(dlse, lse))) Py_RETURN_NONE;
  const int causal = PyObject_IsTrue(a[7]);
  if (causal < 0) return nullptr;
  float scale = 0.f;
  if (a[8] == Py_None)
    scale = D == 64 ? 0.125f : 0.088388347648318440550f;  // D^-1/2 (other D are refused)
  else if (!as_float(a[8], &scale))
    Py_RETURN_NONE;
  if (varlen) {
    if (!view(a[9], kI32, &cq) || !view(a[10], kI32, &ck) || cq.dims != 1 || ck.dims != 1 || cq.size[0] != ck.size[0] ||
        cq.size[0] < 2 || !small(cq) || !as_int(a[11], &max_q) || !as_int(a[12], &max_k))
      Py_RETURN_NONE;
    B = cq.size[0] - 1;
  }
  const long long dev = device_of(q);
  if (dev < 0 || !together(q, {&d, &k, &v, &o, &lse, &dlse, &cq, &ck})) Py_RETURN_NONE;
  const int iB = static_cast<int>(B), iHq = static_cast<int>(Hq), iHkv = static_cast<int>(Hkv), iSq = static_cast<int>(Sq),
            iSkv = static_cast<int>(Skv), iD = static_cast<int>(D);
  const size_t need = varlen ? F.attn_bwd_varlen_bytes(iB, iHq, iHkv, iSq, iSkv, iD) : F.attn_bwd_bytes(iB, iHq, iHkv, iSq, iSkv, iD);
  void *dqp, *dkp, *dvp;
  Ref dq(make_like(dev, q, bf16, &dqp));
  if (!dq.p) return nullptr;
  Ref dk(make_like(dev, k, bf16, &dkp));
  if (!dk.p) return nullptr;
  Ref dv(make_like(dev, v, bf16, &dvp));
  if (!dv.p) return nullptr;
  const c10::DataPtr ws = scratch(need);
  void* s = stream_of(dev);
  const float *l = static_cast<const float*>(lse.ptr), *dl = static_cast<const float*>(dlse.ptr);
  const loom_status st =
      varlen ? F.attn_bwd_varlen(d.ptr, q.ptr, k.ptr, v.ptr, o.ptr, l, dl, dqp, dkp, dvp, static_cast<const int32_t*>(cq.ptr),
                                 static_cast<const int32_t*>(ck.ptr), ws.get(), need, iB, iHq, iHkv, iSq, iSkv,
                                 static_cast<int>(max_q), static_cast<int>(max_k), iD, causal, scale, s)
             : F.attn_bwd(d.ptr, q.ptr, k.ptr, v.ptr, o.ptr, l, dl, dqp, dkp, dvp, ws.get(), need, iB, iHq, iHkv, iSq, iSkv, iD, causal,
                          scale, s);
  if (st != LOOM_OK) return status(st);
  return PyTuple_Pack(3, dq.p, dk.p, dv.p);
}
PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9) Py_RETURN_NONE;
  return bwd(a, false);
}
PyObject* attn_bwd_varlen(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 13) Py_RETURN_NONE;
  return bwd(a, true);
}

constexpr int kMaxPairs = 64;  // pairs of a head of 128 values

// What the norm-and-rotation calls share: qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps; and last
// pair_axis (None, or a tuple of ints).
struct Norm {
  Tensor x, qw, kw, cos, sin, pos;
  long long T, D, row;
  int type, P, R, interleaved, axes;
  int axis[kMaxPairs];
  float eps;
  const int32_t* positions() const { return static_cast<const int32_t*>(pos.ptr); }
  // the tables have the rows that no positions given imply
  bool tables_reach(long long S) const { return pos.t || (S > 0 ? S : T) <= P; }
};
bool norm_args(PyObject* const* a, long long heads, PyObject* pair_axis, Norm* m) {
  if (!view(a[0], kBf16, &m->x, true) || m->x.dims != 2 || !small(m->x)) return false;
  const bool f32 = view(a[1], kF32, &m->qw);
  if ((!f32 && !view(a[1], kBf16, &m->qw)) || m->qw.dims != 1) return false;
  if (!view(a[2], f32 ? kF32 : kBf16, &m->kw) || !same(m->kw, m->qw)) return false;
  if (!view(a[3], kF32, &m->cos) || m->cos.dims != 2 || !view(a[4], kF32, &m->sin) || !same(m->sin, m->cos) || !small(m->cos))
    return false;
  m->T = m->x.size[0];
  m->D = m->qw.size[0];
  if (m->D <= 0 || m->D > 1024 || heads <= 0 || heads > 0x100000 || m->x.size[1] != heads * m->D) return false;
  m->row = m->T > 1 ? m->x.t->stride(0) : m->x.size[1];
  if (m->x.t->stride(1) != 1) return false;
  m->axes = 0;
  if (pair_axis != Py_None) {
    if (!PyTuple_CheckExact(pair_axis) || PyTuple_GET_SIZE(pair_axis) != m->cos.size[1] || PyTuple_GET_SIZE(pair_axis) > kMaxPairs ||
        !view(a[5], kI32, &m->pos) || m->pos.dims != 2 || m->pos.size[1] != m->T || m->pos.size[0] < 1 || m->pos.size[0] > 4)
      return false;
    m->axes = static_cast<int>(m->pos.size[0]);
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(pair_axis); ++i) {
      long long x;
      if (!as_int(PyTuple_GET_ITEM(pair_axis, i), &x) || x >= m->axes) return false;
      m->axis[i] = static_cast<int>(x);
    }
  } else if (a[5] != Py_None && (!view(a[5], kI32, &m->pos) || m->pos.dims != 1 || m->pos.size[0] != m->T)) {
    return false;
  }
  if (!together(m->x, {&m->qw, &m->kw, &m->cos, &m->sin, &m->pos})) return false;
  m->type = f32 ? LOOM_FP32 : LOOM_BF16;
  m->P = static_cast<int>(m->cos.size[0]);
  m->R = m->cos.size[1] > 1024 ? 0 : static_cast<int>(2 * m->cos.size[1]);
  m->interleaved = PyObject_IsTrue(a[6]);
  if (m->interleaved < 0) {  // (the Python code meets it again)
    PyErr_Clear();
    return false;
  }
  return as_float(a[7], &m->eps);
}

// norm_rope(qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps, num_heads, num_kv_heads, seq_len, pair_axis)
PyObject* norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long Hq, Hkv, S;
  Norm m;
  if (n != 12 || !as_int(a[8], &Hq) || !as_int(a[9], &Hkv) || !as_int(a[10], &S) || Hq <= 0 || Hkv <= 0 ||
      !norm_args(a, Hq + 2 * Hkv, a[11], &m) || (S > 0 && m.T % S) || !m.tables_reach(S))
    Py_RETURN_NONE;
  const long long dev = device_of(m.x);
  if (dev < 0) Py_RETURN_NONE;
  const long long qs[4] = {S ? m.T / S : m.T, Hq, S ? S : m.D, m.D}, ks[4] = {qs[0], Hkv, qs[2], m.D};
  const int dims = S ? 4 : 3;
  void *qp, *kp, *vp;
  Ref q(make(dev, dims, qs, kBf16, &qp));
  if (!q.p) return nullptr;
  Ref k(make(dev, dims, ks, kBf16, &kp));
  if (!k.p) return nullptr;
  Ref v(make(dev, dims, ks, kBf16, &vp));
  if (!v.p) return nullptr;
  const float *cos = static_cast<const float*>(m.cos.ptr), *sin = static_cast<const float*>(m.sin.ptr);
  const int T = static_cast<int>(m.T), iS = static_cast<int>(S), iHq = static_cast<int>(Hq), iHkv = static_cast<int>(Hkv),
            D = static_cast<int>(m.D);
  const loom_status st =
      m.axes ? F.norm_rope_axes(m.x.ptr, m.row, m.qw.ptr, m.kw.ptr, m.type, cos, sin, m.P, m.R, m.interleaved, m.positions(), m.T,
                                m.axes, m.axis, qp, kp, vp, T, iS, iHq, iHkv, D, m.eps, stream_of(dev))
             : F.norm_rope(m.x.ptr, m.row, m.qw.ptr, m.kw.ptr, m.type, cos, sin, m.P, m.R, m.interleaved, m.positions(), qp, kp, vp,
                           T, iS, iHq, iHkv, D, m.eps, stream_of(dev));
  if (st != LOOM_OK) return status(st);
  return PyTuple_Pack(3, q.p, k.p, v.p);
}

// norm_rope_cache(qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps, num_heads, slots, k_cache, v_cache,
// head_major, pair_axis): (q,)
PyObject* norm_rope_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  long long Hq;
  Norm m;
  Tensor slots, kc, vc;
  if (n != 14 || !as_int(a[8], &Hq) || Hq <= 0 || !view(a[10], kBf16, &kc) || kc.dims != 4 || !small(kc) ||
      !view(a[11], kBf16, &vc) || !same(kc, vc) || a[5] == Py_None)
    Py_RETURN_NONE;
  const int hnd = a[12] == Py_True;
  const long long Hkv = kc.size[hnd ? 1 : 2], page = kc.size[hnd ? 2 : 1];
  if (!norm_args(a, Hq + 2 * Hkv, a[13], &m) || kc.size[3] != m.D || !view(a[9], kI32, &slots) || slots.dims != 1 ||
      slots.size[0] != m.T || !together(m.x, {&slots, &kc, &vc}))
    Py_RETURN_NONE;
  const long long dev = device_of(m.x);
  if (dev < 0) Py_RETURN_NONE;
  const long long qs[3] = {m.T, Hq, m.D};
  void* qp;
  Ref q(make(dev, 3, qs, kBf16, &qp));
  if (!q.p) return nullptr;
  const float *cos = static_cast<const float*>(m.cos.ptr), *sin = static_cast<const float*>(m.sin.ptr);
  const int32_t* sp = static_cast<const int32_t*>(slots.ptr);
  const int T = static_cast<int>(m.T), iHq = static_cast<int>(Hq), iHkv = static_cast<int>(Hkv), D = static_cast<int>(m.D),
            pages = static_cast<int>(kc.size[0]), rows = static_cast<int>(page);
  const loom_status st =
      m.axes ? F.norm_rope_axes_cache(m.x.ptr, m.row, m.qw.ptr, m.kw.ptr, m.type, cos, sin, m.P, m.R, m.interleaved, m.positions(),
                                      m.T, m.axes, m.axis, sp, qp, kc.ptr, vc.ptr, pages, rows, hnd, T, iHq, iHkv, D, m.eps,
                                      stream_of(dev))
             : F.norm_rope_cache(m.x.ptr, m.row, m.qw.ptr, m.kw.ptr, m.type, cos, sin, m.P, m.R, m.interleaved, m.positions(), sp, qp,
                                 kc.ptr, vc.ptr, pages, rows, hnd, T, iHq, iHkv, D, m.eps, stream_of(dev));
  if (st != LOOM_OK) return status(st);
  return PyTuple_Pack(1, q.p);
}

// norm_rope_bwd(qkv, q_weight, k_weight, cos, sin, positions, interleaved, eps, dq, dk, dv, pair_axis)
PyObject* norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Norm m;
  Tensor dq, dk, dv;
  if (n != 12 || !view(a[8], kBf16, &dq) || dq.dims < 3 || !view(a[9], kBf16, &dk) || dk.dims != dq.dims ||
      !view(a[10], kBf16, &dv) || !same(dv, dk) || !small(dq) || !small(dk))
    Py_RETURN_NONE;
  const long long Hq = dq.size[1], Hkv = dk.size[1], S = dq.dims == 4 ? dq.size[2] : 0;
  if (!norm_args(a, Hq + 2 * Hkv, a[11], &m) || dq.size[0] != dk.size[0] || dq.size[2] != dk.size[2] || dq.size[dq.dims - 1] != m.D ||
      dk.size[dk.dims - 1] != m.D || (S ? dq.size[0] * S : dq.size[0]) != m.T || (dq.dims == 4 && S == 0) ||
      !m.tables_reach(S) || !together(m.x, {&dq, &dk, &dv}))
    Py_RETURN_NONE;
  const long long dev = device_of(m.x);
  if (dev < 0) Py_RETURN_NONE;
  const size_t need = F.norm_rope_bwd_bytes(static_cast<int>(m.D));
  void *xp, *qp, *kp;
  Ref dx(make(dev, 2, m.x.size, kBf16, &xp));
  if (!dx.p) return nullptr;
  Ref dqw(make(dev, 1, m.qw.size, kF32, &qp));
  if (!dqw.p) return nullptr;
  Ref dkw(make(dev, 1, m.qw.size, kF32, &kp));
  if (!dkw.p) return nullptr;
  const c10::DataPtr ws = scratch(need);
  const float *cos = static_cast<const float*>(m.cos.ptr), *sin = static_cast<const float*>(m.sin.ptr);
  float *qg = static_cast<float*>(qp), *kg = static_cast<float*>(kp);
  const int T = static_cast<int>(m.T), iS = static_cast<int>(S), iHq = static_cast<int>(Hq), iHkv = static_cast<int>(Hkv),
            D = static_cast<int>(m.D);
  const loom_status st =
      m.axes ? F.norm_rope_axes_bwd(dq.ptr, dk.ptr, dv.ptr, m.x.ptr, m.row, m.qw.ptr, m.kw.ptr, m.type, cos, sin, m.P, m.R,
                                    m.interleaved, m.positions(), m.T, m.axes, m.axis, xp, m.x.size[1], qg, kg, ws.get(), need, T, iS,
                                    iHq, iHkv, D, m.eps, stream_of(dev))
             : F.norm_rope_bwd(dq.ptr, dk.ptr, dv.ptr, m.x.ptr, m.row, m.qw.ptr, m.kw.ptr, m.type, cos, sin, m.P, m.R, m.interleaved,
                               m.positions(), xp, m.x.size[1], qg, kg, ws.get(), need, T, iS, iHq, iHkv, D, m.eps, stream_of(dev));
  if (st != LOOM_OK) return status(st);
  return PyTuple_Pack(3, dx.p, dqw.p, dkw.p);
}

// chunk(q, k_cache, v_cache, block_table, cu_seqlens_q, seqlens_k, causal, scale, head_major, with_lse): (o,) or (o, lse)
PyObject* chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor q, kc, vc, table, cu, lens;
  if (n != 10 || !view(a[0], kBf16, &q) || q.dims != 3 || !view(a[1], kBf16, &kc) || kc.dims != 4 || !view(a[2], kBf16, &vc) ||
      !same(kc, vc) || !view(a[3], kI32, &table) || table.dims != 2 || !view(a[4], kI32, &cu) || cu.dims != 1 ||
      !view(a[5], kI32, &lens) || lens.dims != 1 || !small(q) || !small(kc) || !small(table))
    Py_RETURN_NONE;
  const int hnd = a[8] == Py_True;
  const long long T = q.size[0], Hq = q.size[1], D = q.size[2], Hkv = kc.size[hnd ? 1 : 2], page = kc.size[hnd ? 2 : 1],
                  B = table.size[0];
  if (kc.size[3] != D || cu.size[0] != B + 1 || lens.size[0] != B) Py_RETURN_NONE;
  const int causal = PyObject_IsTrue(a[6]);
  if (causal < 0) return nullptr;
  float scale = 0.f;
  if (a[7] == Py_None)
    scale = D == 64 ? 0.125f : 0.088388347648318440550f;  // D^-1/2 (other D are refused)
  else if (!as_float(a[7], &scale))
    Py_RETURN_NONE;
  const long long dev = device_of(q);
  if (dev < 0 || !together(q, {&kc, &vc, &table, &cu, &lens})) Py_RETURN_NONE;
  const int iB = static_cast<int>(B), iHq = static_cast<int>(Hq), iHkv = static_cast<int>(Hkv), iT = static_cast<int>(T),
            iD = static_cast<int>(D);
  const size_t need = F.chunk_bytes(iB, iHq, iHkv, iT, iD);
  const bool with_lse = a[9] == Py_True;
  const long long ls[2] = {Hq, T};
  void *op, *lp = nullptr;
  Ref o(make_like(dev, q, kBf16, &op)), lse;
  if (!o.p) return nullptr;
  if (with_lse && !(lse.p = make(dev, 2, ls, kF32, &lp))) return nullptr;
  const c10::DataPtr ws = scratch(need);
  const loom_status st = F.chunk(q.ptr, kc.ptr, vc.ptr, static_cast<const int32_t*>(table.ptr), static_cast<const int32_t*>(cu.ptr),
                                 static_cast<const int32_t*>(lens.ptr), op, static_cast<float*>(lp), ws.get(), need, iB, iHq, iHkv, iT,
                                 static_cast<int>(kc.size[0]), static_cast<int>(page), static_cast<int>(table.size[1]), hnd, iD,
                                 causal, scale, stream_of(dev));
  if (st != LOOM_OK) return status(st);
  return with_lse ? PyTuple_Pack(2, o.p, lse.p) : PyTuple_Pack(1, o.p);
}

// plan(new_lens, lens, block_table, free_pages, free_count, free_count_out, seqlens_k or None, granted or None, num_tokens,
// page_size): (cu_seqlens, seqlens_k, positions, slots, granted)
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Tensor news, lens, table, list, count, out, seqlens, grants;
  long long T, page;
  if (n != 10 || !view(a[0], kI32, &news) || news.dims != 1 || !view(a[1], kI32, &lens) || !same(lens, news) ||
      !view(a[2], kI32, &table) || table.dims != 2 || table.size[0] != news.size[0] || !view(a[3], kI32, &list) || list.dims != 1 ||
      !view(a[4], kI32, &count) || count.dims != 1 || count.size[0] != 1 || !view(a[5], kI32, &out) || !same(out, count) ||
      (a[6] != Py_None && (!view(a[6], kI32, &seqlens) || !same(seqlens, news))) ||
      (a[7] != Py_None && (!view(a[7], kI32, &grants) || !same(grants, news))) || !as_int(a[8], &T) || !as_int(a[9], &page) ||
      !small(table) || !small(list))
    Py_RETURN_NONE;
  const long long dev = device_of(news), B = news.size[0], B1 = B + 1;
  if (dev < 0 || !together(news, {&lens, &table, &list, &count, &out, &seqlens, &grants})) Py_RETURN_NONE;
  // an output of one number a request: the one given, or a new one
  const auto given_or_new = [&](const Tensor& given, void** ptr) {
    if (!given.t) return make(dev, 1, &B, kI32, ptr);
    Py_INCREF(given.obj);
    *ptr = given.ptr;
    return given.obj;
  };
  void *cp, *sp, *pp, *lp, *gp;
  Ref cu(make(dev, 1, &B1, kI32, &cp));
  if (!cu.p) return nullptr;
  Ref lengths(given_or_new(seqlens, &sp));
  if (!lengths.p) return nullptr;
  Ref positions(make(dev, 1, &T, kI32, &pp));
  if (!positions.p) return nullptr;
  Ref slots(make(dev, 1, &T, kI32, &lp));
  if (!slots.p) return nullptr;
  Ref granted(given_or_new(grants, &gp));
  if (!granted.p) return nullptr;
  const auto i32 = [](void* x) { return static_cast<int32_t*>(x); };
  const loom_status st = F.plan(i32(news.ptr), i32(lens.ptr), i32(table.ptr), i32(list.ptr), i32(count.ptr), i32(out.ptr), i32(cp),
                                i32(sp), i32(pp), i32(lp), i32(gp), static_cast<int>(B), static_cast<int>(T),
                                static_cast<int>(list.size[0]), static_cast<int>(page), static_cast<int>(table.size[1]), stream_of(dev));
  if (st != LOOM_OK) return status(st);
  return PyTuple_Pack(5, cu.p, lengths.p, positions.p, slots.p, granted.p);
}

// set_up((addresses ...)): the C functions.
PyObject* set_up(PyObject*, PyObject* args) {
  PyObject* addresses;
  if (!PyArg_ParseTuple(args, "O!", &PyTuple_Type, &addresses)) return nullptr;
  constexpr int kFunctions = 14;
  if (PyTuple_GET_SIZE(addresses) != kFunctions) {
    PyErr_SetString(PyExc_ValueError, "set_up takes 14 addresses");
    return nullptr;
  }
  void* at[kFunctions];
  for (int i = 0; i < kFunctions; ++i) {
    at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (!at[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address");
      return nullptr;
    }
  }
  F.attn_bwd = reinterpret_cast<decltype(F.attn_bwd)>(at[0]);
  F.attn_bwd_bytes = reinterpret_cast<decltype(F.attn_bwd_bytes)>(at[1]);
  F.attn_bwd_varlen = reinterpret_cast<decltype(F.attn_bwd_varlen)>(at[2]);
  F.attn_bwd_varlen_bytes = reinterpret_cast<decltype(F.attn_bwd_varlen_bytes)>(at[3]);
  F.norm_rope = reinterpret_cast<decltype(F.norm_rope)>(at[4]);
  F.norm_rope_cache = reinterpret_cast<decltype(F.norm_rope_cache)>(at[5]);
  F.norm_rope_bwd = reinterpret_cast<decltype(F.norm_rope_bwd)>(at[6]);
  F.norm_rope_bwd_bytes = reinterpret_cast<decltype(F.norm_rope_bwd_bytes)>(at[7]);
  F.norm_rope_axes = reinterpret_cast<decltype(F.norm_rope_axes)>(at[8]);
  F.norm_rope_axes_cache = reinterpret_cast<decltype(F.norm_rope_axes_cache)>(at[9]);
  F.norm_rope_axes_bwd = reinterpret_cast<decltype(F.norm_rope_axes_bwd)>(at[10]);
  F.chunk = reinterpret_cast<decltype(F.chunk)>(at[11]);
  F.chunk_bytes = reinterpret_cast<decltype(F.chunk_bytes)>(at[12]);
  F.plan = reinterpret_cast<decltype(F.plan)>(at[13]);
  Py_RETURN_NONE;
}

// A METH_FASTCALL function that turns C++ exceptions (torch's, out of memory) into Python's.
template <PyObject* (*Fn)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return Fn(self, a, n);
  END_HANDLE_TH_ERRORS
}
template <PyObject* (*Fn)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<Fn>));
}
PyMethodDef methods[] = {{"set_up", set_up, METH_VARARGS, nullptr},
                         {"attn_bwd", fast<attn_bwd>(), METH_FASTCALL, nullptr},
                         {"attn_bwd_varlen", fast<attn_bwd_varlen>(), METH_FASTCALL, nullptr},
                         {"norm_rope", fast<norm_rope>(), METH_FASTCALL, nullptr},
                         {"norm_rope_cache", fast<norm_rope_cache>(), METH_FASTCALL, nullptr},
                         {"norm_rope_bwd", fast<norm_rope_bwd>(), METH_FASTCALL, nullptr},
                         {"chunk", fast<chunk>(), METH_FASTCALL, nullptr},
                         {"plan", fast<plan>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  PyObject* m = PyModule_Create(&module);
  // built for this torch: the caller compares
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
