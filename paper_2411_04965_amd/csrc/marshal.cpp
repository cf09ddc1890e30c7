// Argument marshalling of the linears, the norm, the cache and the attention a serving loop calls most, as a Python module.  The same calls through ctypes cost 2.4 us
// of host time each beside the launches (3.5 us more where workspace and output are allocated), and small layers are bound
// by the host.  Here plain tensors are unpacked directly: 0.7 us, and 1.5 us for both allocations.
//
// A function takes only what it can pass on as it stands -- exact tensors (no subclass, no torch-function mode), contiguous
// input on a GPU, float32 or bfloat16, plain ints and floats -- and returns None for anything else before it has done
// anything: the caller then goes the general way, which also words the errors.  Otherwise it returns the output, or the
// library's status where that is not 0.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>

#include "../../include/bitlinear.h"

namespace {

// the library's functions, handed over by the binding that loaded it (so two copies of this package in one process keep apart)
struct {
  decltype(&::bitlinear_a4) a4;
  decltype(&::bitlinear_a8_sparse) a8_sparse;
  decltype(&::bitlinear_a4_gate_up) gate_up;
  decltype(&::bitlinear_workspace_bytes) workspace_bytes;
  decltype(&::bitlinear_gate_up_workspace_bytes) gate_up_workspace_bytes;
} lib;
struct {
  decltype(&::rmsnorm_quantize) norm;
  decltype(&::quantize_act_bytes) act_bytes;
  decltype(&::kv_pages_append) append;
  decltype(&::kv_pages_attention) attention;
  decltype(&::kv_pages_attention_workspace_bytes) attention_bytes;
  decltype(&::kv_page_bytes) page_bytes;
} att;

PyObject* get_device = nullptr;    // torch._C._cuda_getDevice
PyObject* get_stream = nullptr;    // torch._C._cuda_getCurrentRawStream
PyObject* str_H = nullptr;
PyObject *str_q = nullptr, *str_scale = nullptr, *str_h = nullptr, *str_rstd = nullptr;

struct NotPlain {};

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) throw NotPlain();
  return THPVariable_Unpack(o);
}

void* pointer(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }

int dtype_code(at::ScalarType t) {
  if (t == at::kFloat) return BL_F32;
  if (t == at::kBFloat16) return BL_BF16;
  throw NotPlain();
}

int64_t integer(PyObject* o) {
  if (!PyLong_CheckExact(o)) throw NotPlain();
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow) throw NotPlain();
  return v;
}

float real(PyObject* o) {
  if (!PyFloat_CheckExact(o)) throw NotPlain();
  return (float)PyFloat_AS_DOUBLE(o);
}

bool truth(PyObject* o) {
  if (!PyBool_Check(o)) throw NotPlain();
  return o == Py_True;
}

// the raw handle of the current stream of the current device
void* stream() {
  PyObject* d = PyObject_CallNoArgs(get_device);
  if (!d) throw std::exception_ptr();
  PyObject* s = PyObject_CallOneArg(get_stream, d);
  Py_DECREF(d);
  if (!s) throw std::exception_ptr();
  void* p = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  if (!p && PyErr_Occurred()) throw std::exception_ptr();
  return p;
}

struct Input {
  const at::Tensor& x;
  int dt;
  int64_t M, K;
  void* p;
  explicit Input(PyObject* o) : x(tensor(o)) {
    if (!x.is_cuda() || x.dim() != 2 || !x.is_contiguous()) throw NotPlain();
    dt = dtype_code(x.scalar_type());
    M = x.size(0);
    K = x.size(1);
    p = x.data_ptr();
  }
};

// a caller's workspace, or one of `bytes` (asked for only then) that lives until this object goes
struct Workspace {
  at::Tensor own;
  void* p = nullptr;
  size_t n = 0;
  template <typename F>
  Workspace(PyObject* o, const Input& in, F bytes) {
    if (o != Py_None) {
      const at::Tensor& t = tensor(o);
      p = t.data_ptr();
      n = (size_t)t.numel();
    } else {
      n = bytes();
      if (n < 16) n = 16;
      own = at::empty({(int64_t)n}, in.x.options().dtype(at::kByte).requires_grad(false));
      p = own.data_ptr();
    }
  }
};

struct Output {
  at::Tensor own;
  PyObject* given = nullptr;
  void* p = nullptr;
  int dt = 0;
  Output(PyObject* out, const Input& in, int64_t N, at::ScalarType type) {
    if (out != Py_None) {
      const at::Tensor& t = tensor(out);
      given = out;
      dt = dtype_code(t.scalar_type());
      p = t.data_ptr();
    } else {
      dt = dtype_code(type);
      own = at::empty({in.M, N}, in.x.options().dtype(type).requires_grad(false));
      p = own.data_ptr();
    }
  }
  PyObject* result() noexcept {
    if (!given) return THPVariable_Wrap(std::move(own));
    Py_INCREF(given);
    return given;
  }
};

at::ScalarType scalar_type(PyObject* o) {
  if (!THPDtype_Check(o)) throw NotPlain();
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

bool mx(int64_t layout) { return layout == BL_W_MX4 || layout == BL_W_MX2; }

template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F body) {
  try {
    if (n != want || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    return body();
  } catch (const NotPlain&) {
    Py_RETURN_NONE;
  } catch (const std::exception_ptr&) {
    return nullptr;                                        // (a Python error is set)
  } catch (python_error& e) {                              // (Python code that torch called, a dispatch mode for instance: its own error)
    e.restore();
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  } catch (const std::exception&) {                        // (allocation, a tensor without storage: nothing is enqueued yet,
    if (PyErr_Occurred()) return nullptr;                  //  and the general way meets the same and words it)
    Py_RETURN_NONE;
  }
}

// (X, W_packed, alpha, N, eps, act_fp4, y_dtype, ws, out, layout)
PyObject* a4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const Input in(a[0]);
    void* const w = pointer(a[1]);
    const float* const alpha = (const float*)pointer(a[2]);
    const int64_t N = integer(a[3]), layout = integer(a[9]);
    const float eps = real(a[4]);
    const bool fp4 = truth(a[5]);
    if (in.M < 1 || N < 1 || N > ((int64_t)1 << 31) || layout < 0 || layout > 4) throw NotPlain();
    const int mode = fp4 ? (mx(layout) ? BL_ACT_FP4_E2M1_B32_MX : BL_ACT_FP4_E2M1_B32)
                         : (mx(layout) ? BL_ACT_INT4_ABSMEAN_MX6 : BL_ACT_INT4_ABSMEAN);
    Workspace ws(a[7], in, [&] { return lib.workspace_bytes((bl_act_mode)mode, in.M, N, in.K); });
    Output y(a[8], in, N, scalar_type(a[6]));
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib.a4(in.p, (bl_dtype)in.dt, in.M, in.K, w, (bl_w_layout)layout, alpha, N, eps, fp4 ? 1 : 0, y.p,
                      (bl_dtype)y.dt, nullptr, ws.p, ws.n, s);
    Py_END_ALLOW_THREADS
    return rc ? PyLong_FromLong(rc) : y.result();
  });
}

// (X, topk, W_packed, alpha, N, eps, layout, y_dtype, ws, out)
PyObject* a8_sparse(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const Input in(a[0]);
    const int64_t topk = integer(a[1]), N = integer(a[4]), layout = integer(a[6]);
    void* const w = pointer(a[2]);
    const float* const alpha = (const float*)pointer(a[3]);
    const float eps = real(a[5]);
    if (in.M < 1 || N < 1 || N > ((int64_t)1 << 31) || layout < 0 || layout > 4) throw NotPlain();
    Workspace ws(a[8], in, [&] { return lib.workspace_bytes(BL_ACT_TOPK_INT8_ABSMAX, in.M, N, in.K); });
    Output y(a[9], in, N, scalar_type(a[7]));
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib.a8_sparse(in.p, (bl_dtype)in.dt, in.M, in.K, topk, w, (bl_w_layout)layout, alpha, N, eps, y.p,
                             (bl_dtype)y.dt, nullptr, ws.p, ws.n, s);
    Py_END_ALLOW_THREADS
    return rc ? PyLong_FromLong(rc) : y.result();
  });
}

// (X, W_gate, alpha_gate, W_up, alpha_up, N, eps, layout, want, ws, out): want == ("H",), out None or {"H": tensor}
PyObject* gate_up(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    PyObject* const want = a[8];
    if (!PyTuple_CheckExact(want) || PyTuple_GET_SIZE(want) != 1 || !PyUnicode_CheckExact(PyTuple_GET_ITEM(want, 0)) ||
        PyUnicode_Compare(PyTuple_GET_ITEM(want, 0), str_H) != 0)
      throw NotPlain();
    PyObject* h = Py_None;
    if (a[10] != Py_None) {
      if (!PyDict_CheckExact(a[10]) || PyDict_GET_SIZE(a[10]) > 1) throw NotPlain();
      h = PyDict_GetItemWithError(a[10], str_H);           // (borrowed)
      if (!h || h == Py_None) { PyErr_Clear(); throw NotPlain(); }
    }
    const Input in(a[0]);
    void* const wg = pointer(a[1]);
    const float* const ag = (const float*)pointer(a[2]);
    void* const wu = pointer(a[3]);
    const float* const au = (const float*)pointer(a[4]);
    const int64_t N = integer(a[5]), layout = integer(a[7]);
    const float eps = real(a[6]);
    if (in.M < 1 || N < 1 || N > ((int64_t)1 << 31) || layout < 0 || layout > 4) throw NotPlain();
    Workspace ws(a[9], in, [&] { return lib.gate_up_workspace_bytes(in.M, N, in.K, (bl_w_layout)layout); });
    void* hp;
    at::Tensor own;
    if (h != Py_None) {
      hp = tensor(h).data_ptr();
    } else {
      own = at::empty({in.M, N}, in.x.options().dtype(at::kBFloat16).requires_grad(false));
      hp = own.data_ptr();
    }
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib.gate_up(in.p, (bl_dtype)in.dt, in.M, in.K, wg, ag, wu, au, (bl_w_layout)layout, N, eps, nullptr, nullptr,
                              BL_F32, hp, ws.p, ws.n, s);
    Py_END_ALLOW_THREADS
    if (rc) return PyLong_FromLong(rc);
    PyObject* const r = PyDict_New();
    if (!r) return nullptr;
    PyObject* const v = h != Py_None ? (Py_INCREF(h), h) : THPVariable_Wrap(std::move(own));
    const int bad = v ? PyDict_SetItem(r, str_H, v) : -1;
    Py_XDECREF(v);
    if (bad) { Py_DECREF(r); return nullptr; }
    return r;
  });
}

// A device's tensors: contiguous, of one type, on the device that is the current one (its stream is the call's)
struct Place {
  int index;
  at::Device device;
  explicit Place(const at::Tensor& t) : index(0), device(t.device()) {
    if (!t.is_cuda()) throw NotPlain();
    PyObject* const d = PyObject_CallNoArgs(get_device);
    if (!d) throw std::exception_ptr();
    index = (int)PyLong_AsLong(d);
    Py_DECREF(d);
    if (device.index() != index) throw NotPlain();
  }
  const at::Tensor& dense(PyObject* o, at::ScalarType type) const {
    const at::Tensor& t = tensor(o);
    if (t.device() != device || !t.is_contiguous() || t.scalar_type() != type) throw NotPlain();
    return t;
  }
};

// [T, heads, D] rows a stride apart, as the binding's _rows has them
int64_t rows(const at::Tensor& x, const Place& at) {
  if (x.device() != at.device || x.dim() != 3) throw NotPlain();
  if ((x.size(2) > 1 && x.stride(2) != 1) || (x.size(1) > 1 && x.stride(1) != x.size(2))) throw NotPlain();
  return x.size(0) > 1 ? x.stride(0) : x.size(1) * x.size(2);
}

// pages, page table, row starts, lengths and rotations, as the binding's _batch checks them
struct Paged {
  void *pages, *table, *q_start, *kv_len, *rope = nullptr;
  int64_t n_pages, n_seqs, max_pages, n_pos = 0;
  Paged(PyObject* p, PyObject* t, PyObject* qs, PyObject* ln, PyObject* r, int64_t H, int64_t D, const Place& at) {
    const at::Tensor& pg = at.dense(p, at::kByte);
    const at::Tensor& tb = at.dense(t, at::kInt);
    const at::Tensor& q = at.dense(qs, at::kInt);
    const at::Tensor& l = at.dense(ln, at::kInt);
    n_seqs = l.numel();
    if (tb.dim() != 2 || tb.size(0) != n_seqs || q.numel() != n_seqs + 1) throw NotPlain();
    if (pg.dim() != 2 || pg.size(1) != (int64_t)att.page_bytes(H, D)) throw NotPlain();
    if (r != Py_None) {
      const at::Tensor& f = at.dense(r, at::kFloat);
      if (f.dim() != 2 || f.size(1) != D) throw NotPlain();
      rope = f.data_ptr();
      n_pos = f.size(0);
    }
    pages = pg.data_ptr();
    table = tb.data_ptr();
    q_start = q.data_ptr();
    kv_len = l.data_ptr();
    n_pages = pg.size(0);
    max_pages = tb.size(1);
  }
};

// (K, V, pages, page_table, q_start, kv_len, rope, eps) -> 0
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]);
    const Place at(k);
    const int64_t ldk = rows(k, at), ldv = rows(v, at);
    if (k.sizes() != v.sizes() || k.scalar_type() != v.scalar_type()) throw NotPlain();
    const int dt = dtype_code(k.scalar_type());
    const int64_t T = k.size(0), H = k.size(1), D = k.size(2);
    const Paged b(a[2], a[3], a[4], a[5], a[6], H, D, at);
    const float eps = real(a[7]);
    void *const kp = k.data_ptr(), *const vp = v.data_ptr(), *const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = att.append(kp, ldk, vp, ldv, (bl_dtype)dt, T, H, D, (const int32_t*)b.q_start, (const int32_t*)b.kv_len, b.n_seqs,
                    (const int32_t*)b.table, b.max_pages, (const float*)b.rope, b.n_pos, eps, b.pages, b.n_pages, s);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  });
}

// (Q, pages, page_table, q_start, kv_len, H, rope, scale, window, sinks, q_bits, eps, ws, out)
PyObject* kv_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> PyObject* {
    const at::Tensor& q = tensor(a[0]);
    const Place at(q);
    const int64_t ldq = rows(q, at), T = q.size(0), Hq = q.size(1), D = q.size(2), H = integer(a[5]);
    const int dt = dtype_code(q.scalar_type());
    const Paged b(a[1], a[2], a[3], a[4], a[6], H, D, at);
    if (D < 1) throw NotPlain();
    const float scale = a[7] == Py_None ? (float)std::pow((double)D, -0.5) : real(a[7]), eps = real(a[11]);
    const int64_t window = integer(a[8]), sinks = integer(a[9]), q_bits = integer(a[10]);
    if (q_bits != 16 && q_bits != 4) throw NotPlain();
    const auto options = q.options().requires_grad(false);
    at::Tensor ws, own;
    size_t bytes = att.attention_bytes(T, b.n_seqs, Hq, H, D, b.max_pages);
    void* wp = nullptr;
    if (a[12] != Py_None) {
      const at::Tensor& t = tensor(a[12]);
      if (t.device() != at.device || !t.is_contiguous()) throw NotPlain();
      wp = t.data_ptr();
      bytes = t.nbytes();
    } else if (bytes) {
      ws = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
      wp = ws.data_ptr();
    }
    void* op;
    if (a[13] != Py_None) {
      const at::Tensor& t = at.dense(a[13], at::kBFloat16);
      if (t.sizes() != q.sizes()) throw NotPlain();
      op = t.data_ptr();
    } else {
      own = at::empty({T, Hq, D}, options.dtype(at::kBFloat16));
      op = own.data_ptr();
    }
    void *const qp = q.data_ptr(), *const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = att.attention(qp, ldq, (bl_dtype)dt, T, Hq, H, D, (int)q_bits, (const int32_t*)b.q_start, (const int32_t*)b.kv_len, b.n_seqs,
                       (const int32_t*)b.table, b.max_pages, (const float*)b.rope, b.n_pos, scale, eps, window, sinks, b.pages,
                       b.n_pages, op, wp, bytes, s);
    Py_END_ALLOW_THREADS
    if (rc) return PyLong_FromLong(rc);
    if (a[13] == Py_None) return THPVariable_Wrap(std::move(own));
    Py_INCREF(a[13]);
    return a[13];
  });
}

// (X, gamma, mode, residual, norm_eps, eps) -> dict(q, scale, h, rstd)
PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Input in(a[0]);
    const Place at(in.x);
    const at::Tensor& g = at.dense(a[1], at::kFloat);
    const int64_t mode = integer(a[2]);
    if (in.M < 1 || in.K < 1 || g.numel() != in.K || mode < 0 || mode > 64) throw NotPlain();
    const float norm_eps = real(a[4]), eps = real(a[5]);
    const void* r = nullptr;
    const auto options = in.x.options().requires_grad(false);
    at::Tensor h;
    void* hp = nullptr;
    if (a[3] != Py_None) {
      const at::Tensor& t = at.dense(a[3], in.x.scalar_type());
      if (t.sizes() != in.x.sizes()) throw NotPlain();
      r = t.data_ptr();
      h = at::empty({in.M, in.K}, options);
      hp = h.data_ptr();
    }
    const size_t bytes = att.act_bytes((bl_act_mode)mode, in.M, in.K);
    if (!bytes) throw NotPlain();
    at::Tensor q = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
    at::Tensor scale = at::empty({in.M}, options.dtype(at::kFloat)), rstd = at::empty({in.M}, options.dtype(at::kFloat));
    void* const s = stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = att.norm(in.p, r, (bl_dtype)in.dt, in.M, in.K, (const float*)g.data_ptr(), norm_eps, (bl_act_mode)mode, eps, hp,
                  (float*)rstd.data_ptr(), q.data_ptr(), (float*)scale.data_ptr(), s);
    Py_END_ALLOW_THREADS
    if (rc) return PyLong_FromLong(rc);
    PyObject* const d = PyDict_New();
    if (!d) return nullptr;
    bool bad = false;
    auto put = [&](PyObject* key, PyObject* v) {
      bad = bad || !v || PyDict_SetItem(d, key, v) != 0;
      Py_XDECREF(v);
    };
    put(str_q, THPVariable_Wrap(std::move(q)));
    put(str_scale, THPVariable_Wrap(std::move(scale)));
    if (hp) put(str_h, THPVariable_Wrap(std::move(h)));
    else { Py_INCREF(a[0]); put(str_h, a[0]); }
    put(str_rstd, THPVariable_Wrap(std::move(rstd)));
    if (bad) { Py_DECREF(d); return nullptr; }
    return d;
  });
}

// (addresses of bitlinear_a4, bitlinear_a8_sparse, bitlinear_a4_gate_up, bitlinear_workspace_bytes, bitlinear_gate_up_workspace_bytes)
template <size_t N>
bool addresses(PyObject* const* a, Py_ssize_t n, void* (&p)[N]) {
  if (n != (Py_ssize_t)N) {
    PyErr_Format(PyExc_TypeError, "%zu addresses expected", N);
    return false;
  }
  for (size_t i = 0; i < N; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return false;
    }
  }
  return true;
}
PyObject* use(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[5];
  if (!addresses(a, n, p)) return nullptr;
  lib = {(decltype(lib.a4))p[0], (decltype(lib.a8_sparse))p[1], (decltype(lib.gate_up))p[2], (decltype(lib.workspace_bytes))p[3],
         (decltype(lib.gate_up_workspace_bytes))p[4]};
  Py_RETURN_NONE;
}
// (addresses of rmsnorm_quantize, quantize_act_bytes, kv_pages_append, kv_pages_attention, kv_pages_attention_workspace_bytes,
// kv_page_bytes)
PyObject* use_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[6];
  if (!addresses(a, n, p)) return nullptr;
  att = {(decltype(att.norm))p[0], (decltype(att.act_bytes))p[1], (decltype(att.append))p[2], (decltype(att.attention))p[3],
         (decltype(att.attention_bytes))p[4], (decltype(att.page_bytes))p[5]};
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"use", (PyCFunction)(void (*)(void))use, METH_FASTCALL, "the library's functions, by address; before any other call"},
    {"a4", (PyCFunction)(void (*)(void))a4, METH_FASTCALL, "bitlinear_a4"},
    {"a8_sparse", (PyCFunction)(void (*)(void))a8_sparse, METH_FASTCALL, "bitlinear_a8_sparse"},
    {"gate_up", (PyCFunction)(void (*)(void))gate_up, METH_FASTCALL, "bitlinear_a4_gate_up, H only"},
    {"use_attention", (PyCFunction)(void (*)(void))use_attention, METH_FASTCALL, "those of the three below, by address"},
    {"norm", (PyCFunction)(void (*)(void))norm, METH_FASTCALL, "rmsnorm_quantize"},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, "kv_pages_append"},
    {"kv_attention", (PyCFunction)(void (*)(void))kv_attention, METH_FASTCALL, "kv_pages_attention"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "bitlinear_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_bitlinear_marshal() {
  PyObject* const c = PyImport_ImportModule("torch._C");
  if (!c) return nullptr;
  get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
  get_stream = get_device ? PyObject_GetAttrString(c, "_cuda_getCurrentRawStream") : nullptr;
  Py_DECREF(c);
  if (!get_stream) {
    if (PyErr_Occurred()) PyErr_Clear();
    PyErr_SetString(PyExc_ImportError, "torch without GPU support");
    return nullptr;
  }
  str_H = PyUnicode_InternFromString("H");
  str_q = PyUnicode_InternFromString("q");
  str_scale = PyUnicode_InternFromString("scale");
  str_h = PyUnicode_InternFromString("h");
  str_rstd = PyUnicode_InternFromString("rstd");
  return str_H && str_q && str_scale && str_h && str_rstd ? PyModule_Create(&module) : nullptr;
}
