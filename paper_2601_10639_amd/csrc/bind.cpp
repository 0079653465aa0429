// The hot calls of stemlib.py natively: tensors to pointers, the current stream, and the C call without the interpreter's lock.
//
// A small layer's call spends as long on the host as on the GPU: a launch takes 2.7 to 3.5 us there, and forward_residual's arguments took
// 2.9 in Python (0.22 for each tensor's checks, 0.36 for the stream, 0.6 for ctypes), 0.46 here.  A training step of 128 tokens of 64 x 256
// fp32, four calls and six launches, 33.8 -> 24.0 us.
//
// Only the ordinary call is made here: plain torch tensors of the right type in contiguous device memory, ints, floats and bools.
// Every function returns None, having done nothing, where anything else is among the arguments, and stemlib.py then makes the call as it
// does without this module: its checks say what is wrong, or take what this one does not know.  It looks into torch's and Python's objects,
// so stemlib.py uses it only with the versions it was built for.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include "../../include/stem.h"

namespace {

PyObject *g_ctx_type, *g_get_device, *g_raw_stream, *g_handle, *g_value, *g_dtype, *g_cuda_stream;   // set by setup()
PyObject *g_norm_type, *g_leave_type, *g_quant_type, *g_tensor, *g_norms, *g_gate_tensor, *g_step_tensor, *g_d_model, *g_d_ff, *g_q, *g_scale, *g_N, *g_K;
bool g_off = true;                                        // before setup(), and in a forked process

struct Unusual {};

struct Hold {                  // a new reference, or Unusual
  PyObject* o;
  explicit Hold(PyObject* p) : o(p) {
    if (!p) { PyErr_Clear(); throw Unusual(); }
  }
  ~Hold() { Py_DECREF(o); }
};

enum Kind { ACT, F32, I32, I64, I8 };   // ACT: the context's type

// The memory of one of stemlib.py's ctypes structures, of exactly this type
template <class T>
const T* structure(PyObject* o, PyObject* type) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != type) throw Unusual();
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) < 0) {
    PyErr_Clear();
    throw Unusual();
  }
  void* const p = b.buf;
  const bool whole = b.len == (Py_ssize_t)sizeof(T);
  PyBuffer_Release(&b);        // (the object, which the caller's arguments hold, keeps its memory)
  if (!whole) throw Unusual();
  return static_cast<const T*>(p);
}

// The arguments of one call
struct Args {
  PyObject* const* v;
  PyObject* ctx;
  int dtype;
  mutable bool device_seen;    // a device tensor is among them: the runtime is up

  template <class T = void>
  T* ptr(int i, Kind kind) const { return static_cast<T*>(pointer_of(v[i], kind, -1, -1)); }
  // of this shape: [rows, cols], or [rows] where cols is -1
  template <class T = void>
  T* shaped(int i, Kind kind, int64_t rows, int64_t cols = -1) const { return static_cast<T*>(pointer_of(v[i], kind, rows, cols)); }

  void* pointer_of(PyObject* o, Kind kind, int64_t rows, int64_t cols) const {
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) throw Unusual();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (rows >= 0 && (t.dim() != (cols < 0 ? 1 : 2) || t.size(0) != rows || (cols >= 0 && t.size(1) != cols))) throw Unusual();
    const at::ScalarType want = kind == I32 ? at::kInt : kind == I64 ? at::kLong : kind == I8 ? at::kChar
                                : kind == ACT && dtype == STEM_BF16 ? at::kBFloat16 : at::kFloat;
    if (t.layout() != at::kStrided || t.scalar_type() != want || !t.is_cuda() || !t.is_contiguous()) throw Unusual();
    device_seen = true;
    // (as data_ptr() in Python: a tensor that shares its storage with another until one is written gets its own first.  Inputs too, as a
    // call may write to the same tensor)
    return t.mutable_data_ptr();
  }

  int64_t attribute(PyObject* o, PyObject* name) const { return as_integer(Hold(PyObject_GetAttr(o, name)).o); }
  // dropout's device counter, of one element
  const uint64_t* counter(PyObject* o) const {
    if (o != Py_None && THPVariable_CheckExact(o) && THPVariable_Unpack(o).numel() != 1) throw Unusual();
    return static_cast<const uint64_t*>(pointer_of(o, I64, -1, -1));
  }
  // The structures with the pointers that their tensors have now
  struct Norm {
    stem_norm norm;
    bool given;
    const stem_norm* get() const { return given ? &norm : nullptr; }
  };
  const void* weight(PyObject* norm, const void* as_is, int64_t width) const {
    const Hold t(PyObject_GetAttr(norm, g_tensor));
    return t.o == Py_None ? as_is : pointer_of(t.o, ACT, width, -1);
  }
  // a norm of rows of `width` (None: none)
  Norm norm(int i, int64_t width) const {
    if (v[i] == Py_None) return {{}, false};
    Norm n = {*structure<stem_norm>(v[i], g_norm_type), true};
    n.norm.weight = weight(v[i], n.norm.weight, width);
    return n;
  }
  stem_leave leave(int i, int64_t T, int64_t d) const {
    stem_leave L = *structure<stem_leave>(v[i], g_leave_type);
    const Hold norms(PyObject_GetAttr(v[i], g_norms)), gate(PyObject_GetAttr(v[i], g_gate_tensor)), step(PyObject_GetAttr(v[i], g_step_tensor));
    if (!PyTuple_CheckExact(norms.o) || PyTuple_GET_SIZE(norms.o) != 2) throw Unusual();
    L.out.weight = weight(PyTuple_GET_ITEM(norms.o, 0), L.out.weight, d);
    L.next.weight = weight(PyTuple_GET_ITEM(norms.o, 1), L.next.weight, d);
    if (gate.o != Py_None)
      L.gate = pointer_of(gate.o, ACT, L.gate_kind == STEM_GATE_CHANNEL ? d : T, L.gate_kind == STEM_GATE_FULL ? d : -1);
    if (step.o != Py_None && L.drop.step) L.drop.step = counter(step.o);
    return L;
  }
  // weights in 8 bits
  struct Quant { const void* q; const float* scale; int64_t N, K; };
  Quant quant(int i) const {
    if (reinterpret_cast<PyObject*>(Py_TYPE(v[i])) != g_quant_type) throw Unusual();
    const int64_t N = attribute(v[i], g_N), K = attribute(v[i], g_K);
    const Hold q(PyObject_GetAttr(v[i], g_q)), scale(PyObject_GetAttr(v[i], g_scale));
    return {pointer_of(q.o, I8, stem_quant_bytes(N, K), -1), static_cast<const float*>(pointer_of(scale.o, F32, N, -1)), N, K};
  }
  int64_t d_model() const { return attribute(ctx, g_d_model); }
  int64_t d_ff() const { return attribute(ctx, g_d_ff); }

  static int64_t as_integer(PyObject* o) {
    if (!PyLong_CheckExact(o)) throw Unusual();
    int overflow = 0;
    const int64_t x = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) throw Unusual();
    return x;
  }
  int64_t integer(int i) const { return as_integer(v[i]); }
  int flag(int i) const {
    if (!PyBool_Check(v[i])) throw Unusual();
    return v[i] == Py_True;
  }
  float number(int i) const {
    if (!PyFloat_CheckExact(v[i])) throw Unusual();
    return (float)PyFloat_AS_DOUBLE(v[i]);
  }
  void* pointer(int i) const { return v[i] == Py_None ? nullptr : reinterpret_cast<void*>(integer(i)); }

  // argument i (-1: there is none), or where it is None the rows of tensor t (0 where that is None and may be)
  int64_t rows(int i, int t, bool none_is_0 = false) const {
    if (i >= 0 && v[i] != Py_None) return integer(i);
    if (v[t] == Py_None && none_is_0) return 0;
    if (!THPVariable_CheckExact(v[t])) throw Unusual();
    const at::Tensor& x = THPVariable_Unpack(v[t]);
    if (x.dim() < 1) throw Unusual();
    return x.size(0);
  }

  // a stream's handle, or the current stream's; after the tensors
  void* stream(int i) const {
    if (PyLong_CheckExact(v[i])) return reinterpret_cast<void*>(integer(i));
    if (v[i] != Py_None) return reinterpret_cast<void*>(as_integer(Hold(PyObject_GetAttr(v[i], g_cuda_stream)).o));
    if (!device_seen) throw Unusual();
    const Hold device(PyObject_CallNoArgs(g_get_device));
    return reinterpret_cast<void*>(as_integer(Hold(PyObject_CallOneArg(g_raw_stream, device.o)).o));
  }
};

// f gets the arguments behind the context, and its handle, and returns the call.
template <class F>
PyObject* enter(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want + 1) return PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want + 1, n);
  if (g_off || reinterpret_cast<PyObject*>(Py_TYPE(args[0])) != g_ctx_type) Py_RETURN_NONE;
  try {
    const Hold handle(PyObject_GetAttr(args[0], g_handle)), value(PyObject_GetAttr(handle.o, g_value)), dtype(PyObject_GetAttr(args[0], g_dtype));
    stem_ctx* const c = reinterpret_cast<stem_ctx*>(Args::as_integer(value.o));   // (closed: None)
    const Args a{args + 1, args[0], (int)Args::as_integer(dtype.o), false};
    auto call = f(a, c);
    stem_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  } catch (...) {              // Unusual, or what a tensor without storage throws
    Py_RETURN_NONE;
  }
}

PyObject* ffn_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 12, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(11, 0), E_rows = a.rows(10, 4);
    auto x = a.ptr(0, ACT); auto ids = a.ptr<int32_t>(1, I32); auto Wg = a.ptr(2, ACT); auto Wd = a.ptr(3, ACT);
    auto E = a.ptr(4, ACT); auto y = a.ptr(5, ACT); auto G = a.ptr(6, ACT); auto H = a.ptr(7, ACT);
    auto event = a.pointer(8); auto s = a.stream(9);
    return [=] { return stem_ffn_forward(c, x, ids, Wg, Wd, E, E_rows, T, y, G, H, event, s); };
  });
}

PyObject* ffn_forward_residual(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 10, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(9, 0), E_rows = a.rows(8, 4);
    auto x = a.ptr(0, ACT); auto ids = a.ptr<int32_t>(1, I32); auto Wg = a.ptr(2, ACT); auto Wd = a.ptr(3, ACT);
    auto E = a.ptr(4, ACT); auto r = a.ptr(5, ACT); auto y = a.ptr(6, ACT); auto s = a.stream(7);
    return [=] { return stem_ffn_forward_residual(c, x, ids, Wg, Wd, E, E_rows, T, r, y, s); };
  });
}

PyObject* ffn_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 16, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(15, 0), E_rows = a.rows(14, 5);
    auto dy = a.ptr(0, ACT); auto x = a.ptr(1, ACT); auto ids = a.ptr<int32_t>(2, I32); auto Wg = a.ptr(3, ACT);
    auto Wd = a.ptr(4, ACT); auto E = a.ptr(5, ACT); auto G = a.ptr(6, ACT); auto H = a.ptr(7, ACT);
    auto dx = a.ptr(8, ACT); auto dWg = a.ptr<float>(9, F32); auto dWd = a.ptr<float>(10, F32);
    auto dU = a.ptr(11, ACT); const int accumulate = a.flag(12); auto s = a.stream(13);
    return [=] { return stem_ffn_backward(c, dy, x, ids, Wg, Wd, E, E_rows, G, H, T, dx, dWg, dWd, dU, accumulate, s); };
  });
}

PyObject* ffn_up_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 13, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(12, 0), E_rows = a.rows(11, 5, true);
    auto x = a.ptr(0, ACT); auto ids = a.ptr<int32_t>(1, I32); auto Wg = a.ptr(2, ACT); auto Wu = a.ptr(3, ACT);
    auto Wd = a.ptr(4, ACT); auto E = a.ptr(5, ACT); auto y = a.ptr(6, ACT); auto G = a.ptr(7, ACT);
    auto Up = a.ptr(8, ACT); auto H = a.ptr(9, ACT); auto s = a.stream(10);
    return [=] { return stem_ffn_up_forward(c, x, ids, Wg, Wu, Wd, E, E_rows, T, y, G, Up, H, s); };
  });
}

PyObject* ffn_up_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 19, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(18, 0), E_rows = a.rows(17, 6, true);
    auto dy = a.ptr(0, ACT); auto x = a.ptr(1, ACT); auto ids = a.ptr<int32_t>(2, I32); auto Wg = a.ptr(3, ACT);
    auto Wu = a.ptr(4, ACT); auto Wd = a.ptr(5, ACT); auto E = a.ptr(6, ACT); auto G = a.ptr(7, ACT);
    auto Up = a.ptr(8, ACT); auto H = a.ptr(9, ACT); auto dx = a.ptr(10, ACT);
    auto dWg = a.ptr<float>(11, F32); auto dWu = a.ptr<float>(12, F32); auto dWd = a.ptr<float>(13, F32);
    auto dV = a.ptr(14, ACT); const int accumulate = a.flag(15); auto s = a.stream(16);
    return [=] { return stem_ffn_up_backward(c, dy, x, ids, Wg, Wu, Wd, E, E_rows, G, Up, H, T, dx, dWg, dWu, dWd, dV, accumulate, s); };
  });
}

PyObject* embed_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 10, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(9, 0);
    auto ids = a.ptr<int32_t>(0, I32); auto dU = a.ptr(1, ACT); auto sorted = a.ptr<int32_t>(2, I32);
    auto perm = a.ptr<int32_t>(3, I32); auto uniq = a.ptr<int32_t>(4, I32); auto offs = a.ptr<int32_t>(5, I32);
    auto nu = a.ptr<int32_t>(6, I32); auto dE = a.ptr<float>(7, F32); auto s = a.stream(8);
    return [=] { return stem_embed_grad(c, ids, dU, T, sorted, perm, uniq, offs, nu, dE, s); };
  });
}

PyObject* embed_grad_presorted(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 6, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(5, 0);
    auto dU = a.ptr(0, ACT); auto perm = a.ptr<int32_t>(1, I32); auto offs = a.ptr<int32_t>(2, I32);
    auto dE = a.ptr<float>(3, F32); auto s = a.stream(4);
    return [=] { return stem_embed_grad_presorted(c, dU, T, perm, offs, dE, s); };
  });
}

PyObject* embed_sparse_adamw(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 15, [](const Args& a, stem_ctx* c) {
    const int64_t max_rows = a.rows(14, 2);
    auto uniq = a.ptr<int32_t>(0, I32); auto nu = a.ptr<int32_t>(1, I32); auto dE = a.ptr<float>(2, F32);
    auto E = a.ptr(3, ACT); auto master = a.ptr<float>(4, F32); auto m = a.ptr<float>(5, F32); auto v = a.ptr<float>(6, F32);
    stem_adamw_hparams hp;
    hp.lr = a.number(7); hp.beta1 = a.number(8); hp.beta2 = a.number(9); hp.eps = a.number(10); hp.weight_decay = a.number(11);
    hp.step = a.integer(12);
    auto s = a.stream(13);
    return [=] { return stem_embed_sparse_adamw(c, uniq, nu, max_rows, dE, E, master, m, v, &hp, s); };
  });
}

PyObject* block_enter_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 4, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(-1, 0), d = a.d_model();
    auto x = a.shaped(0, ACT, T, d); auto norm = a.norm(1, d); auto to = a.shaped(2, ACT, T, d); auto s = a.stream(3);
    return [=] { return stem_block_enter_forward(c, x, T, norm.get(), to, s); };
  });
}

PyObject* block_enter_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 8, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(-1, 1), d = a.d_model();
    auto dn = a.shaped(0, ACT, T, d); auto x = a.shaped(1, ACT, T, d); auto norm = a.norm(2, d); auto dx = a.shaped(3, ACT, T, d);
    auto dw = a.shaped<float>(4, F32, d); auto dres = a.shaped(5, ACT, T, d); const int accumulate = a.flag(6); auto s = a.stream(7);
    return [=] { return stem_block_enter_backward(c, dn, x, T, norm.get(), dres, dx, dw, accumulate, s); };
  });
}

PyObject* block_leave_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 6, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(-1, 1), d = a.d_model();
    auto f = a.shaped(0, ACT, T, d); auto x = a.shaped(1, ACT, T, d); auto L = a.leave(2, T, d); auto y = a.shaped(3, ACT, T, d);
    auto to = a.shaped(4, ACT, T, d); auto s = a.stream(5);
    return [=] { return stem_block_leave_forward(c, f, x, T, &L, y, to, s); };
  });
}

PyObject* block_leave_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 12, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(-1, a.v[0] == Py_None ? 1 : 0), d = a.d_model();
    auto dy = a.shaped(0, ACT, T, d); auto dn = a.shaped(1, ACT, T, d); auto f = a.shaped(2, ACT, T, d); auto y = a.shaped(3, ACT, T, d);
    auto L = a.leave(4, T, d); auto dx = a.shaped(5, ACT, T, d); auto df = a.shaped(6, ACT, T, d);
    auto dg = L.gate_kind == STEM_GATE_CHANNEL ? a.shaped(7, F32, d) : L.gate_kind == STEM_GATE_TOKEN ? a.shaped(7, ACT, T) : a.shaped(7, ACT, T, d);
    auto dwo = a.shaped<float>(8, F32, d); auto dwn = a.shaped<float>(9, F32, d); const int accumulate = a.flag(10); auto s = a.stream(11);
    return [=] { return stem_block_leave_backward(c, dy, dn, f, y, T, &L, dx, df, dg, dwo, dwn, accumulate, s); };
  });
}

PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 7, [](const Args& a, stem_ctx* c) {
    if (!THPVariable_CheckExact(a.v[0])) throw Unusual();
    const at::Tensor& t = THPVariable_Unpack(a.v[0]);
    if (t.dim() != 2) throw Unusual();
    const int64_t T = t.size(0), width = t.size(1), seed = a.integer(3), offset = a.integer(4);
    if (seed < 0 || offset < 0) throw Unusual();
    auto x = a.shaped(0, ACT, T, width); auto y = a.shaped(1, ACT, T, width);
    const stem_drop drop = {a.number(2), (uint64_t)seed, (uint64_t)offset, a.counter(a.v[5])};
    auto s = a.stream(6);
    return [=] { return stem_dropout(c, x, T, width, &drop, y, s); };
  });
}

PyObject* quant_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 6, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(-1, 0);
    const Args::Quant w = a.quant(1);
    auto x = a.shaped(0, ACT, T, w.K); auto y = a.shaped(2, ACT, T, w.N); auto r = a.shaped(3, ACT, T, w.N); auto norm = a.norm(4, w.K);
    auto s = a.stream(5);
    return [=] { return stem_quant_linear(c, x, T, w.K, norm.get(), w.q, w.scale, w.N, r, y, s); };
  });
}

PyObject* quant_ffn_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return enter(args, n, 10, [](const Args& a, stem_ctx* c) {
    const int64_t T = a.rows(-1, 0), d = a.d_model(), F = a.d_ff(), rows = a.rows(-1, 4), E_rows = a.rows(9, 4);
    const Args::Quant g = a.quant(2), w = a.quant(3);
    if (g.N != F || g.K != d || w.N != d || w.K != F) throw Unusual();
    auto x = a.shaped(0, ACT, T, d); auto ids = a.shaped<int32_t>(1, I32, T); auto E = a.shaped(4, ACT, rows, F); auto y = a.shaped(5, ACT, T, d);
    auto r = a.shaped(6, ACT, T, d); auto norm = a.norm(7, d); auto s = a.stream(8);
    return [=] { return stem_quant_ffn_forward(c, x, ids, T, norm.get(), g.q, g.scale, w.q, w.scale, E, E_rows, r, y, s); };
  });
}

// (StemCtx, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, stem_norm, stem_leave, StemQuant)
PyObject* setup(PyObject*, PyObject* args) {
  if (!PyArg_ParseTuple(args, "OOOOOO", &g_ctx_type, &g_get_device, &g_raw_stream, &g_norm_type, &g_leave_type, &g_quant_type)) return nullptr;
  for (PyObject* o : {g_ctx_type, g_get_device, g_raw_stream, g_norm_type, g_leave_type, g_quant_type}) Py_INCREF(o);
  g_tensor = PyUnicode_InternFromString("tensor");
  g_norms = PyUnicode_InternFromString("norms");
  g_gate_tensor = PyUnicode_InternFromString("gate_tensor");
  g_step_tensor = PyUnicode_InternFromString("step_tensor");
  g_d_model = PyUnicode_InternFromString("d_model");
  g_d_ff = PyUnicode_InternFromString("d_ff");
  g_q = PyUnicode_InternFromString("q");
  g_scale = PyUnicode_InternFromString("scale");
  g_N = PyUnicode_InternFromString("N");
  g_K = PyUnicode_InternFromString("K");
  if (!g_tensor || !g_norms || !g_gate_tensor || !g_step_tensor || !g_d_model || !g_d_ff || !g_q || !g_scale || !g_N || !g_K) return nullptr;
  g_handle = PyUnicode_InternFromString("handle");
  g_value = PyUnicode_InternFromString("value");
  g_dtype = PyUnicode_InternFromString("dtype");
  g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  if (!g_handle || !g_value || !g_dtype || !g_cuda_stream) return nullptr;
  g_off = false;
  Py_RETURN_NONE;
}

PyObject* off(PyObject*, PyObject*) {
  g_off = true;
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(ffn_forward), FAST(ffn_forward_residual), FAST(ffn_backward), FAST(ffn_up_forward), FAST(ffn_up_backward),
                         FAST(embed_grad), FAST(embed_grad_presorted), FAST(embed_sparse_adamw),
                         FAST(block_enter_forward), FAST(block_enter_backward), FAST(block_leave_forward), FAST(block_leave_backward), FAST(dropout),
                         FAST(quant_linear), FAST(quant_ffn_forward),
                         {"setup", setup, METH_VARARGS, nullptr}, {"off", off, METH_NOARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#define STR_(x) #x
#define STR(x) STR_(x)
PyMODINIT_FUNC PyInit__bind() {
  PyObject* const m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "BUILT_FOR", "torch " TORCH_VERSION ", Python " STR(PY_MAJOR_VERSION) "." STR(PY_MINOR_VERSION)) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
