// The Python side of include/kv.h: reads the arguments of a call, checks its tensors and makes it.  Marshalling only.
//
// These calls are small in a step that generates one token, where the host's time is the call's: ten tensors cost 3.7 us to check in
// Python and 1.2 us to pass through ctypes, beside 3.5 us for the launch; here both are 0.5.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>

#include "../../include/kv.h"

namespace {

// The arguments of one call.  What is wrong is raised once (`bad`), and no call is made then.
struct Args {
  PyObject* const* v;
  long device;  // the current one, -1 without a GPU
  bool bad = false;

  void refuse(PyObject* kind, const char* format, ...) {
    if (bad) return;
    bad = true;
    va_list list;
    va_start(list, format);
    PyErr_FormatV(kind, format, list);
    va_end(list);
  }
  long long whole(int i) {
    const long long x = PyLong_Check(v[i]) ? PyLong_AsLongLong(v[i]) : other_whole(v[i]);
    if (x == -1 && PyErr_Occurred()) bad = true;
    return x;
  }
  static long long other_whole(PyObject* o) {  // (numpy's, and whatever else says that it is one)
    PyObject* const n = PyNumber_Index(o);
    if (!n) return -1;
    const long long x = PyLong_AsLongLong(n);
    Py_DECREF(n);
    return x;
  }
  int size(int i) {
    const long long x = whole(i);
    if (x != (int)x) refuse(PyExc_OverflowError, "%lld does not fit 32 bits", x);
    return (int)x;
  }
  float real(int i) {
    const double x = PyFloat_AsDouble(v[i]);
    if (x == -1.0 && PyErr_Occurred()) bad = true;
    return (float)x;
  }
  int truth(int i) {
    const int x = PyObject_IsTrue(v[i]);
    if (x < 0) bad = true;
    return x;
  }
  // the tensor, or null where the argument is None or an address (which is then in *address)
  const at::Tensor* tensor(int i, const char* name, void** address) {
    *address = nullptr;
    if (bad || v[i] == Py_None) return nullptr;
    if (THPVariable_Check(v[i])) return &THPVariable_Unpack(v[i]);
    if (!PyLong_Check(v[i])) {
      refuse(PyExc_TypeError, "%s is %s, not a tensor or an address", name, Py_TYPE(v[i])->tp_name);
      return nullptr;
    }
    *address = PyLong_AsVoidPtr(v[i]);
    if (!*address && PyErr_Occurred()) bad = true;
    return nullptr;
  }
  void* found(const at::Tensor& t, const char* name) {
    const long on = t.is_cuda() ? (long)t.get_device() : -1;
    if (on < 0) refuse(PyExc_ValueError, "%s is not on a GPU", name);
    else if (on != device) refuse(PyExc_ValueError, "%s is on device %ld, the current one is %ld", name, on, device);
    return bad ? nullptr : t.data_ptr();
  }
  bool typed(const at::Tensor& t, const char* name, bool as_wanted, const char* wanted) {
    if (!as_wanted) refuse(PyExc_ValueError, "%s is %s, not %s", name, c10::toString(t.scalar_type()), wanted);
    return as_wanted;
  }
  // a dense tensor of at least `least` elements (what the call reads or writes; sizes may be any numbers, so their product is a double)
  void* dense(const at::Tensor& t, const char* name, double least) {
    if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", name);
    else if ((double)t.numel() < least) refuse(PyExc_ValueError, "%s has %lld elements, %lld are needed", name, (long long)t.numel(), (long long)least);
    return bad ? nullptr : found(t, name);
  }
  void* of(int i, const char* name, at::ScalarType type, const char* wanted, double least) {
    void* address;
    const at::Tensor* const t = tensor(i, name, &address);
    if (!t) return address;
    return typed(*t, name, t->scalar_type() == type, wanted) ? dense(*t, name, least) : nullptr;
  }
  void* bf16(int i, const char* name, double least) { return of(i, name, at::kBFloat16, "BFloat16", least); }
  float* f32(int i, const char* name, double least) { return (float*)of(i, name, at::kFloat, "Float", least); }
  int* i32(int i, const char* name, double least) { return (int*)of(i, name, at::kInt, "Int", least); }
  void* cache(int i, const char* name, int dtype, double least) {
    if (dtype != ATTN_FP8_E4M3) return bf16(i, name, least);
    void* address;
    const at::Tensor* const t = tensor(i, name, &address);
    if (!t) return address;
    const bool fits = t->scalar_type() == at::kByte || t->scalar_type() == at::kFloat8_e4m3fn;
    return typed(*t, name, fits, "Byte or Float8_e4m3fn") ? dense(*t, name, least) : nullptr;
  }
  // `rows` rows of `width` bf16 features, ld elements apart: a dense buffer of any shape, or a view whose leading dimensions are those rows
  void* rows(int i, const char* name, long long ld, double rows, double width) {
    void* address;
    const at::Tensor* const t = tensor(i, name, &address);
    if (!t) return address;
    if (!typed(*t, name, t->scalar_type() == at::kBFloat16, "BFloat16")) return nullptr;
    bool ok;
    if (t->is_contiguous()) {
      ok = (double)t->numel() >= (rows - 1) * (double)ld + width;
    } else {
      const auto shape = t->sizes(), stride = t->strides();
      const int n = (int)shape.size();
      ok = n >= 1 && (double)shape[n - 1] >= width && stride[n - 1] == 1;
      double step = (double)ld, count = 1;
      for (int k = n - 2; k >= 0; --k) {
        ok = ok && (shape[k] == 1 || (double)stride[k] == step);
        step *= (double)shape[k];
        count *= (double)shape[k];
      }
      ok = ok && count >= rows;
    }
    if (!ok) {
      PyObject* const shape = PyObject_GetAttrString(v[i], "shape");
      refuse(PyExc_ValueError, "%s of shape %S does not hold %lld rows of %lld, %lld apart", name, shape ? shape : Py_None, (long long)rows, (long long)width, ld);
      Py_XDECREF(shape);
      return nullptr;
    }
    return found(*t, name);
  }
};

// qkv .. pos, in the order of kv.h, from argument `at` on
struct Rows {
  void *qkv, *wq, *wk;
  long long ld;
  float eps;
  float* table;
  int npos, rot, interleaved;
  int* pos;
};
Rows rows_of(Args& a, int at, double T, double width, double d, bool read = true) {  // (read: whether the rows are)
  Rows r;
  r.ld = a.whole(at + 1);
  r.qkv = read ? a.rows(at, "qkv", r.ld, T, width) : nullptr;
  r.wq = a.bf16(at + 2, "q_weight", d);
  r.wk = a.bf16(at + 3, "k_weight", d);
  r.eps = a.real(at + 4);
  r.npos = a.size(at + 6);
  r.rot = a.size(at + 7);
  r.table = a.f32(at + 5, "table", (double)r.npos * r.rot);
  r.interleaved = a.truth(at + 8);
  r.pos = a.i32(at + 9, "pos", T);
  return r;
}

// Makes the call.  The interpreter is free for other threads meanwhile, as it is inside a ctypes call: a launch waits where the device's queue is
// full, and what it waits for can need the interpreter.  (The caller's frame holds the arguments.)
template <typename F, typename... T>
int made(const Args& a, F function, T... arguments) {
  if (a.bad) return 0;
  PyThreadState* const state = PyEval_SaveThread();
  const int status = function(arguments...);
  PyEval_RestoreThread(state);
  return status;
}

// the first two arguments of every call: the current device, the stream
template <int COUNT, typename F>
PyObject* call(const char* name, PyObject* const* v, Py_ssize_t n, F f) {
  if (n != COUNT + 2) {
    PyErr_Format(PyExc_TypeError, "%s: %zd arguments, not %d", name, n - 2, COUNT);
    return nullptr;
  }
  try {
    Args a{v + 2, -1};
    const long device = PyLong_AsLong(v[0]);
    void* const stream = PyLong_AsVoidPtr(v[1]);
    if (PyErr_Occurred()) return nullptr;
    a.device = device;
    const int status = f(a, stream);
    return a.bad ? nullptr : PyLong_FromLong(status);
  } catch (const std::exception& e) {  // (a tensor without memory of its own, for one)
    PyErr_Format(PyExc_RuntimeError, "%s: %s", name, e.what());
    return nullptr;
  }
}

PyObject* py_rope_qkv(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call<18>("rope_qkv", v, n, [](Args& a, void* stream) {
    const int B = a.size(13), Hq = a.size(14), Hkv = a.size(15), N = a.size(16), d = a.size(17);
    const double T = (double)B * N, nk = T * Hkv * d;
    const Rows r = rows_of(a, 0, T, ((double)Hq + 2.0 * Hkv) * d, d);
    void *const q = a.bf16(10, "q", T * Hq * d), *const k = a.bf16(11, "k", nk), *const w = a.bf16(12, "v", nk);
    return made(a, rope_qkv, r.qkv, r.ld, r.wq, r.wk, r.eps, r.table, r.npos, r.rot, r.interleaved, r.pos, q, k, w, B, Hq, Hkv, N, d, stream);
  });
}

PyObject* py_rope_qkv_bwd(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call<23>("rope_qkv_bwd", v, n, [](Args& a, void* stream) {
    const int B = a.size(18), Hq = a.size(19), Hkv = a.size(20), N = a.size(21), d = a.size(22);
    const double T = (double)B * N, nk = T * Hkv * d, width = ((double)Hq + 2.0 * Hkv) * d;
    const bool norm = a.v[5] != Py_None || a.v[6] != Py_None;  // (without weights neither the rows nor the sums are looked at)
    const Rows r = rows_of(a, 3, T, width, d, norm);
    void *const dq = a.bf16(0, "dq", T * Hq * d), *const dk = a.bf16(1, "dk", nk), *const dv = a.bf16(2, "dv", nk);
    const long long dld = a.whole(14);
    void* const dqkv = a.rows(13, "dqkv", dld, T, width);
    float *const dwq = norm ? a.f32(15, "dq_weight", d) : nullptr, *const dwk = norm ? a.f32(16, "dk_weight", d) : nullptr;
    float* const ws = norm ? a.f32(17, "workspace", (double)(rope_qkv_bwd_workspace_bytes(B, Hq, Hkv, N, d) / 4)) : nullptr;
    return made(a, rope_qkv_bwd, dq, dk, dv, r.qkv, r.ld, r.wq, r.wk, r.eps, r.table, r.npos, r.rot, r.interleaved, r.pos, dqkv, dld, dwq, dwk, ws, B, Hq, Hkv, N, d, stream);
  });
}

PyObject* py_kv_append(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call<26>("kv_append", v, n, [](Args& a, void* stream) {
    const int T = a.size(15), S = a.size(16), Hq = a.size(17), Hkv = a.size(18), d = a.size(19), W = a.size(20), page = a.size(21), num = a.size(22), dtype = a.size(23);
    const float kd = a.real(24), vd = a.real(25);
    const double held = (double)num * Hkv * page * d;
    const Rows r = rows_of(a, 0, T, ((double)Hq + 2.0 * Hkv) * d, d);
    int *const seq = a.i32(10, "seq", T), *const pages = a.i32(11, "pages", (double)S * W);
    void *const q = a.bf16(12, "q", (double)T * Hq * d), *const k = a.cache(13, "k_cache", dtype, held), *const w = a.cache(14, "v_cache", dtype, held);
    return made(a, kv_append, r.qkv, r.ld, r.wq, r.wk, r.eps, r.table, r.npos, r.rot, r.interleaved, r.pos, seq, pages, q, k, w, T, S, Hq, Hkv, d, W, page, num, dtype, kd, vd, stream);
  });
}

PyObject* py_kv_decode(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return call<19>("kv_decode", v, n, [](Args& a, void* stream) {
    const int B = a.size(8), Hq = a.size(9), Hkv = a.size(10), d = a.size(11), W = a.size(12), page = a.size(13), num = a.size(14), dtype = a.size(16);
    const float scale = a.real(15), kd = a.real(17), vd = a.real(18);
    const double held = (double)num * Hkv * page * d, rows = (double)B * Hq;
    void *const q = a.bf16(0, "q", rows * d), *const k = a.cache(1, "k_cache", dtype, held), *const w = a.cache(2, "v_cache", dtype, held);
    int *const pages = a.i32(3, "pages", (double)B * W), *const lens = a.i32(4, "lens", B);
    void* const o = a.bf16(5, "o", rows * d);
    float *const lse = a.f32(6, "lse", rows), *const ws = a.f32(7, "workspace", (double)(kv_decode_workspace_bytes(B, Hq, Hkv, d) / 4));
    return made(a, kv_decode, q, k, w, pages, lens, o, lse, ws, B, Hq, Hkv, d, W, page, num, scale, dtype, kd, vd, stream);
  });
}

PyMethodDef methods[] = {
    {"rope_qkv", (PyCFunction)(void (*)())py_rope_qkv, METH_FASTCALL, nullptr},
    {"rope_qkv_bwd", (PyCFunction)(void (*)())py_rope_qkv_bwd, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)())py_kv_append, METH_FASTCALL, nullptr},
    {"kv_decode", (PyCFunction)(void (*)())py_kv_decode, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (tensors are read by their layout in memory: built_for_torch, the version that this was built for, is compared by kv.py)
PyMODINIT_FUNC PyInit__kv_call() {
  PyObject* const m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for_torch", BUILT_FOR_TORCH) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
