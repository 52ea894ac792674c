// Argument marshalling of the calls on a cache in a microscaling format (n5), as a CPython extension.  A step makes two or three
// of these calls per layer, and a small one's kernel takes about as long as Python needs to look at a dozen tensors and ctypes to
// convert some twenty-five arguments.  An append and a read of a short prompt in a row take 16.4 us that way and 9.1 us this
// way, four commits and reads 65 and 34.  Addresses of the C entry points come from api.py, and so does the function that turns
// an error code into an exception.
#include <Python.h>

#include <ATen/ops/empty_like.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include "ss.h"

namespace {

// api._check; torch's current device and that device's current stream (handle); api.ss_msa_mx_workspace
PyObject *g_check, *g_device, *g_stream, *g_workspace;
decltype(&ss_kv_append_mx) g_append;
decltype(&ss_kv_commit_mx) g_commit;
decltype(&ss_kv_read_mx) g_read;
decltype(&ss_msa_attention_mx) g_attend;

struct Raised {};  // a Python exception is set
thread_local int g_on;  // device of the call's tensors; -1 before the first
#define REFUSE(type, ...)           \
  do {                              \
    PyErr_Format(type, __VA_ARGS__); \
    throw Raised();                 \
  } while (0)

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) REFUSE(PyExc_TypeError, "%s must be a tensor", name);
  return THPVariable_Unpack(o);
}
const char* name_of(at::ScalarType t) {
  return t == at::kInt ? "torch.int32" : t == at::kByte ? "torch.uint8" : t == at::kFloat ? "torch.float32" : "torch.bfloat16";
}
void* ptr(const at::Tensor& t, at::ScalarType type, const char* name) {
  if (!(t.is_cuda() && t.is_contiguous() && t.scalar_type() == type))
    REFUSE(PyExc_TypeError, "%s must be a contiguous GPU tensor of dtype %s", name, name_of(type));
  const int on = t.device().index();
  if (g_on < 0) g_on = on;
  if (on != g_on) REFUSE(PyExc_ValueError, "%s is on device %d, tensors before it on device %d", name, on, g_on);
  return t.data_ptr();
}
int32_t* ints(const at::Tensor& t, const char* name) { return (int32_t*)ptr(t, at::kInt, name); }
int32_t* lens(PyObject* o, int64_t B, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.dim() != 1 || t.size(0) != B) REFUSE(PyExc_ValueError, "%s must be [B]", name);
  return ints(t, name);
}
bool is(const at::Tensor& t, int64_t a, int64_t b, int64_t c, int64_t d) {
  return t.dim() == 4 && t.size(0) == a && t.size(1) == b && t.size(2) == c && t.size(3) == d;
}
int small(int64_t v, const char* name) {
  if (v < INT32_MIN || v > INT32_MAX) REFUSE(PyExc_ValueError, "%s does not fit 32 bits", name);
  return (int)v;
}
int number(PyObject* o, const char* name) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return small(v, name);
}
// Rows [B,S or R,Hkv,D] in fp32 or bf16, both of one type.
int row_type(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return SS_F32;
  if (t.scalar_type() == at::kBFloat16) return SS_BF16;
  REFUSE(PyExc_TypeError, "rows must be fp32 or bf16");
}
void four(const at::Tensor& t, const char* name) {
  if (t.dim() != 4) REFUSE(PyExc_ValueError, "%s must have four dimensions", name);
}

struct Cache {  // the format follows from the bytes of a row
  void *k, *ks, *v, *vs;
  int32_t* table;
  int max_pages, num_pages, page, format;
  Cache(PyObject* const* a, int64_t B, int64_t Hkv, int64_t D) {
    const at::Tensor &tk = tensor(a[0], "k_cache"), &tks = tensor(a[1], "k_scale"), &tv = tensor(a[2], "v_cache"), &tvs = tensor(a[3], "v_scale"),
                     &tt = tensor(a[4], "block_table");
    four(tk, "k_cache");
    const int64_t P = tk.size(0), pg = tk.size(2), row = tk.size(3);
    if (row != D && row != D / 2) REFUSE(PyExc_ValueError, "rows of k_cache must be D bytes (8 bits) or D/2 (4 bits)");
    if (!is(tk, P, Hkv, pg, row) || !is(tv, P, Hkv, pg, row)) REFUSE(PyExc_ValueError, "k_cache and v_cache must be [P,Hkv,page,D or D/2]");
    if (!is(tks, P, Hkv, pg, D / 32) || !is(tvs, P, Hkv, pg, D / 32)) REFUSE(PyExc_ValueError, "k_scale and v_scale must be [P,Hkv,page,D/32]");
    if (tt.dim() != 2 || tt.size(0) != B) REFUSE(PyExc_ValueError, "block_table batch size mismatch");
    k = ptr(tk, at::kByte, "k_cache");
    ks = ptr(tks, at::kByte, "k_scale");
    v = ptr(tv, at::kByte, "v_cache");
    vs = ptr(tvs, at::kByte, "v_scale");
    table = ints(tt, "block_table");
    max_pages = small(tt.size(1), "max_pages");
    num_pages = small(P, "num_pages");
    page = small(pg, "page");
    format = row == D ? SS_KV_MXFP8 : SS_KV_MXFP4;
  }
};

// The current stream, of the device that the tensors are on.  Asked for once they are known to be fit: without a GPU it is
// their refusal that a caller should see.
void* stream() {
  PyObject* dev = PyObject_CallNoArgs(g_device);
  if (!dev) throw Raised();
  const long current = PyLong_AsLong(dev);
  if (current != g_on) {
    Py_DECREF(dev);
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "tensors on device %d, but the current device is %ld", g_on, current);
    throw Raised();
  }
  PyObject* st = PyObject_CallOneArg(g_stream, dev);
  Py_DECREF(dev);
  if (!st) throw Raised();
  void* p = PyLong_AsVoidPtr(st);
  Py_DECREF(st);
  if (!p && PyErr_Occurred()) throw Raised();
  return p;
}
void checked(int rc) {
  if (rc == SS_OK) return;
  PyObject* r = PyObject_CallFunction(g_check, "i", rc);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "libss error");
  throw Raised();
}
PyObject* same(PyObject* o) {
  Py_INCREF(o);
  return o;
}
// new_seq_lens: the caller's, or a tensor made like seq_lens.
PyObject* new_lens(PyObject* given, PyObject* seq_lens) {
  return given != Py_None ? same(given) : THPVariable_Wrap(at::empty_like(tensor(seq_lens, "seq_lens")));
}

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  HANDLE_TH_ERRORS
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, want);
    return nullptr;
  }
  g_on = -1;
  try {
    return f();
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
struct Owned {  // released unless handed out
  PyObject* o;
  ~Owned() { Py_XDECREF(o); }
  PyObject* out() {
    PyObject* r = o;
    o = nullptr;
    return r;
  }
};

// k_rows, v_rows, k_cache, k_scale, v_cache, v_scale, block_table, seq_lens, n_rows, new_seq_lens or None
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[0], "k_rows"), &v = tensor(a[1], "v_rows");
    four(k, "k_rows");
    const int64_t B = k.size(0), S = k.size(1), Hkv = k.size(2), D = k.size(3);
    if (!v.sizes().equals(k.sizes())) REFUSE(PyExc_ValueError, "k_rows and v_rows must have one shape");
    const Cache c(a + 2, B, Hkv, D);
    const int dtype = row_type(k);
    void *kp = ptr(k, k.scalar_type(), "k_rows"), *vp = ptr(v, k.scalar_type(), "v_rows");
    int32_t *sl = lens(a[7], B, "seq_lens"), *nr = lens(a[8], B, "n_rows");
    Owned out{new_lens(a[9], a[7])};
    checked(g_append(kp, vp, c.k, c.ks, c.v, c.vs, c.table, c.max_pages, c.num_pages, sl, nr, small(B, "B"), small(S, "S"), small(Hkv, "Hkv"),
                     small(D, "D"), c.page, dtype, c.format, lens(out.o, B, "new_seq_lens"), stream()));
    return out.out();
  });
}

// k_new, v_new, k_cache, k_scale, v_cache, v_scale, block_table, seq_lens, path, n_accept, gamma, new_seq_lens or None
PyObject* commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[0], "k_new"), &v = tensor(a[1], "v_new"), &path = tensor(a[8], "path");
    four(k, "k_new");
    const int gamma = number(a[10], "gamma");
    const int64_t B = k.size(0), R = k.size(1), Hkv = k.size(2), D = k.size(3), per = 1 + (int64_t)gamma, T = gamma < 0 ? 0 : R / per;
    if (gamma < 0 || R != T * per || !v.sizes().equals(k.sizes())) REFUSE(PyExc_ValueError, "k_new / v_new must be [B,T*(1+gamma),Hkv,D]");
    if (path.dim() != 2 || path.size(0) != B) REFUSE(PyExc_ValueError, "path must be [B,max_depth+1]");
    const Cache c(a + 2, B, Hkv, D);
    const int dtype = row_type(k);
    void *kp = ptr(k, k.scalar_type(), "k_new"), *vp = ptr(v, k.scalar_type(), "v_new");
    int32_t *sl = lens(a[7], B, "seq_lens"), *pp = ints(path, "path"), *na = lens(a[9], B, "n_accept");
    Owned out{new_lens(a[11], a[7])};
    checked(g_commit(kp, vp, c.k, c.ks, c.v, c.vs, c.table, c.max_pages, c.num_pages, sl, pp, na, small(B, "B"), small(T, "T"), gamma,
                     small(Hkv, "Hkv"), small(D, "D"), c.page, small(path.size(1) - 1, "max_depth"), dtype, c.format,
                     lens(out.o, B, "new_seq_lens"), stream()));
    return out.out();
  });
}

// k_cache, k_scale, v_cache, v_scale, block_table, seq_lens, k_rows, v_rows, first or None
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const at::Tensor &k = tensor(a[6], "k_rows"), &v = tensor(a[7], "v_rows");
    four(k, "k_rows");
    const int64_t B = k.size(0), S = k.size(1), Hkv = k.size(2), D = k.size(3);
    if (!v.sizes().equals(k.sizes())) REFUSE(PyExc_ValueError, "k_rows and v_rows must have one shape");
    const Cache c(a, B, Hkv, D);
    int32_t *first = a[8] == Py_None ? nullptr : lens(a[8], B, "first"), *sl = lens(a[5], B, "seq_lens");
    const int dtype = row_type(k);
    void *kp = ptr(k, k.scalar_type(), "k_rows"), *vp = ptr(v, k.scalar_type(), "v_rows");
    checked(g_read(c.k, c.ks, c.v, c.vs, c.table, c.max_pages, c.num_pages, first, sl, small(B, "B"), small(S, "S"), small(Hkv, "Hkv"),
                   small(D, "D"), c.page, dtype, c.format, kp, vp, stream()));
    return PyTuple_Pack(2, a[6], a[7]);
  });
}

// q, k_new, v_new, k_cache, k_scale, v_cache, v_scale, block_table, seq_lens, parent, gamma, scale, flags, out, workspace, n_nodes (the last
// three or None)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 16, [&]() -> PyObject* {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k_new"), &v = tensor(a[2], "v_new"), &parent = tensor(a[9], "parent");
    four(q, "q");
    four(k, "k_new");
    const int64_t B = q.size(0), R = q.size(1), H = q.size(2), D = q.size(3), Hkv = k.size(2);
    const int gamma = number(a[10], "gamma");
    if (parent.dim() != 2 || parent.size(0) != B) REFUSE(PyExc_ValueError, "parent batch size mismatch");
    const int64_t T = parent.size(1);
    if (R != T * (1 + (int64_t)gamma) || !is(k, B, R, Hkv, D) || !is(v, B, R, Hkv, D))
      REFUSE(PyExc_ValueError, "q / k_new / v_new shapes do not match B,R,H,Hkv,D");
    const Cache c(a + 3, B, Hkv, D);
    Owned out{a[13] != Py_None ? same(a[13]) : THPVariable_Wrap(at::empty_like(q))};
    const at::Tensor& o = tensor(out.o, "out");
    if (!o.sizes().equals(q.sizes())) REFUSE(PyExc_ValueError, "out must have q's shape");
    const double scale = PyFloat_AsDouble(a[11]);
    if (scale == -1.0 && PyErr_Occurred()) throw Raised();
    const int flags = number(a[12], "flags");
    void *qp = ptr(q, at::kBFloat16, "q"), *kp = ptr(k, at::kBFloat16, "k_new"), *vp = ptr(v, at::kBFloat16, "v_new");
    int32_t *sl = lens(a[8], B, "seq_lens"), *pa = ints(parent, "parent"), *nn = a[15] == Py_None ? nullptr : lens(a[15], B, "n_nodes");
    void* op = ptr(o, at::kBFloat16, "out");
    void* const st = stream();
    Owned made{nullptr};
    if (a[14] == Py_None) {
      PyObject* dev = PyObject_GetAttrString(a[0], "device");
      if (!dev) throw Raised();
      made.o = PyObject_CallFunction(g_workspace, "LLiLLLLN", (long long)B, (long long)T, gamma, (long long)H, (long long)Hkv, (long long)D,
                                     (long long)c.max_pages * c.page, dev);
      if (!made.o) throw Raised();
    }
    const at::Tensor& ws = tensor(made.o ? made.o : a[14], "workspace");
    void* wp = ptr(ws, at::kByte, "workspace");
    checked(g_attend(qp, kp, vp, c.k, c.ks, c.v, c.vs, c.table, c.max_pages, c.num_pages, sl, pa, nn, small(B, "B"), small(T, "T"), gamma,
                     small(H, "H"), small(Hkv, "Hkv"), small(D, "D"), c.page, (float)scale, c.format, (uint32_t)flags, op, wp,
                     (size_t)ws.numel(), st));
    return out.out();
  });
}

// check, current device, its current stream, workspace, addresses of the entry points in the order append, commit, read, attend
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    void* at[4];
    for (int i = 0; i < 4; ++i) {
      at[i] = PyLong_AsVoidPtr(a[4 + i]);
      if (!at[i] && PyErr_Occurred()) throw Raised();
    }
    g_append = (decltype(g_append))at[0];
    g_commit = (decltype(g_commit))at[1];
    g_read = (decltype(g_read))at[2];
    g_attend = (decltype(g_attend))at[3];
    g_check = same(a[0]);
    g_device = same(a[1]);
    g_stream = same(a[2]);
    g_workspace = same(a[3]);
    Py_RETURN_NONE;
  });
}

PyMethodDef kMethods[] = {{"init", (PyCFunction)(void (*)(void))init, METH_FASTCALL, nullptr},
                          {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
                          {"commit", (PyCFunction)(void (*)(void))commit, METH_FASTCALL, nullptr},
                          {"read", (PyCFunction)(void (*)(void))read, METH_FASTCALL, nullptr},
                          {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "ss_bind", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_ss_bind() { return PyModule_Create(&kModule); }
