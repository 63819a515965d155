// CPython entries to the operators around the cache for binding.py: they read torch tensors and host arrays, check what the C functions cannot see
// (element types, shapes, devices, lengths of host arrays) and call them.  A serving step makes three of these calls for every layer, and
// building ctypes structures took 5 to 11 us a call; here it is one to two.  Nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include "../../include/hack.h"

namespace {

PyObject *s_get_device, *s_is_contiguous, *s_data_ptr, *s_shape, *s_stride, *s_dtype, *s_k, *s_v, *s_pos, *s_off, *s_len;

bool refuse(const char* text) {
  PyErr_SetString(PyExc_AssertionError, text);
  return false;
}

// What a Hack object knows about its context.
struct Info {
  long head_dim, heads, device;
  PyObject *type, *f32, *i32, *u8;
};
bool read_info(PyObject* t, Info* i) {
  if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 7) return refuse("info has seven entries");
  i->head_dim = PyLong_AsLong(PyTuple_GET_ITEM(t, 0));
  i->heads = PyLong_AsLong(PyTuple_GET_ITEM(t, 1));
  i->device = PyLong_AsLong(PyTuple_GET_ITEM(t, 2));
  i->type = PyTuple_GET_ITEM(t, 3);
  i->f32 = PyTuple_GET_ITEM(t, 4);
  i->i32 = PyTuple_GET_ITEM(t, 5);
  i->u8 = PyTuple_GET_ITEM(t, 6);
  return !PyErr_Occurred();
}

constexpr int kDims = 4;
struct View {
  void* p;
  int dim;
  int64_t shape[kDims], stride[kDims];
  bool is(int64_t a, int64_t b, int64_t c, int64_t d) const { return dim == 4 && shape[0] == a && shape[1] == b && shape[2] == c && shape[3] == d; }
};

bool read_sizes(PyObject* t, int64_t* v, int* dim) {   // steals t
  if (!t) return false;
  PyObject* f = PySequence_Fast(t, "sizes");
  Py_DECREF(t);
  if (!f) return false;
  *dim = (int)PySequence_Fast_GET_SIZE(f);
  for (int i = 0; i < *dim && i < kDims; ++i) v[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(f, i));
  Py_DECREF(f);
  return !PyErr_Occurred();
}

// A device tensor of the context's device and the given element type; contiguous unless its strides are asked for.
bool read_tensor(PyObject* t, const Info& info, PyObject* type, bool strides, View* v) {
  PyObject* o = PyObject_CallMethodNoArgs(t, s_get_device);
  if (!o) return false;
  const long device = PyLong_AsLong(o);
  Py_DECREF(o);
  if (device == -1 && PyErr_Occurred()) return false;
  if (device != info.device) return refuse("device tensors must lie on the context's device");
  o = PyObject_GetAttr(t, s_dtype);
  if (!o) return false;
  const bool typed = o == type;
  Py_DECREF(o);
  if (!typed) return refuse("a tensor has another element type than the call takes");
  if (!read_sizes(PyObject_GetAttr(t, s_shape), v->shape, &v->dim)) return false;
  if (strides) {
    int n;
    if (!read_sizes(PyObject_CallMethodNoArgs(t, s_stride), v->stride, &n)) return false;
  } else {
    o = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!o) return false;
    const int ok = PyObject_IsTrue(o);
    Py_DECREF(o);
    if (ok < 0) return false;
    if (!ok) return refuse("device tensors must be contiguous CUDA/HIP tensors");
  }
  o = PyObject_CallMethodNoArgs(t, s_data_ptr);
  if (!o) return false;
  v->p = PyLong_AsVoidPtr(o);
  Py_DECREF(o);
  return !PyErr_Occurred();
}

// A contiguous host array of at least n elements of a struct-module type code.
struct HostArray {
  Py_buffer b{};
  bool held = false;
  ~HostArray() { if (held) PyBuffer_Release(&b); }
  bool is(PyObject* o, char code, char other) {   // false, without an exception, for any other object
    if (PyObject_GetBuffer(o, &b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) {
      PyErr_Clear();
      return false;
    }
    held = true;
    return b.format && (b.format[0] == code || b.format[0] == other) && b.format[1] == 0;
  }
  int64_t count() const { return b.len / b.itemsize; }
};

// A Cache or PackedCache object as the structure that the C functions take.
template <typename T> struct CacheArgs {
  T c{};
  HostArray off, len;
  bool read(PyObject* o, const Info& info, PyObject* type, int64_t units, int64_t width, int64_t rows_each) {
    View k, v, pos;
    PyObject* t = PyObject_GetAttr(o, s_k);
    bool ok = t && read_tensor(t, info, type, false, &k);
    Py_XDECREF(t);
    if (!ok) return false;
    t = PyObject_GetAttr(o, s_v);
    ok = t && read_tensor(t, info, type, false, &v);
    Py_XDECREF(t);
    if (!ok) return false;
    if (k.dim != 2 || v.dim != 2 || k.shape[1] != width || v.shape[1] != width || k.shape[0] != v.shape[0]) return refuse("a cache has another head_dim or K and V differ");
    t = PyObject_GetAttr(o, s_pos);
    if (!t) return false;
    ok = true;
    if (t != Py_None) {
      ok = read_tensor(t, info, info.i32, false, &pos);
      if (ok && (pos.dim != 1 || pos.shape[0] < k.shape[0] * rows_each)) ok = refuse("pos has an entry for every row");
      c.pos = static_cast<int32_t*>(pos.p);
    }
    Py_DECREF(t);
    if (!ok) return false;
    t = PyObject_GetAttr(o, s_off);
    ok = t && (off.is(t, 'l', 'q') || refuse("off is an int64 array"));
    Py_XDECREF(t);
    if (!ok) return false;
    t = PyObject_GetAttr(o, s_len);
    ok = t && (len.is(t, 'i', 'i') || refuse("len is an int32 array"));
    Py_XDECREF(t);
    if (!ok) return false;
    if (off.count() != units || len.count() != units) return refuse("a cache has an offset and a length for every unit");
    c.k = k.p;
    c.v = v.p;
    c.rows = k.shape[0] * rows_each;
    c.off = static_cast<const int64_t*>(off.b.buf);
    c.len = static_cast<const int32_t*>(len.b.buf);
    return true;
  }
};
typedef CacheArgs<hack_cache> RowCache;
typedef CacheArgs<hack_packed_cache> Packed;
bool read_rows(RowCache& a, PyObject* o, const Info& i, int64_t units) { return a.read(o, i, i.type, units, i.head_dim, 1); }
bool read_packed(Packed& a, PyObject* o, const Info& i, int64_t units) { return a.read(o, i, i.u8, units, 34 * i.head_dim, 64); }

void* address(PyObject* o) { return o == Py_None ? nullptr : PyLong_AsVoidPtr(o); }
bool int32_arg(PyObject* o, int32_t* v) {
  const long x = PyLong_AsLong(o);
  *v = (int32_t)x;
  if (PyErr_Occurred()) return false;
  if (x < INT32_MIN || x > INT32_MAX) PyErr_SetString(PyExc_OverflowError, "a number of more than 32 bits");
  return x >= INT32_MIN && x <= INT32_MAX;
}
bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "takes %zd arguments", want);
  return false;
}

// One operand of a rotation: x [B, heads, N, head_dim] in any strides with the head's elements side by side, out contiguous.
bool read_operand(PyObject* x, PyObject* out, PyObject* weight, const Info& info, hack_rows* r, int64_t* B, int64_t* N) {
  View a, o, w;
  if (!read_tensor(x, info, info.type, true, &a) || !read_tensor(out, info, info.type, false, &o)) return false;
  if (a.dim != 4 || a.shape[3] != info.head_dim || a.stride[3] != 1) return refuse("rows: [B, heads, N, head_dim], head_dim side by side");
  if (!o.is(a.shape[0], a.shape[1], a.shape[2], a.shape[3])) return refuse("out: the shape of x");
  if (a.shape[1] > INT32_MAX || a.shape[0] > INT32_MAX || a.shape[2] > INT32_MAX) return refuse("rows: too many of them");
  *r = hack_rows{a.p, o.p, (int32_t)a.shape[1], 0, 0, 0, nullptr, 0};
  // a dimension of one element may have any stride
  if (a.shape[0] > 1) r->stride_b = a.stride[0];
  if (a.shape[1] > 1) r->stride_h = a.stride[1];
  if (a.shape[2] > 1) r->stride_n = a.stride[2];
  if (weight != Py_None) {
    if (!read_tensor(weight, info, info.f32, false, &w)) return false;
    if (!(w.dim == 1 && w.shape[0] == info.head_dim) && !(w.dim == 2 && w.shape[0] == a.shape[1] && w.shape[1] == info.head_dim))
      return refuse("weight: [head_dim] or [heads, head_dim]");
    r->weight = static_cast<const float*>(w.p);
    r->weight_stride_h = w.dim == 2 ? info.head_dim : 0;
  }
  *B = a.shape[0];
  *N = a.shape[2];
  return true;
}

// rotate(fn, ctx, info, q, q_out, q_weight, k, k_out, k_weight, norm, eps, rope, axes, pos, pos0, stream) -> status; norm < 0: fn is hack_rotate, else
// hack_norm_rotate.
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 16)) return nullptr;
  Info info;
  if (!read_info(a[2], &info)) return nullptr;
  void *fn = address(a[0]), *ctx = address(a[1]), *rope = address(a[11]), *stream = address(a[15]);
  const long norm = PyLong_AsLong(a[9]), axes = PyLong_AsLong(a[12]);
  const double eps = PyFloat_AsDouble(a[10]);
  int32_t pos0;
  if (PyErr_Occurred() || !int32_arg(a[14], &pos0)) return nullptr;
  hack_rows q, k;
  int64_t B, N, Bk, Nk;
  if (!read_operand(a[3], a[4], a[5], info, &q, &B, &N)) return nullptr;
  const bool two = a[6] != Py_None;
  if (two) {
    if (!read_operand(a[6], a[7], a[8], info, &k, &Bk, &Nk)) return nullptr;
    if (Bk != B || Nk != N) {
      refuse("q and k: the same batch and rows");
      return nullptr;
    }
  }
  const int32_t* pos = nullptr;
  int64_t stride = 0;
  if (rope && a[13] != Py_None) {   // [axes, N], the same for all batch elements, or [B, axes, N]; with one axis also [N]
    View p;
    if (!read_tensor(a[13], info, info.i32, false, &p)) return nullptr;
    const bool each = p.dim == 3 && p.shape[0] == B && p.shape[1] == axes && p.shape[2] == N;
    if (!each && !(p.dim == 2 && p.shape[0] == axes && p.shape[1] == N) && !(p.dim == 1 && axes == 1 && p.shape[0] == N)) {
      refuse("positions: [axes, N] or [B, axes, N]");
      return nullptr;
    }
    pos = static_cast<const int32_t*>(p.p);
    stride = each ? axes * N : 0;
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  if (norm < 0)
    status = reinterpret_cast<decltype(&hack_rotate)>(fn)((hack_ctx*)ctx, (int32_t)B, (int32_t)N, &q, (const hack_rope*)rope, pos, stride, pos0, stream);
  else
    status = reinterpret_cast<decltype(&hack_norm_rotate)>(fn)((hack_ctx*)ctx, (int32_t)B, (int32_t)N, &q, two ? &k : nullptr, (int32_t)norm, (float)eps,
                                                              (const hack_rope*)rope, pos, stride, pos0, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// A host array of a row number for every unit, int32 or int64; None: NULL.  Sets convert for another object, which the caller makes one of.
struct First {
  HostArray a;
  int32_t* own = nullptr;
  const int32_t* p = nullptr;
  bool convert = false;
  ~First() { PyMem_Free(own); }
  bool read(PyObject* o, int64_t units) {
    if (o == Py_None) return true;
    const bool narrow = a.is(o, 'i', 'i');
    if (!narrow && !(a.held && a.b.format && (a.b.format[0] == 'l' || a.b.format[0] == 'q') && a.b.format[1] == 0 && a.b.itemsize == 8)) {
      convert = true;
      return true;
    }
    if (a.count() != units) return refuse("a row number for every unit");
    if (narrow) {
      p = static_cast<const int32_t*>(a.b.buf);
      return true;
    }
    p = own = static_cast<int32_t*>(PyMem_Malloc(units * sizeof(int32_t) + 1));
    if (!own) {
      PyErr_NoMemory();
      return false;
    }
    const int64_t* from = static_cast<const int64_t*>(a.b.buf);
    bool fits = true;
    for (int64_t i = 0; i < units; ++i) {
      own[i] = (int32_t)from[i];
      fits &= own[i] == from[i];
    }
    if (!fits) PyErr_SetString(PyExc_OverflowError, "a number of more than 32 bits");
    return fits;
  }
};

// pack(fn, ctx, info, B, N_k, cache_in, k_new, v_new, pos_new, kept, first, packed, stream) -> status, None where first is no array of integers
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 13)) return nullptr;
  Info info;
  if (!read_info(a[2], &info)) return nullptr;
  void *fn = address(a[0]), *ctx = address(a[1]), *stream = address(a[12]);
  int32_t B, N_k, pos_new;
  if (!int32_arg(a[3], &B) || !int32_arg(a[4], &N_k) || !int32_arg(a[8], &pos_new)) return nullptr;
  const int64_t units = (int64_t)B * info.heads;
  First first;
  if (!first.read(a[10], units)) return nullptr;
  if (first.convert) Py_RETURN_NONE;
  RowCache in;
  Packed out;
  if (a[5] != Py_None && !read_rows(in, a[5], info, units)) return nullptr;
  if (!read_packed(out, a[11], info, units)) return nullptr;
  View k{}, v{}, kept{};
  for (int i = 0; i < 2; ++i) {
    View& x = i ? v : k;
    if (a[6 + i] == Py_None) continue;
    if (!read_tensor(a[6 + i], info, info.type, false, &x)) return nullptr;
    if (!x.is(B, info.heads, N_k, info.head_dim)) {
      refuse("new rows: [B, heads, N_k, head_dim]");
      return nullptr;
    }
  }
  if (a[9] != Py_None) {
    if (!read_tensor(a[9], info, info.i32, false, &kept)) return nullptr;
    if (kept.dim != 2 || kept.shape[0] != units) {
      refuse("kept_idx: a row for every unit");
      return nullptr;
    }
    // without columns the tensor has no address; NULL would say that there is no list, and the rows come in order
    static int32_t nothing;
    if (!kept.p) kept.p = &nothing;
  }
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = reinterpret_cast<decltype(&hack_pack)>(fn)((hack_ctx*)ctx, B, N_k, a[5] == Py_None ? nullptr : &in.c, k.p, v.p, pos_new, (const int32_t*)kept.p,
                                                     kept.p ? kept.shape[1] : 0, first.p, &out.c, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// unpack(fn, ctx, info, B, packed, first, out, stream) -> status, None where first is no array of integers
PyObject* unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  Info info;
  if (!read_info(a[2], &info)) return nullptr;
  void *fn = address(a[0]), *ctx = address(a[1]), *stream = address(a[7]);
  int32_t B;
  if (!int32_arg(a[3], &B)) return nullptr;
  const int64_t units = (int64_t)B * info.heads;
  First first;
  if (!first.read(a[5], units)) return nullptr;
  if (first.convert) Py_RETURN_NONE;
  Packed in;
  RowCache out;
  if (!read_packed(in, a[4], info, units) || !read_rows(out, a[6], info, units)) return nullptr;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = reinterpret_cast<decltype(&hack_unpack)>(fn)((hack_ctx*)ctx, B, &in.c, first.p, &out.c, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// attn(fn, ctx, info, q, packed, scale, out, stream) -> status
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arity(n, 8)) return nullptr;
  Info info;
  if (!read_info(a[2], &info)) return nullptr;
  void *fn = address(a[0]), *ctx = address(a[1]), *stream = address(a[7]);
  const double scale = PyFloat_AsDouble(a[5]);
  if (PyErr_Occurred()) return nullptr;
  View q, out;
  if (!read_tensor(a[3], info, info.type, false, &q) || !read_tensor(a[6], info, info.type, false, &out)) return nullptr;
  if (q.dim != 4 || q.shape[3] != info.head_dim || q.shape[1] % info.heads != 0 || !out.is(q.shape[0], q.shape[1], q.shape[2], q.shape[3])) {
    refuse("q and out: [B, G heads, N, head_dim]");
    return nullptr;
  }
  const int64_t N_k = q.shape[1] / info.heads * q.shape[2];
  if (N_k > INT32_MAX || q.shape[0] > INT32_MAX) {
    refuse("q: too many rows");
    return nullptr;
  }
  Packed kv;
  if (!read_packed(kv, a[4], info, q.shape[0] * info.heads)) return nullptr;
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = reinterpret_cast<decltype(&hack_attn_packed)>(fn)((hack_ctx*)ctx, (int32_t)q.shape[0], (int32_t)N_k, q.p, &kv.c, (float)scale, out.p, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

#define ENTRY(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(rotate), ENTRY(pack), ENTRY(unpack), ENTRY(attn), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_call() {
  struct { PyObject** s; const char* name; } names[] = {{&s_get_device, "get_device"}, {&s_is_contiguous, "is_contiguous"}, {&s_data_ptr, "data_ptr"},
                                                        {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_k, "k"}, {&s_v, "v"},
                                                        {&s_pos, "pos"}, {&s_off, "off"}, {&s_len, "len"}};
  for (auto& x : names)
    if (!(*x.s = PyUnicode_InternFromString(x.name))) return nullptr;
  return PyModule_Create(&module);
}
