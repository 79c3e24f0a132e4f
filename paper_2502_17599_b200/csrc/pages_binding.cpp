// Argument marshalling of the paged-cache calls (binding.Pages): checks torch tensors against a handle's geometry and
// passes their addresses to the C ABI (include/meda.h).  A decoding step makes a few of these calls per layer, each around a
// kernel of a few microseconds; the same checks in Python cost 5 us a call, here 0.5 us.  No arithmetic
// lives here, and the C functions are reached through the addresses binding.py took from libmeda.so.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/cuda/CUDAStream.h>

#include <exception>
#include <initializer_list>
#include <sstream>
#include <string>

#include "../../include/meda.h"

namespace {

struct Refused : std::exception {
  std::string text;
  explicit Refused(std::string t) : text(std::move(t)) {}
  const char* what() const noexcept override { return text.c_str(); }
};

struct Native {
  meda_pages* h = nullptr;
  int device = 0;
  at::ScalarType dtype = at::kFloat;
  int64_t n_pages = 0, width = 0, hq = 0, hkv = 0, page = 0, d = 0;
  decltype(&meda_page_tables) page_tables = nullptr;
  decltype(&meda_page_store) page_store = nullptr;
  decltype(&meda_page_bounds) page_bounds = nullptr;
  decltype(&meda_rope_append) rope_append = nullptr;
  decltype(&meda_select_pages) select_pages = nullptr;
  decltype(&meda_paged_attention) paged_attention = nullptr;
};

const char* kCapsule = "meda.pages";

Native* native_of(PyObject* o) {
  auto* n = static_cast<Native*>(PyCapsule_GetPointer(o, kCapsule));
  if (!n) throw Refused("not a handle of paged caches");
  if (!n->h) throw Refused("the handle has been closed");
  return n;
}

std::string shape_text(at::IntArrayRef s) {
  std::ostringstream o;
  o << "(";
  for (size_t i = 0; i < s.size(); ++i) o << (i ? ", " : "") << s[i];
  o << ")";
  return o.str();
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refused(std::string(what) + ": a tensor is wanted");
  return THPVariable_Unpack(o);
}

[[noreturn]] void refuse(const Native* n, const at::Tensor& t, at::ScalarType type, const std::string& wanted, const char* what) {
  std::ostringstream o;
  o << what << ": " << toString(type) << " " << wanted << " on cuda:" << n->device << " is wanted, got " << toString(t.scalar_type())
    << " " << shape_text(t.sizes()) << " with strides " << shape_text(t.strides()) << " on " << t.device().str();
  throw Refused(o.str());
}

bool on(const Native* n, const at::Tensor& t, at::ScalarType type) {
  return t.scalar_type() == type && t.is_cuda() && t.get_device() == n->device;
}

// Address of a contiguous tensor of the handle's device with this type and shape.
void* dense(const Native* n, PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (!on(n, t, type) || t.sizes() != at::IntArrayRef(shape.begin(), shape.size()) || !t.is_contiguous())
    refuse(n, t, type, "contiguous " + shape_text(at::IntArrayRef(shape.begin(), shape.size())), what);
  return t.data_ptr();
}

// 1-D int32 lengths of any stride.
const int32_t* lengths(const Native* n, const at::Tensor& t, int64_t count, const char* what) {
  if (!on(n, t, at::kInt) || t.dim() != 1 || t.size(0) != count) refuse(n, t, at::kInt, "[" + std::to_string(count) + "]", what);
  return static_cast<const int32_t*>(t.data_ptr());
}

int32_t small(int64_t x, const char* what) {
  if (x > INT32_MAX || x < INT32_MIN) throw Refused(std::string(what) + " does not fit 32 bits");
  return (int32_t)x;
}

// [n][heads][head_dim] rows that are dense inside a token: address and token stride.
void* heads_of(const Native* n, PyObject* o, int64_t count, int64_t heads, int64_t* stride, const char* what) {
  const at::Tensor& t = tensor(o, what);
  const int64_t want[3] = {count, heads, n->d};
  if (!on(n, t, n->dtype) || t.sizes() != at::IntArrayRef(want, 3) || t.stride(2) != 1 || (heads > 1 && t.stride(1) != n->d))
    refuse(n, t, n->dtype, shape_text(at::IntArrayRef(want, 3)) + " with dense heads", what);
  *stride = count > 1 ? t.stride(0) : 0;
  return t.data_ptr();
}

void* stream_of(const Native* n, PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)n->device).stream();
  PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
  if (!v) throw Refused("stream: a torch.cuda.Stream is wanted");
  void* p = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  if (PyErr_Occurred()) throw Refused("stream: a torch.cuda.Stream is wanted");
  return p;
}

int64_t whole(PyObject* o, const char* what) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Refused(std::string(what) + ": a whole number is wanted");
  return x;
}

using Args = PyObject* const*;

// One C call without the interpreter's lock: a launch waits where the stream's queue is full, and what it waits for may be
// a host function that needs the lock.  (The arguments, which may use the interpreter, are ready before it is let go.)
template <typename F, typename... A>
meda_status unlocked(F f, A... a) {
  PyThreadState* s = PyEval_SaveThread();
  const meda_status r = f(a...);
  PyEval_RestoreThread(s);
  return r;
}

meda_status page_tables(Args a) {              // lens, new_lens, free_pages, free_top, free_top_out, table, cu_new, slots, stream
  Native* n = native_of(a[0]);
  const at::Tensor& nl = tensor(a[2], "new_lens");
  if (nl.dim() != 1) refuse(n, nl, at::kInt, "[n]", "new_lens");
  const int64_t c = nl.size(0);
  const int32_t* new_lens = lengths(n, nl, c, "new_lens");
  const int32_t* lens = nullptr;
  int64_t stride = 0;
  if (a[1] != Py_None) {
    const at::Tensor& l = tensor(a[1], "lens");
    lens = lengths(n, l, c, "lens");
    stride = l.stride(0);
  }
  const at::Tensor& sl = tensor(a[8], "slots");
  if (!on(n, sl, at::kLong) || sl.dim() != 1 || !sl.is_contiguous()) refuse(n, sl, at::kLong, "contiguous [capacity]", "slots");
  return unlocked(n->page_tables, n->h, lens, small(stride, "stride"), new_lens, small(nl.stride(0), "stride"), small(c, "n_seqs"),
                        static_cast<int32_t*>(dense(n, a[3], at::kInt, {n->n_pages}, "free_pages")),
                        static_cast<const int32_t*>(dense(n, a[4], at::kInt, {1}, "free_top")),
                        static_cast<int32_t*>(dense(n, a[5], at::kInt, {1}, "free_top_out")),
                        static_cast<int32_t*>(dense(n, a[6], at::kInt, {c, n->width}, "table")),
                        static_cast<int32_t*>(dense(n, a[7], at::kInt, {c + 1}, "cu_new")),
                        static_cast<int64_t*>(sl.data_ptr()), sl.size(0), stream_of(n, a[9]));
}

meda_status page_store(Args a) {               // k, v, lens, table, k_pages, v_pages, bounds, stream
  Native* n = native_of(a[0]);
  const at::Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &l = tensor(a[3], "lens");
  if (l.dim() != 1) refuse(n, l, at::kInt, "[n]", "lens");
  const int64_t c = l.size(0);
  const auto alike = [&k](const at::Tensor& t) {  // (the stride of an axis of one element means nothing)
    for (int64_t x = 0; x < 4; ++x)
      if (t.size(x) != k.size(x) || (t.size(x) > 1 && t.stride(x) != k.stride(x))) return false;
    return true;
  };
  for (const at::Tensor* t : {&k, &v}) {
    const char* what = t == &k ? "k" : "v";
    if (!on(n, *t, n->dtype) || k.dim() != 4 || t->dim() != 4 || t->size(0) != c || t->size(1) != n->hkv || t->size(3) != n->d ||
        !alike(*t) || t->stride(3) != 1 || (t->size(2) > 1 && t->stride(2) != n->d))
      refuse(n, *t, n->dtype, "[" + std::to_string(c) + "][" + std::to_string(n->hkv) + "][capacity][" + std::to_string(n->d) +
             "], rows dense, k and v laid out alike,", what);
  }
  return unlocked(n->page_store, n->h, k.data_ptr(), v.data_ptr(), c > 1 ? k.stride(0) : 0, n->hkv > 1 ? k.stride(1) : 0, small(k.size(2), "capacity"),
                       lengths(n, l, c, "lens"), small(l.stride(0), "stride"), small(c, "n_seqs"),
                       static_cast<const int32_t*>(dense(n, a[4], at::kInt, {c, n->width}, "table")),
                       dense(n, a[5], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "k_pages"),
                       dense(n, a[6], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "v_pages"),
                       a[7] == Py_None ? nullptr : dense(n, a[7], n->dtype, {n->n_pages, n->hkv, 2, n->d}, "bounds"), stream_of(n, a[8]));
}

meda_status page_bounds(Args a) {              // k_pages, table, lens_from, lens, bounds, stream
  Native* n = native_of(a[0]);
  const at::Tensor& l = tensor(a[4], "lens");
  if (l.dim() != 1) refuse(n, l, at::kInt, "[n]", "lens");
  const int64_t c = l.size(0);
  const int32_t* from = nullptr;
  if (a[3] != Py_None) {
    const at::Tensor& f = tensor(a[3], "lens_from");
    from = lengths(n, f, c, "lens_from");
    if (c > 1 && f.stride(0) != l.stride(0)) throw Refused("lens_from and lens have to have the same stride");
  }
  return unlocked(n->page_bounds, n->h, dense(n, a[1], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "k_pages"),
                        static_cast<const int32_t*>(dense(n, a[2], at::kInt, {c, n->width}, "table")), from, lengths(n, l, c, "lens"),
                        small(l.stride(0), "stride"), small(c, "n_seqs"), dense(n, a[5], n->dtype, {n->n_pages, n->hkv, 2, n->d}, "bounds"),
                        stream_of(n, a[6]));
}

meda_status rope_append(Args a) {              // q, k, v, positions, slots, q_out, k_pages, v_pages, stream
  Native* n = native_of(a[0]);
  const at::Tensor& sl = tensor(a[5], "slots");
  if (!on(n, sl, at::kLong) || sl.dim() != 1 || !sl.is_contiguous()) refuse(n, sl, at::kLong, "contiguous [n_tokens]", "slots");
  const int64_t c = sl.size(0);
  int64_t qs = 0, ks = 0, vs = 0, ax = 0;
  const void* k = heads_of(n, a[2], c, n->hkv, &ks, "k");
  const void* v = heads_of(n, a[3], c, n->hkv, &vs, "v");
  const void* q = nullptr;
  void* q_out = nullptr;
  if (a[1] != Py_None) {
    q = heads_of(n, a[1], c, n->hq, &qs, "q");
    q_out = dense(n, a[6], n->dtype, {c, n->hq, n->d}, "q_out");
  } else if (a[6] != Py_None) {
    throw Refused("q_out without q");
  }
  const int32_t* pos = nullptr;
  if (a[4] != Py_None) {
    const at::Tensor& t = tensor(a[4], "positions");
    if (!on(n, t, at::kInt) || t.dim() != 2 || t.size(0) != 3 || t.size(1) != c || (c > 1 && t.stride(1) != 1))
      refuse(n, t, at::kInt, "[3][" + std::to_string(c) + "] with dense axes", "positions");
    pos = static_cast<const int32_t*>(t.data_ptr());
    ax = t.stride(0);
  }
  return unlocked(n->rope_append, n->h, q, qs, k, ks, v, vs, pos, ax, static_cast<const int64_t*>(sl.data_ptr()), small(c, "n_tokens"), q_out,
                        dense(n, a[7], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "k_pages"),
                        dense(n, a[8], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "v_pages"), stream_of(n, a[9]));
}

meda_status select_pages(Args a) {             // q, bounds, table, lens, n_first, n_last, sel, stream
  Native* n = native_of(a[0]);
  const at::Tensor &l = tensor(a[4], "lens"), &s = tensor(a[7], "sel");
  if (l.dim() != 1) refuse(n, l, at::kInt, "[n]", "lens");
  if (s.dim() != 3) refuse(n, s, at::kInt, "[n_seqs][n_kv_heads][keep]", "sel");
  const int64_t c = l.size(0), keep = s.size(2);
  return unlocked(n->select_pages, n->h, dense(n, a[1], n->dtype, {c, n->hq, n->d}, "q"), dense(n, a[2], n->dtype, {n->n_pages, n->hkv, 2, n->d}, "bounds"),
                         static_cast<const int32_t*>(dense(n, a[3], at::kInt, {c, n->width}, "table")), lengths(n, l, c, "lens"),
                         small(l.stride(0), "stride"), small(c, "n_seqs"), small(whole(a[5], "n_first"), "n_first"),
                         small(whole(a[6], "n_last"), "n_last"), small(keep, "keep"),
                         static_cast<int32_t*>(dense(n, a[7], at::kInt, {c, n->hkv, keep}, "sel")), stream_of(n, a[8]));
}

meda_status paged_attention(Args a) {          // q, k_pages, v_pages, table, lens, out, lse, sel, stream
  Native* n = native_of(a[0]);
  const at::Tensor& l = tensor(a[5], "lens");
  if (l.dim() != 1) refuse(n, l, at::kInt, "[n]", "lens");
  const int64_t c = l.size(0);
  const int32_t* sel = nullptr;
  int64_t keep = 0;
  if (a[8] != Py_None) {
    const at::Tensor& s = tensor(a[8], "sel");
    if (s.dim() != 3) refuse(n, s, at::kInt, "[n_seqs][n_kv_heads][keep]", "sel");
    keep = s.size(2);
    sel = static_cast<const int32_t*>(dense(n, a[8], at::kInt, {c, n->hkv, keep}, "sel"));
  }
  return unlocked(n->paged_attention, n->h, dense(n, a[1], n->dtype, {c, n->hq, n->d}, "q"),
                            dense(n, a[2], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "k_pages"),
                            dense(n, a[3], n->dtype, {n->n_pages, n->hkv, n->page, n->d}, "v_pages"),
                            static_cast<const int32_t*>(dense(n, a[4], at::kInt, {c, n->width}, "table")), lengths(n, l, c, "lens"),
                            small(l.stride(0), "stride"), small(c, "n_seqs"), sel, small(keep, "keep"),
                            dense(n, a[6], n->dtype, {c, n->hq, n->d}, "out"),
                            a[7] == Py_None ? nullptr : static_cast<float*>(dense(n, a[7], at::kFloat, {c, n->hq}, "lse")), stream_of(n, a[9]));
}

// Exceptions end here: a refusal is a ValueError, anything else a RuntimeError; a call's status is returned as a number.
template <meda_status (*F)(Args), Py_ssize_t COUNT>
PyObject* entry(PyObject*, Args a, Py_ssize_t n) {
  try {
    if (n != COUNT) throw Refused("wrong number of arguments");
    return PyLong_FromLong((long)F(a));
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

void drop(PyObject* o) { delete static_cast<Native*>(PyCapsule_GetPointer(o, kCapsule)); }

// bind(handle, device, is_f32, (n_pages, width, hq, hkv, page_size, head_dim), (six addresses)) -> capsule
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long h, f[6];
  int device, f32;
  long long g[6];
  if (!PyArg_ParseTuple(args, "Kip(LLLLLL)(KKKKKK)", &h, &device, &f32, g, g + 1, g + 2, g + 3, g + 4, g + 5, f, f + 1, f + 2, f + 3, f + 4, f + 5))
    return nullptr;
  auto* n = new (std::nothrow) Native();
  if (!n) return PyErr_NoMemory();
  n->h = reinterpret_cast<meda_pages*>(h);
  n->device = device;
  n->dtype = f32 ? at::kFloat : at::kBFloat16;
  n->n_pages = g[0];
  n->width = g[1];
  n->hq = g[2];
  n->hkv = g[3];
  n->page = g[4];
  n->d = g[5];
  n->page_tables = reinterpret_cast<decltype(n->page_tables)>(f[0]);
  n->page_store = reinterpret_cast<decltype(n->page_store)>(f[1]);
  n->page_bounds = reinterpret_cast<decltype(n->page_bounds)>(f[2]);
  n->rope_append = reinterpret_cast<decltype(n->rope_append)>(f[3]);
  n->select_pages = reinterpret_cast<decltype(n->select_pages)>(f[4]);
  n->paged_attention = reinterpret_cast<decltype(n->paged_attention)>(f[5]);
  return PyCapsule_New(n, kCapsule, drop);
}

// unbind(capsule): later calls with it are refused.
PyObject* unbind(PyObject*, PyObject* o) {
  auto* n = static_cast<Native*>(PyCapsule_GetPointer(o, kCapsule));
  if (!n) return nullptr;
  n->h = nullptr;
  Py_RETURN_NONE;
}

#define MEDA_ENTRY(name, count) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<name, count>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    MEDA_ENTRY(page_tables, 10), MEDA_ENTRY(page_store, 9), MEDA_ENTRY(page_bounds, 7), MEDA_ENTRY(rope_append, 10),
    MEDA_ENTRY(select_pages, 9), MEDA_ENTRY(paged_attention, 10),
    {"bind", bind, METH_VARARGS, nullptr}, {"unbind", unbind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pages", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// Read from the file by build.py before anything of it is loaded.
extern "C" __attribute__((visibility("default"), used)) const char meda_pages_built_for[] = MEDA_BUILT_FOR;

PyMODINIT_FUNC PyInit__pages() { return PyModule_Create(&module); }
