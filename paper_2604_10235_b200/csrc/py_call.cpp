// Python extension `_cccall`: calls an entry point of libcodecomp with tensors as arguments.
//
// bind(name, address, spec) makes a callable of an entry point that takes only pointers and integers: it
// turns every argument into one machine word as the characters of spec say, converts the words to the
// parameter types that codecomp.h declares, calls the function with the GIL released and returns its status.
// A call marshalled argument by argument through ctypes costs about 8 us of host time, as much as a short
// prompt's kernels take; this costs 1.5 us.
//   i  an integer                         t  a CUDA tensor, or None for NULL
//   p  a CUDA or page-locked host tensor, or None
//   w  a CUDA tensor as two words: address, number of elements
//   L  a sequence of tensors as a host array of addresses, or None
//   d  a device number (no word): the tensors of the kinds below are on that device
//   n  a contiguous CUDA tensor of int32, or None
//   W  a contiguous CUDA tensor as two words: address, number of elements; None: two zeros
//   h  a contiguous host array (numpy) of 32-bit integers
// and, where the second argument is a cc_cache_desc, tensors that hold what it describes, or None:
//   A  q_new      B  k_new, v_new      C  q      K  k, v      O  out         bfloat16
//   P  positions (int32), S  lse (float32)                                   contiguous
//   M  a sequence of k or v (none of them None) as a host array of addresses
// A tensor for which the descriptor gives no strides has to be contiguous; the memory from a tensor's first element to
// its last one has to hold all rows and heads at the descriptor's strides, whatever the shape in which it comes.
//
// What a torch.Tensor is and where it lies comes from torch's DLPack table in one call, where this torch has one: the eight tensors of a
// rotation take 0.8 us with all checks; by their methods, and without the checks of sizes and strides, they took 2.9.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "codecomp.h"

namespace {

constexpr int kMaxWords = 20;

PyObject *s_data_ptr, *s_is_cuda, *s_is_pinned, *s_numel, *s_dtype, *s_get_device, *s_shape, *s_stride;
PyObject *t_bf16, *t_i32, *t_f32;      // torch's types, looked up with the first spec that names one
const char kTyped[] = "nABCKOPSM";     // kinds whose type and device are checked
const char kLaidOut[] = "ABCKOPSM";    // of them those that the descriptor lays out

bool word_of(PyObject* o, uint64_t* out) {
  *out = PyLong_AsUnsignedLongLongMask(o);
  return !(*out == (uint64_t)-1 && PyErr_Occurred());
}

// result of a method without arguments as a word
bool word_from(PyObject* o, PyObject* method, uint64_t* out) {
  PyObject* r = PyObject_CallMethodNoArgs(o, method);
  if (!r) return false;
  const bool ok = word_of(r, out);
  Py_DECREF(r);
  return ok;
}

bool is_true(PyObject* r) {
  const bool yes = r == Py_True;
  Py_XDECREF(r);
  return yes;
}

bool tensor_word(PyObject* o, bool pinned_ok, uint64_t* out) {
  if (o == Py_None) {
    *out = 0;
    return true;
  }
  if (!is_true(PyObject_GetAttr(o, s_is_cuda))) {
    if (PyErr_Occurred()) return false;
    if (!pinned_ok || !is_true(PyObject_CallMethodNoArgs(o, s_is_pinned))) {
      if (!PyErr_Occurred())
        PyErr_SetString(PyExc_ValueError, pinned_ok ? "libcodecomp takes CUDA tensors only (or page-locked host memory here)"
                                                    : "libcodecomp takes CUDA tensors only");
      return false;
    }
  }
  return word_from(o, s_data_ptr, out);
}

// What the checks need of a tensor.
struct Tensor {
  PyObject* dtype;             // borrowed
  long device;                 // -1: the host
  uint64_t address;
  bool contiguous;
  int64_t reach;               // elements from the first one to the last one
};

// From the sizes and strides, innermost last.
template <class Dim>
void lay_out(Py_ssize_t dims, const Dim& dim, Tensor* t) {
  int64_t dense = 1, last = 0;
  bool none = false;
  t->contiguous = true;
  for (Py_ssize_t i = dims - 1; i >= 0; --i) {
    const std::pair<int64_t, int64_t> d = dim(i);          // size, stride
    none |= d.first == 0;
    if (d.first == 1) continue;
    t->contiguous &= d.second == dense;
    dense *= d.first;
    last += (d.first - 1) * d.second;
  }
  t->contiguous |= none;
  t->reach = none ? 0 : last + 1;
}

// By the object's own methods (a subclass of torch.Tensor, or whatever else behaves like one).
bool describe_by_methods(PyObject* o, Tensor* t) {
  uint64_t at = 0;
  t->dtype = PyObject_GetAttr(o, s_dtype);
  if (!t->dtype) return false;
  Py_DECREF(t->dtype);                                     // (torch keeps its types)
  if (!word_from(o, s_get_device, &at) || !word_from(o, s_data_ptr, &t->address)) return false;
  t->device = (long)at;
  PyObject* shape = PyObject_GetAttr(o, s_shape);
  PyObject* stride = shape ? PyObject_CallMethodNoArgs(o, s_stride) : nullptr;
  bool ok = stride && PyTuple_Check(shape) && PyTuple_Check(stride) && PyTuple_GET_SIZE(shape) == PyTuple_GET_SIZE(stride);
  if (ok)
    lay_out(PyTuple_GET_SIZE(shape), [&](Py_ssize_t i) {
      return std::make_pair((int64_t)PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)), (int64_t)PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i)));
    }, t);
  Py_XDECREF(shape);
  Py_XDECREF(stride);
  if (!ok && !PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "a tensor is needed");
  return ok && !PyErr_Occurred();
}

// The C interface of DLPack 1.3 and later 1.x, as far as it is used: what a tensor is, without a reference to it.
struct DlTensor {
  void* data;
  struct { int32_t type, id; } device;                     // type 2: CUDA
  int32_t dims;
  struct { uint8_t code, bits; uint16_t lanes; } dtype;    // code 0: integers, 2: floats, 4: bfloat
  int64_t *shape, *strides;
  uint64_t byte_offset;
};
struct DlTable {
  uint32_t major, minor;
  void *older, *allocate, *to_managed, *from_managed;
  int (*describe)(void* object, DlTensor* out);
};
const DlTable* g_table;        // of torch.Tensor, or null: a torch without one
PyTypeObject* g_tensor;

void find_table(PyObject* torch) {
  PyObject* type = PyObject_GetAttrString(torch, "Tensor");
  PyObject* capsule = type ? PyObject_GetAttrString(type, "__dlpack_c_exchange_api__") : nullptr;
  const DlTable* table = capsule ? static_cast<const DlTable*>(PyCapsule_GetPointer(capsule, "dlpack_exchange_api")) : nullptr;
  if (table && table->major == 1 && table->minor >= 3 && table->describe) {
    g_table = table;                   // (alive as long as the process)
    g_tensor = reinterpret_cast<PyTypeObject*>(type);
    Py_INCREF(type);
  }
  Py_XDECREF(capsule);
  Py_XDECREF(type);
  PyErr_Clear();
}

bool describe_by_table(PyObject* o, Tensor* t) {
  DlTensor d;
  if (g_table->describe(o, &d) != 0) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a tensor that DLPack cannot describe");
    return false;
  }
  const auto is = [&](int code, int bits) { return d.dtype.code == code && d.dtype.bits == bits && d.dtype.lanes == 1; };
  t->dtype = is(4, 16) ? t_bf16 : is(2, 32) ? t_f32 : is(0, 32) ? t_i32 : nullptr;
  t->device = d.device.type == 2 ? d.device.id : -1;
  t->address = (uint64_t)(uintptr_t)d.data + d.byte_offset;
  lay_out(d.dims, [&](Py_ssize_t i) { return std::make_pair(d.shape[i], d.strides[i]); }, t);
  return true;
}

bool describe(PyObject* o, Tensor* t) {
  return g_table && Py_TYPE(o) == g_tensor ? describe_by_table(o, t) : describe_by_methods(o, t);
}

// A tensor of the given type on the given device.
bool typed(PyObject* o, PyObject* dtype, long device, bool contiguous, Tensor* t) {
  if (!describe(o, t)) return false;
  if (t->dtype != dtype || t->device != device) {
    PyErr_Format(PyExc_ValueError, "libcodecomp takes a tensor of %S on cuda:%ld here", dtype, device);
    return false;
  }
  if (contiguous && !t->contiguous) {
    PyErr_SetString(PyExc_ValueError, "libcodecomp takes a contiguous tensor here");
    return false;
  }
  return true;
}

bool workspace_words(PyObject* o, long device, uint64_t* out) {
  Tensor t = {};
  if (o != Py_None) {
    if (!describe(o, &t)) return false;
    if (t.device != device || !t.contiguous) {
      PyErr_Format(PyExc_ValueError, "libcodecomp takes a contiguous workspace on cuda:%ld here", device);
      return false;
    }
  }
  out[0] = t.address;
  out[1] = (uint64_t)t.reach;
  return true;
}

PyObject* dtype_of(char kind) { return kind == 'n' || kind == 'P' ? t_i32 : kind == 'S' ? t_f32 : t_bf16; }

// New tokens of all sequences; -1: a descriptor that the call refuses.
int64_t new_tokens(const cc_cache_desc* d) {
  if (!d || d->num_seqs < 1 || d->num_seqs > CC_MAX_SEQS) return -1;
  if (!d->new_lens) return d->num_seqs;
  int64_t tokens = 0;
  for (int s = 0; s < d->num_seqs; ++s) {
    if (d->new_lens[s] < 0) return -1;
    tokens += d->new_lens[s];
  }
  return tokens;
}
// Elements that a tensor of the kind reaches over, by the descriptor; whether it has to be contiguous.  False: nothing to check (no work, or
// a descriptor that the call refuses).
struct Wanted {
  __int128 reach;
  bool dense;
};
bool wanted(const cc_cache_desc* d, int64_t tokens, char kind, Wanted* w) {
  if (tokens < 0 || d->n_heads_q < 1 || d->n_heads_kv < 1 || (tokens == 0 && kind != 'M')) return false;
  const bool pool = kind == 'K' || kind == 'M';
  if (pool && (d->pool_pages < 1 || d->page_size < 1)) return false;
  const __int128 rows = pool ? (__int128)d->pool_pages * d->page_size : tokens;
  if (kind == 'P' || kind == 'S') {
    *w = {rows * (kind == 'S' ? d->n_heads_q : 1), true};
    return true;
  }
  const int64_t heads = kind == 'B' || pool ? d->n_heads_kv : d->n_heads_q;
  int64_t tok = pool ? d->kv_stride_tok : kind == 'A' ? d->q_new_stride_tok : kind == 'B' ? d->kv_new_stride_tok
                : kind == 'C' ? d->q_stride_tok : d->out_stride_tok;
  int64_t head = pool ? d->kv_stride_head : kind == 'A' ? d->q_new_stride_head : kind == 'B' ? d->kv_new_stride_head
                 : kind == 'C' ? d->q_stride_head : d->out_stride_head;
  if (tok < 0 || head < 0) return false;
  w->dense = tok == 0 && head == 0;
  if (tok == 0) tok = heads * d->head_dim;
  if (head == 0) head = d->head_dim;
  w->reach = (rows - 1) * tok + (__int128)(heads - 1) * head + d->head_dim;
  return true;
}

bool holds(const Tensor& t, const cc_cache_desc* d, int64_t tokens, char kind, const char* name) {
  Wanted w;
  if (!wanted(d, tokens, kind, &w)) return true;
  const char* what = kind == 'A' ? "q_new" : kind == 'B' ? "k_new or v_new" : kind == 'C' ? "q" : kind == 'O' ? "out"
                     : kind == 'P' ? "positions" : kind == 'S' ? "lse" : "k or v";
  if (w.dense && !t.contiguous) {
    PyErr_Format(PyExc_ValueError, "%s: the descriptor gives no strides for %s, which is not contiguous", name, what);
    return false;
  }
  if (w.reach > t.reach) {
    PyErr_Format(PyExc_ValueError, "%s: %s reaches over %lld elements, fewer than the descriptor describes", name, what, (long long)t.reach);
    return false;
  }
  return true;
}

bool host_word(PyObject* o, uint64_t* out) {
  Py_buffer view;
  if (PyObject_GetBuffer(o, &view, PyBUF_C_CONTIGUOUS) != 0) return false;
  const bool ok = view.itemsize == 4;
  *out = (uint64_t)(uintptr_t)view.buf;            // (the caller's array outlives the call)
  PyBuffer_Release(&view);
  if (!ok) PyErr_SetString(PyExc_ValueError, "an array of 32-bit integers is needed");
  return ok;
}

template <class T>
T from_word(uint64_t w) {
  if constexpr (std::is_pointer_v<T>) return reinterpret_cast<T>((uintptr_t)w);
  else return static_cast<T>(w);
}

template <class F> struct Caller;
template <class... A>
struct Caller<int (*)(A...)> {
  static constexpr int words = sizeof...(A);
  static_assert(words <= kMaxWords, "words of a call");
  static int call(void* fn, const uint64_t* a) { return spread(fn, a, std::index_sequence_for<A...>()); }
  template <size_t... I>
  static int spread(void* fn, const uint64_t* a, std::index_sequence<I...>) {
    return reinterpret_cast<int (*)(A...)>(fn)(from_word<A>(a[I])...);
  }
};

struct Entry {
  const char* name;
  int words;
  int (*call)(void* fn, const uint64_t* a);
};
#define ENTRY(f) {#f, Caller<decltype(&f)>::words, Caller<decltype(&f)>::call}
const Entry kEntries[] = {ENTRY(cc_score_window), ENTRY(cc_fuse_prior_pool), ENTRY(cc_topk_select),
                          ENTRY(cc_topk_select_static), ENTRY(cc_compact_kv), ENTRY(cc_compress_layer),
                          ENTRY(cc_compress_layers), ENTRY(cc_ppl_chunk_scores), ENTRY(cc_select_chunks),
                          ENTRY(cc_rope_append), ENTRY(cc_paged_attention), ENTRY(cc_fork_pages)};
#undef ENTRY

struct Bound {                // what a callable holds: an entry point of a loaded library and the spec of its arguments
  const Entry* entry;
  void* fn;
  int n_args;
  char spec[kMaxWords];
};
const char* const kBound = "_cccall.Bound";

PyObject* call_bound(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  const Bound* f = static_cast<const Bound*>(PyCapsule_GetPointer(self, kBound));
  if (!f) return nullptr;
  if (n_args != f->n_args) {
    PyErr_Format(PyExc_TypeError, "%s takes %d arguments, %zd were given", f->entry->name, f->n_args, n_args);
    return nullptr;
  }
  uint64_t a[kMaxWords];
  std::vector<std::vector<uint64_t>> lists;      // host arrays of the call (moving the outer one keeps their storage)
  struct Laid { char kind; Tensor t; };
  std::vector<Laid> laid;                        // checked when the type of every argument is
  int n = 0;
  long device = -1;
  for (Py_ssize_t i = 0; i < n_args; ++i) {
    PyObject* o = args[i];
    bool ok = true;
    switch (f->spec[i]) {
      case 'i': ok = word_of(o, &a[n++]); break;
      case 't': ok = tensor_word(o, false, &a[n++]); break;
      case 'p': ok = tensor_word(o, true, &a[n++]); break;
      case 'w': ok = tensor_word(o, false, &a[n]) && word_from(o, s_numel, &a[n + 1]); n += 2; break;
      case 'W': ok = workspace_words(o, device, &a[n]); n += 2; break;
      case 'd':
        device = PyLong_AsLong(o);
        ok = !(device == -1 && PyErr_Occurred());
        break;
      case 'h': ok = host_word(o, &a[n++]); break;
      case 'n':
      case 'A': case 'B': case 'C': case 'K': case 'O': case 'P': case 'S': {
        const char kind = f->spec[i];
        Tensor t = {};
        if (o != Py_None) ok = typed(o, dtype_of(kind), device, strchr("nPS", kind), &t);
        a[n++] = t.address;
        if (ok && o != Py_None && kind != 'n') {
          if (laid.empty()) laid.reserve(8);
          laid.push_back({kind, t});
        }
        break;
      }
      case 'M':
      case 'L': {
        if (o == Py_None && f->spec[i] == 'L') { a[n++] = 0; break; }
        PyObject* seq = PySequence_Fast(o, "a sequence of tensors");
        if (!seq) return nullptr;
        const Py_ssize_t m = PySequence_Fast_GET_SIZE(seq);
        lists.emplace_back((size_t)m + 1);
        for (Py_ssize_t j = 0; j < m && ok; ++j) {
          PyObject* item = PySequence_Fast_GET_ITEM(seq, j);
          if (f->spec[i] == 'L') {
            ok = word_from(item, s_data_ptr, &lists.back()[j]);
            continue;
          }
          Tensor t = {};
          ok = typed(item, t_bf16, device, false, &t);
          lists.back()[j] = t.address;
          if (ok) laid.push_back({'M', t});
        }
        Py_DECREF(seq);
        a[n++] = (uint64_t)(uintptr_t)lists.back().data();
        break;
      }
    }
    if (!ok) return nullptr;
  }
  if (!laid.empty()) {
    const cc_cache_desc* desc = reinterpret_cast<const cc_cache_desc*>((uintptr_t)a[1]);
    const int64_t tokens = new_tokens(desc);
    for (const Laid& x : laid)
      if (!holds(x.t, desc, tokens, x.kind, f->entry->name)) return nullptr;
  }
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f->entry->call(f->fn, a);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  try {
    return call_bound(self, args, n_args);
  } catch (const std::bad_alloc&) {            // of a host array of addresses
    return PyErr_NoMemory();
  }
}

PyMethodDef bound_call = {"bound", (PyCFunction)(void (*)(void))call, METH_FASTCALL, "an entry point: (*args) -> status"};

PyObject* bind(PyObject*, PyObject* args) {
  const char *name, *spec;
  Py_ssize_t len;
  PyObject* address;
  uint64_t fn;
  if (!PyArg_ParseTuple(args, "sOy#", &name, &address, &spec, &len) || !word_of(address, &fn)) return nullptr;
  const Entry* entry = nullptr;
  for (const Entry& e : kEntries)
    if (strcmp(e.name, name) == 0) entry = &e;
  if (!entry) return PyErr_Format(PyExc_ValueError, "%s cannot be bound", name);
  if (len > kMaxWords) return PyErr_Format(PyExc_ValueError, "the spec of %s is too long", name);
  int words = 0;
  for (Py_ssize_t i = 0; i < len; ++i) {
    if (!spec[i] || !strchr("itpwWLdnhABCKOPSM", spec[i])) return PyErr_Format(PyExc_ValueError, "unknown kind of argument in the spec of %s", name);
    words += spec[i] == 'w' || spec[i] == 'W' ? 2 : spec[i] == 'd' ? 0 : 1;
    if (strchr(kTyped, spec[i]) && !t_f32) {
      PyObject* torch = PyImport_ImportModule("torch");
      if (!torch) return nullptr;
      t_bf16 = PyObject_GetAttrString(torch, "bfloat16");
      t_i32 = PyObject_GetAttrString(torch, "int32");
      t_f32 = PyObject_GetAttrString(torch, "float32");
      find_table(torch);
      Py_DECREF(torch);
      if (!t_bf16 || !t_i32 || !t_f32) return nullptr;
    }
  }
  if (strpbrk(spec, kLaidOut) && strncmp(spec, "iid", 3) != 0)
    return PyErr_Format(PyExc_ValueError, "the spec of %s has no descriptor", name);
  if (words != entry->words) return PyErr_Format(PyExc_ValueError, "%s takes %d words, its spec gives %d", name, entry->words, words);
  Bound* f = new (std::nothrow) Bound{entry, reinterpret_cast<void*>((uintptr_t)fn), (int)len, {}};
  if (!f) return PyErr_NoMemory();
  memcpy(f->spec, spec, (size_t)len);
  PyObject* capsule = PyCapsule_New(f, kBound, [](PyObject* c) { delete static_cast<Bound*>(PyCapsule_GetPointer(c, kBound)); });
  if (!capsule) {
    delete f;
    return nullptr;
  }
  PyObject* callable = PyCFunction_New(&bound_call, capsule);
  Py_DECREF(capsule);
  return callable;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "bind(name, address, spec) -> callable"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cccall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cccall(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_is_cuda = PyUnicode_InternFromString("is_cuda");
  s_is_pinned = PyUnicode_InternFromString("is_pinned");
  s_numel = PyUnicode_InternFromString("numel");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  return PyModule_Create(&module);
}
