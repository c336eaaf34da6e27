// The calls of the Python binding.  ptr and stream: the device pointer of a tensor (with the check that it is a contiguous CUDA
// tensor) and the current stream.  bind: callables for entry points of libdet.so that convert their own arguments, tensors, numbers, a
// workspace and the current stream, call with the interpreter's lock released and raise on a status that is not DET_OK.  One call of 19
// arguments took some 7 us of the host through a Python expression per argument and ctypes, and those calls, not the GPU,
// are what a single small linear waits for.  Numbers that are no Python int or float go through ctypes as before.
#include <Python.h>
#include <dlfcn.h>

#include <cstring>
#include <memory>
#include <string>
#include <type_traits>
#include <utility>
#include <vector>

#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Exceptions.h>
#include <ATen/Context.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "../../include/det.h"

// address of a contiguous CUDA tensor; None is 0 and integers are taken as they are; false with an error set
static bool address_of(PyObject* t, unsigned long long& out) {
  if (THPVariable_Check(t)) {
    const at::Tensor& x = THPVariable_Unpack(t);
    if (!x.is_cuda() || !x.is_contiguous()) {
      PyErr_SetString(PyExc_AssertionError, "tensors must be contiguous CUDA tensors");
      return false;
    }
    out = reinterpret_cast<unsigned long long>(x.data_ptr());
    return true;
  }
  if (t == Py_None) { out = 0; return true; }
  if (PyLong_Check(t)) {
    out = PyLong_AsUnsignedLongLongMask(t);
    return !PyErr_Occurred();
  }
  PyErr_Format(PyExc_TypeError, "expected a CUDA tensor, an address or None, got %s", Py_TYPE(t)->tp_name);
  return false;
}
// the same for calls that refuse a tensor on another device than the current one, where the kernels run: 8-bit linears, AdamW with moments in 8 bits
static bool address_on(PyObject* t, unsigned long long& out, int device) {
  if (!address_of(t, out)) return false;
  if (THPVariable_Check(t) && THPVariable_Unpack(t).get_device() != device) {
    PyErr_SetString(PyExc_AssertionError, "tensors must be on the current CUDA device");
    return false;
  }
  return true;
}
// the current device, none where there is no GPU (a tensor on one is refused then as any is that is on the host)
static int current_device() {
  c10::DeviceIndex d = -1;
  return c10::cuda::GetDevice(&d) == cudaSuccess ? d : -1;
}
static unsigned long long current_stream() {
  at::globalContext().lazyInitDevice(c10::DeviceType::CUDA);
  return reinterpret_cast<unsigned long long>(c10::cuda::getCurrentCUDAStream().stream());
}

// None and integers pass through, a tensor becomes its address
static PyObject* ptr(PyObject*, PyObject* t) {
  HANDLE_TH_ERRORS
  if (t == Py_None || PyLong_Check(t)) {
    Py_INCREF(t);
    return t;
  }
  unsigned long long a;
  return address_of(t, a) ? PyLong_FromUnsignedLongLong(a) : nullptr;
  END_HANDLE_TH_ERRORS
}
static PyObject* stream(PyObject*, PyObject*) {
  HANDLE_TH_ERRORS
  return PyLong_FromUnsignedLongLong(current_stream());
  END_HANDLE_TH_ERRORS
}

// ---- entry points ---------------------------------------------------------------------------------------------------
union Slot {                                   // one C argument
  unsigned long long u;
  float f;
};
constexpr int MAX_ARGS = 24;
template <class A>
static A slot_as(const Slot& s) {
  if constexpr (std::is_pointer<A>::value) return reinterpret_cast<A>(s.u);
  else if constexpr (std::is_same<A, float>::value) return s.f;
  else return static_cast<A>(s.u);
}
template <class A>
static constexpr char kind_of() {              // the letters of a signature; v: void*, what a workspace and a stream are declared as
  return std::is_same<A, void*>::value ? 'v' : std::is_pointer<A>::value ? 'p' : std::is_same<A, float>::value ? 'f' : sizeof(A) == 8 ? 'z' : 'i';
}
// whether a pattern gives each C argument what its type takes: a stream and a workspace only where there is a void*
static bool fits(const char* pattern, const std::string& kinds) {
  size_t n = 0;
  for (const char* c = pattern; *c; ++c) {
    const char k = n < kinds.size() ? kinds[n++] : 0;
    if (*c == 'w' ? k != 'v' || kinds[n++] != 'z' : *c == 's' ? k != 'v' : *c == 'p' ? k != 'p' && k != 'v' : k != *c || k == 'v') return false;
  }
  return n == kinds.size();
}
template <class... A, size_t... I>
static int invoke(int (*fn)(A...), const Slot* s, std::index_sequence<I...>) { return fn(slot_as<A>(s[I])...); }
template <class F> struct Typed;
template <class... A>
struct Typed<int(A...)> {
  static_assert(sizeof...(A) <= MAX_ARGS, "more arguments than slots");
  static int call(void* fn, const Slot* s) { return invoke(reinterpret_cast<int (*)(A...)>(fn), s, std::index_sequence_for<A...>()); }
  static std::string kinds() { return std::string{kind_of<A>()...}; }
};

struct Entry {
  const char* name;
  int (*call)(void*, const Slot*);
  std::string (*kinds)();
  PyMethodDef def;
};
static PyObject* entry_call(PyObject* self, PyObject* const* args, Py_ssize_t nargs);
#define DET_ENTRY(f) \
  {#f, &Typed<decltype(f)>::call, &Typed<decltype(f)>::kinds, {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry_call)), METH_FASTCALL, nullptr}}
static Entry entries[] = {
    DET_ENTRY(det_sum), DET_ENTRY(det_sum_static), DET_ENTRY(det_scale_inplace), DET_ENTRY(det_lsq_weight_scale), DET_ENTRY(det_lsq_act_scale_init),
    DET_ENTRY(det_lsq_quantize_weight), DET_ENTRY(det_linear_fwd), DET_ENTRY(det_linear_fwd_q), DET_ENTRY(det_linear_bwd), DET_ENTRY(det_rmsnorm_fwd),
    DET_ENTRY(det_rmsnorm_fwd_q), DET_ENTRY(det_residual_rmsnorm_fwd), DET_ENTRY(det_headnorm_fwd), DET_ENTRY(det_headnorm_bwd), DET_ENTRY(det_rope),
    DET_ENTRY(det_rmsnorm_bwd), DET_ENTRY(det_rmsnorm_bwd_residual), DET_ENTRY(det_xent_fwd), DET_ENTRY(det_xent_bwd), DET_ENTRY(det_attn_fwd),
    DET_ENTRY(det_attn_fwd_q), DET_ENTRY(det_attn_fwd_int8pv), DET_ENTRY(det_attn_bwd), DET_ENTRY(det_attn_bwd_fixq), DET_ENTRY(det_swiglu_fwd),
    DET_ENTRY(det_swiglu_fwd_q), DET_ENTRY(det_swiglu_bwd), DET_ENTRY(det_residual_add), DET_ENTRY(det_embed_fwd), DET_ENTRY(det_embed_bwd),
    DET_ENTRY(det_lmhead_fwd), DET_ENTRY(det_lmhead_fwd_v2), DET_ENTRY(det_lmhead_bwd), DET_ENTRY(det_lmhead_bwd_v2), DET_ENTRY(det_attn_fwd_v2),
    DET_ENTRY(det_tensor_hash_async), DET_ENTRY(det_layernorm_fwd), DET_ENTRY(det_residual_layernorm_fwd), DET_ENTRY(det_layernorm_bwd),
    DET_ENTRY(det_layernorm_bwd_residual), DET_ENTRY(det_layernorm_bwd_act8), DET_ENTRY(det_act8_pack), DET_ENTRY(det_act8_unpack),
    DET_ENTRY(det_swiglu_fwd_act8), DET_ENTRY(det_swiglu_act8), DET_ENTRY(det_swiglu_bwd_act8), DET_ENTRY(det_linrec_fwd), DET_ENTRY(det_linrec_bwd),
    DET_ENTRY(det_tok8_quant), DET_ENTRY(det_tok8_transpose), DET_ENTRY(det_tok8_linear_fwd), DET_ENTRY(det_tok8_linear_fwd_q), DET_ENTRY(det_tok8_linear_bwd),
    DET_ENTRY(det_tok8_glu_fwd), DET_ENTRY(det_tok8_glu_fwd_q), DET_ENTRY(det_tok8_glu_bwd)};

// One callable that bind returns, owned by the capsule that is its self: nothing is shared between two results of bind.
struct Callable {
  const Entry* entry;
  void* fn;
  std::string pattern;                         // per Python argument: p i z f, or w a workspace (its address and size); s the current stream
  bool here = false;                           // tensors have to be on the current device
  PyObject* general = nullptr;                 // the entry point with its C types declared (ctypes)
  PyObject* raise_status = nullptr;            // raise_status(name, status)
  ~Callable() { Py_XDECREF(general); Py_XDECREF(raise_status); }
};
static void callable_free(PyObject* capsule) { delete static_cast<Callable*>(PyCapsule_GetPointer(capsule, nullptr)); }

// The call with arguments that are not plain Python numbers: addresses, sizes and the stream as they have been found, the numbers as
// they came, so that what is taken for a number, and the error for what is not, are those of the declared types.
static bool call_general(const Callable& e, const Slot* s, PyObject* const* args, int& rc) {
  PyObject* t = PyTuple_New((Py_ssize_t)e.entry->kinds().size());
  if (!t) return false;
  Py_ssize_t n = 0;
  for (const char c : e.pattern) {
    if (c != 's') ++args;
    for (int k = 0; k < (c == 'w' ? 2 : 1); ++k, ++n) {
      PyObject* x = c == 'i' || c == 'z' || c == 'f' ? Py_NewRef(args[-1]) : PyLong_FromUnsignedLongLong(s[n].u);
      if (!x) { Py_DECREF(t); return false; }
      PyTuple_SET_ITEM(t, n, x);
    }
  }
  PyObject* r = PyObject_CallObject(e.general, t);
  Py_DECREF(t);
  if (!r) return false;
  rc = (int)PyLong_AsLong(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}
static PyObject* entry_call(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  const Callable* e = static_cast<const Callable*>(PyCapsule_GetPointer(self, nullptr));
  if (!e) return nullptr;
  const char* name = e->entry->name;
  const int device = e->here ? current_device() : -1;
  const auto address = [&](PyObject* x, unsigned long long& out) { return e->here ? address_on(x, out, device) : address_of(x, out); };
  Slot s[MAX_ARGS];
  int n = 0, rc;
  Py_ssize_t a = 0;
  bool plain = true;                           // every number is a Python int or float
  for (const char c : e->pattern) {
    if (c == 's') { s[n++].u = current_stream(); continue; }
    if (a == nargs) { PyErr_Format(PyExc_TypeError, "%s: too few arguments", name); return nullptr; }
    PyObject* x = args[a++];
    switch (c) {
      case 'p':
        if (!address(x, s[n++].u)) return nullptr;
        break;
      case 'w':                                // the size comes from the tensor, so an address alone is no workspace
        if (!address(x, s[n].u)) return nullptr;
        if (x == Py_None) s[n + 1].u = 0;
        else if (THPVariable_Check(x)) s[n + 1].u = THPVariable_Unpack(x).nbytes();
        else { PyErr_Format(PyExc_AttributeError, "%s: a workspace is a tensor or None", name); return nullptr; }
        n += 2;
        break;
      case 'f':
        plain = plain && (PyFloat_Check(x) || PyLong_Check(x));
        if (plain) {
          const double d = PyFloat_AsDouble(x);
          s[n].f = static_cast<float>(d);
          if (d == -1.0 && PyErr_Occurred()) { PyErr_Clear(); plain = false; }   // an integer beyond the range
        }
        ++n;
        break;
      default:
        plain = plain && PyLong_Check(x);
        if (plain) s[n].u = PyLong_AsUnsignedLongLongMask(x);
        ++n;
    }
  }
  if (a != nargs) { PyErr_Format(PyExc_TypeError, "%s: too many arguments", name); return nullptr; }
  if (plain) {
    Py_BEGIN_ALLOW_THREADS
    rc = e->entry->call(e->fn, s);
    Py_END_ALLOW_THREADS
  } else if (!call_general(*e, s, args, rc)) {
    return nullptr;
  }
  if (rc != DET_OK) return PyObject_CallFunction(e->raise_status, "si", name, rc);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// ---- the calls with tables of tensors --------------------------------------------------------------------------------
// AdamW with moments in 8 bits takes eleven tables; through Python expressions and ctypes sixty tensors took the host 180 us, the GPU 16.
static int (*adamw8_batch_fn)(const det_adamw_desc*, const int*, const void* const*, float* const*, const void* const*, const void* const*, const float* const*,
                              void* const*, void* const*, void* const*, float* const*, const size_t*, int, const float*, void*);
static int (*adamw8_pack_fn)(const float* const*, const float* const*, int8_t* const*, uint8_t* const*, float* const*, const size_t*, int, void*);
static int (*adamw8_unpack_fn)(const int8_t* const*, const uint8_t* const*, const float* const*, float* const*, float* const*, const size_t*, int, void*);

struct Table {                                 // a list or tuple of tensors
  PyObject* seq = nullptr;
  std::vector<void*> p;
  std::vector<size_t> n;
  std::vector<int> width;                      // bytes of an element, 0 for None
  ~Table() { Py_XDECREF(seq); }
  bool take(PyObject* list, bool may_be_none, int device) {
    seq = PySequence_Fast(list, "a table is a list of tensors");
    if (!seq) return false;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(seq);
    p.resize(k); n.resize(k); width.resize(k);
    for (Py_ssize_t i = 0; i < k; ++i) {
      PyObject* t = PySequence_Fast_GET_ITEM(seq, i);
      unsigned long long a = 0;
      if (t == Py_None && may_be_none) { p[i] = nullptr; n[i] = 0; width[i] = 0; continue; }
      if (!THPVariable_Check(t)) { PyErr_SetString(PyExc_AssertionError, "a table holds tensors"); return false; }
      if (!address_on(t, a, device)) return false;
      const at::Tensor& x = THPVariable_Unpack(t);
      p[i] = reinterpret_cast<void*>(a);
      n[i] = (size_t)x.numel();
      width[i] = (int)x.element_size();
    }
    return true;
  }
  template <class T> T* as() { return static_cast<T*>(static_cast<void*>(p.data())); }
};
static size_t adamw8_scale_floats(size_t n) { return (n + 255) / 256 * 2; }

// adamw8_batch(descs, kinds, ps, gs, ms, vs, ss, coef, outs): outs is (ps, ms, vs, ss) or None
static PyObject* adamw8_batch(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  PyObject *descs, *kinds, *lists[5], *coef, *outs;
  if (!PyArg_ParseTuple(args, "OOOOOOOOO", &descs, &kinds, &lists[0], &lists[1], &lists[2], &lists[3], &lists[4], &coef, &outs)) return nullptr;
  const int device = current_device();
  Table in[5], out[4];
  const int of_out[4] = {0, 2, 3, 4};
  for (int i = 0; i < 5; ++i)
    if (!in[i].take(lists[i], i == 4, device)) return nullptr;
  if (outs != Py_None) {
    PyObject* four[4];
    if (!PyArg_ParseTuple(outs, "OOOO", &four[0], &four[1], &four[2], &four[3])) return nullptr;
    for (int i = 0; i < 4; ++i)
      if (!out[i].take(four[i], i == 3, device)) return nullptr;
  }
  Table* to[4];
  for (int i = 0; i < 4; ++i) to[i] = outs == Py_None ? &in[of_out[i]] : &out[i];
  Table hold;                                  // releases the sequences of the descriptors and kinds
  PyObject* ds = PySequence_Fast(descs, "descriptors are a list");
  hold.seq = ds;
  Table hold2;
  PyObject* ks = ds ? PySequence_Fast(kinds, "types are a list") : nullptr;
  hold2.seq = ks;
  if (!ks) return nullptr;
  const size_t k = in[0].p.size();
  bool fit = (size_t)PySequence_Fast_GET_SIZE(ds) == k && (size_t)PySequence_Fast_GET_SIZE(ks) == k;
  for (const Table& t : in) fit = fit && t.p.size() == k;
  for (const Table* t : to) fit = fit && t->p.size() == k;
  std::vector<det_adamw_desc> d(k);
  std::vector<int> kind(k);
  for (size_t i = 0; fit && i < k; ++i) {
    kind[i] = (int)PyLong_AsLong(PySequence_Fast_GET_ITEM(ks, i));
    if (PyErr_Occurred()) return nullptr;
    Py_buffer b;
    if (PyObject_GetBuffer(PySequence_Fast_GET_ITEM(ds, i), &b, PyBUF_SIMPLE) != 0) return nullptr;
    const bool whole = b.len == (Py_ssize_t)sizeof(det_adamw_desc);
    if (whole) d[i] = *static_cast<const det_adamw_desc*>(b.buf);
    PyBuffer_Release(&b);
    const size_t n = in[0].n[i], sc = adamw8_scale_floats(n);
    const bool eight = in[4].width[i] != 0;
    const int wp = kind[i] == DET_BF16 ? 2 : 4, wm = eight ? 1 : 4;
    fit = whole && in[0].width[i] == wp && in[1].n[i] == n && in[1].width[i] == 4;
    for (int t = 2; t < 4; ++t) fit = fit && in[t].n[i] == n && in[t].width[i] == wm;
    for (int t = 0; t < 3; ++t) fit = fit && to[t]->n[i] == n && to[t]->width[i] == (t ? wm : wp);
    fit = fit && (to[3]->width[i] != 0) == eight && (!eight || (in[4].n[i] == sc && in[4].width[i] == 4 && to[3]->n[i] == sc && to[3]->width[i] == 4));
  }
  if (!fit) {
    PyErr_SetString(PyExc_AssertionError, "one entry per tensor in every list; parameter, gradient and moments of a tensor have the same number of elements, "
                                          "two scales for every 256");
    return nullptr;
  }
  unsigned long long c = 0;
  if (!address_on(coef, c, device)) return nullptr;
  void* st = reinterpret_cast<void*>(current_stream());
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = adamw8_batch_fn(d.data(), kind.data(), in[0].as<const void*>(), in[1].as<float*>(), in[2].as<const void*>(), in[3].as<const void*>(),
                       in[4].as<const float*>(), to[0]->as<void*>(), to[1]->as<void*>(), to[2]->as<void*>(), to[3]->as<float*>(), in[0].n.data(), (int)k,
                       reinterpret_cast<const float*>(c), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}
// adamw8_numbers(pack, m8s, v8s, ss, ms, vs)
static PyObject* adamw8_numbers(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  int pack;
  PyObject* lists[5];
  if (!PyArg_ParseTuple(args, "pOOOOO", &pack, &lists[0], &lists[1], &lists[2], &lists[3], &lists[4])) return nullptr;
  const int device = current_device();
  Table t[5];
  for (int i = 0; i < 5; ++i)
    if (!t[i].take(lists[i], false, device)) return nullptr;
  const size_t k = t[0].p.size();
  bool fit = true;
  for (const Table& x : t) fit = fit && x.p.size() == k;
  for (size_t i = 0; fit && i < k; ++i)
    for (int x = 0; x < 5; ++x) fit = fit && t[x].n[i] == (x == 2 ? adamw8_scale_floats(t[0].n[i]) : t[0].n[i]) && t[x].width[i] == (x < 2 ? 1 : 4);
  if (!fit) {
    PyErr_SetString(PyExc_AssertionError, "one entry per tensor in every list; codes and moments of a tensor have the same number of elements, two scales for "
                                          "every 256");
    return nullptr;
  }
  void* st = reinterpret_cast<void*>(current_stream());
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = pack ? adamw8_pack_fn(t[3].as<const float*>(), t[4].as<const float*>(), t[0].as<int8_t*>(), t[1].as<uint8_t*>(),
                             t[2].as<float*>(), t[0].n.data(), (int)k, st)
            : adamw8_unpack_fn(t[0].as<const int8_t*>(), t[1].as<const uint8_t*>(), t[2].as<const float*>(), t[3].as<float*>(), t[4].as<float*>(),
                               t[0].n.data(), (int)k, st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// bind(path of libdet.so, {name: pattern}, raise_status, the library with its C types declared) -> {name: callable}
static PyObject* bind(PyObject*, PyObject* args) {
  HANDLE_TH_ERRORS
  const char* path;
  PyObject *patterns, *raise, *declared;
  if (!PyArg_ParseTuple(args, "sO!OO", &path, &PyDict_Type, &patterns, &raise, &declared)) return nullptr;
  void* lib = dlopen(path, RTLD_NOW);
  if (!lib) { PyErr_Format(PyExc_ImportError, "%s", dlerror()); return nullptr; }
  adamw8_batch_fn = reinterpret_cast<decltype(adamw8_batch_fn)>(dlsym(lib, "det_adamw8_batch"));
  adamw8_pack_fn = reinterpret_cast<decltype(adamw8_pack_fn)>(dlsym(lib, "det_adamw8_pack"));
  adamw8_unpack_fn = reinterpret_cast<decltype(adamw8_unpack_fn)>(dlsym(lib, "det_adamw8_unpack"));
  static_assert(std::is_same<decltype(adamw8_batch_fn), decltype(&det_adamw8_batch)>::value, "the declaration");
  static_assert(std::is_same<decltype(adamw8_pack_fn), decltype(&det_adamw8_pack)>::value, "the declaration");
  static_assert(std::is_same<decltype(adamw8_unpack_fn), decltype(&det_adamw8_unpack)>::value, "the declaration");
  if (!adamw8_batch_fn || !adamw8_pack_fn || !adamw8_unpack_fn) { PyErr_SetString(PyExc_ImportError, "det_adamw8_*: not in the library"); return nullptr; }
  PyObject* out = PyDict_New();
  if (!out) return nullptr;
  for (Entry& e : entries) {
    PyObject* pat = PyDict_GetItemString(patterns, e.name);
    const char* p = pat ? PyUnicode_AsUTF8(pat) : nullptr;
    std::unique_ptr<Callable> own(new Callable);
    own->entry = &e;
    own->fn = dlsym(lib, e.name);
    if (!own->fn || !p || !fits(p, e.kinds())) {
      PyErr_Format(PyExc_ImportError, "%s: %s", e.name, own->fn ? "the pattern does not fit the declaration" : "not in the library");
      Py_DECREF(out);
      return nullptr;
    }
    own->pattern = p;
    own->here = std::strncmp(e.name, "det_tok8_", 9) == 0;
    own->general = PyObject_GetAttrString(declared, e.name);
    own->raise_status = Py_NewRef(raise);
    PyObject* self = own->general ? PyCapsule_New(own.get(), nullptr, callable_free) : nullptr;
    if (self) own.release();
    PyObject* f = self ? PyCFunction_New(&e.def, self) : nullptr;
    Py_XDECREF(self);
    const int bad = f ? PyDict_SetItemString(out, e.name, f) : -1;
    Py_XDECREF(f);
    if (bad) { Py_DECREF(out); return nullptr; }
  }
  return out;
  END_HANDLE_TH_ERRORS
}
static PyMethodDef methods[] = {{"ptr", ptr, METH_O, "device address of a contiguous CUDA tensor; None and integers as they are"},
                                {"stream", stream, METH_NOARGS, "handle of the current CUDA stream"},
                                {"bind", bind, METH_VARARGS, "callables for the library's entry points"},
                                {"adamw8_batch", adamw8_batch, METH_VARARGS, "det_adamw8_batch with tables of tensors; returns its status"},
                                {"adamw8_numbers", adamw8_numbers, METH_VARARGS, "det_adamw8_pack or det_adamw8_unpack with tables of tensors"},
                                {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods};
PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
