// Marshalling of the library's calls from Python in native code: binding.py's functions, argument by argument, without ctypes.
//
// A decode step is one launch of 8 us and its caller's program is a loop of such calls, so the time that a call takes the host
// is a large part of it: through ctypes it took 6.2 us (14 tensor addresses, 26 conversions, a structure reference, the current
// stream), here 4.4, of which about 3 are the launch; a call that launches nothing 1.31 and 0.34.  16 steps of one 7B sequence, both
// forms timed in turn, 230..238 -> 190..201 us (1.15..1.19), the float32 path 153 -> 115..124 (1.22..1.26).
//
// Each entry point is a callable that holds the Python function of the same name.  What it does not convert itself -- a number, a
// torch.Tensor or Parameter, the binding's own descriptors, None -- or an argument that is missing, it leaves to that function,
// called with the very same arguments: what is accepted, refused and raised is decided there.  The C functions are those of the
// library that the Python function calls, by their addresses in it; when that function has been given another library
// (binding._lib), the call is left to it, and another binding._stream is asked for the stream.
#include <Python.h>
#include <pthread.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <tuple>
#include <type_traits>
#include <utility>

#include "dllava.h"
#include "dllava_mx.h"

namespace {

constexpr size_t kMaxArgs = 32;

// Set once by binding.py (init): its classes, its error check, and where torch keeps the current stream.
PyObject *g_cache_type, *g_predictor_type, *g_check, *g_current_device, *g_get_device, *g_raw_stream;
PyObject *g_c, *g_lib_name, *g_stream_name, *g_check_name;  // "c", "_lib", "_stream", "_check"
bool g_device_ready = false;  // torch has initialised the device in this process

// The C structure behind a descriptor object (its ctypes field c), held for the length of a call.
struct Held {
  Py_buffer view{};
  ~Held() {
    if (view.obj) PyBuffer_Release(&view);
  }
  bool take(PyObject* owner) {
    PyObject* c = PyObject_GetAttr(owner, g_c);
    if (!c) return false;
    const bool ok = PyObject_GetBuffer(c, &view, PyBUF_SIMPLE) == 0;
    Py_DECREF(c);
    return ok;
  }
};

template <typename T>
struct Slot {  // one C argument
  static_assert(std::is_pointer_v<T> || std::is_arithmetic_v<T>, "argument type");
  T value{};
  bool take(PyObject* o) {
    if constexpr (std::is_pointer_v<T>) {
      if (o == Py_None) return true;
      if (!THPVariable_CheckExact(o)) return false;
      value = static_cast<T>(THPVariable_Unpack(o).data_ptr());
      return true;
    } else if constexpr (std::is_integral_v<T>) {
      if (!PyLong_Check(o)) return false;
      value = static_cast<T>(PyLong_AsUnsignedLongLongMask(o));
      return true;
    } else {
      if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
      value = static_cast<T>(PyFloat_AsDouble(o));
      return !PyErr_Occurred();
    }
  }
};
template <typename T, PyObject** TYPE>
struct DescriptorSlot {
  const T* value = nullptr;
  Held held;
  bool take(PyObject* o) {
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != *TYPE || !held.take(o) || held.view.len < static_cast<Py_ssize_t>(sizeof(T))) return false;
    value = static_cast<const T*>(held.view.buf);
    return true;
  }
};
template <>
struct Slot<const dllava_kv_cache*> : DescriptorSlot<dllava_kv_cache, &g_cache_type> {};
template <>
struct Slot<const dllava_predictor*> : DescriptorSlot<dllava_predictor, &g_predictor_type> {};

// The callable, and what of the binding its C function was found by.
struct Kind;
struct Call {
  PyObject_HEAD
  vectorcallfunc vectorcall;
  const Kind* kind;
  PyObject* python;      // the function of the same name
  PyObject* names;       // its parameters, in order; the last one is the stream and defaults to None
  PyObject* name;
  PyObject* globals;     // the binding
  PyObject* c_function;  // _lib.<name>
  void (*address)();     // where it points
  PyObject* stream;      // the binding's _stream
  PyObject *dict, *weak_references;
};

// torch's current stream of the current device, as binding._stream finds it
bool current_stream(const Call& c, void*& stream) {
  PyObject* const f = PyDict_GetItemWithError(c.globals, g_stream_name);
  if (f != c.stream) {  // replaced
    PyObject* r = f ? PyObject_CallOneArg(f, Py_None) : nullptr;
    const bool ok = r && (r == Py_None || PyLong_Check(r));
    if (ok) stream = r == Py_None ? nullptr : PyLong_AsVoidPtr(r);
    Py_XDECREF(r);
    return ok && !PyErr_Occurred();
  }
  PyObject* dev = g_device_ready ? PyObject_CallNoArgs(g_get_device) : PyObject_CallNoArgs(g_current_device);
  if (!dev) return false;
  g_device_ready = true;
  PyObject* s = PyObject_CallOneArg(g_raw_stream, dev);
  Py_DECREF(dev);
  if (!s) return false;
  stream = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

enum class Outcome { kDone, kFallback };

// A C function of type int(A...): its last argument is the stream; a size_t is the size of the buffer before it.
template <typename F>
struct Entry;
template <typename... A>
struct Entry<int (*)(A...)> {
  static constexpr size_t N = sizeof...(A);
  using Slots = std::tuple<Slot<std::remove_cv_t<A>>...>;

  template <size_t I>
  static bool take(Slots& s, PyObject* const* args, size_t& at, bool no_cache) {
    using T = std::tuple_element_t<I, std::tuple<A...>>;
    if constexpr (std::is_same_v<T, size_t>) {
      PyObject* o = args[at - 1];  // the workspace
      if (o != Py_None) std::get<I>(s).value = THPVariable_Unpack(o).numel() * THPVariable_Unpack(o).element_size();
      return true;
    } else {
      PyObject* o = args[at++];
      if constexpr (std::is_same_v<T, const dllava_kv_cache*>)
        if (o == Py_None) return no_cache;
      if constexpr (std::is_same_v<T, const dllava_predictor*>)
        if (o == Py_None) return false;
      return std::get<I>(s).take(o);
    }
  }
  // no_cache: the function may be called without a cache
  static Outcome call(const Call& c, PyObject* const* args, bool no_cache, int& rc) {
    Slots s;
    return all(c, s, args, no_cache, rc, std::make_index_sequence<N - 1>{}, std::make_index_sequence<N>{});
  }
  template <size_t... I, size_t... J>
  static Outcome all(const Call& c, Slots& s, PyObject* const* args, bool no_cache, int& rc, std::index_sequence<I...>, std::index_sequence<J...>) {
    size_t at = 0;
    if (!(take<I>(s, args, at, no_cache) && ...)) return Outcome::kFallback;
    if (args[at] != Py_None || !current_stream(c, std::get<N - 1>(s).value)) return Outcome::kFallback;
    const auto f = reinterpret_cast<int (*)(A...)>(c.address);
    Py_BEGIN_ALLOW_THREADS
    [&]() noexcept { rc = f(std::get<J>(s).value...); }();
    Py_END_ALLOW_THREADS
    return Outcome::kDone;
  }
  static constexpr size_t python_args() { return N - (0 + ... + (std::is_same_v<A, size_t> ? 1 : 0)); }
};

struct Kind {
  const char* name;
  size_t n_args;
  bool no_cache;
  Outcome (*call)(const Call&, PyObject* const*, bool, int&);
};
template <typename F>
constexpr Kind kind(const char* name, bool no_cache = false) {
  static_assert(Entry<F>::python_args() <= kMaxArgs);
  return {name, Entry<F>::python_args(), no_cache, Entry<F>::call};
}
const Kind kKinds[] = {
    kind<decltype(&dllava_score)>("dllava_score"),
    kind<decltype(&dllava_select_compact)>("dllava_select_compact", true),
    kind<decltype(&dllava_compact)>("dllava_compact", true),
    kind<decltype(&dllava_prefill_attn)>("dllava_prefill_attn", true),
    kind<decltype(&dllava_decode_attn_append)>("dllava_decode_attn_append"),
    kind<decltype(&dllava_decode_attn_append_static)>("dllava_decode_attn_append_static"),
    kind<decltype(&dllava_decode_step)>("dllava_decode_step"),
    kind<decltype(&dllava_decode_commit)>("dllava_decode_commit"),
    kind<decltype(&dllava_qkv_project)>("dllava_qkv_project"),
    kind<decltype(&dllava_predict)>("dllava_predict"),
    kind<decltype(&dllava_linear)>("dllava_linear"),
    kind<decltype(&dllava_layer_norm)>("dllava_layer_norm"),
    kind<decltype(&dllava_rms_norm)>("dllava_rms_norm"),
    kind<decltype(&dllava_span_attn)>("dllava_span_attn"),
    kind<decltype(&dllava_masked_attn)>("dllava_masked_attn"),
    kind<decltype(&dllava_linear_few)>("dllava_linear_few"),
    kind<decltype(&dllava_rope)>("dllava_rope"),
    kind<decltype(&dllava_qkv_few)>("dllava_qkv_few"),
    kind<decltype(&dllava_gated_few)>("dllava_gated_few"),
    kind<decltype(&dllava_mx_quantize)>("dllava_mx_quantize"),
    kind<decltype(&dllava_mx_dequantize)>("dllava_mx_dequantize"),
    kind<decltype(&dllava_mx_linear)>("dllava_mx_linear"),
    kind<decltype(&dllava_mx_linear_few)>("dllava_mx_linear_few"),
    kind<decltype(&dllava_mx_cache_store)>("dllava_mx_cache_store"),
    kind<decltype(&dllava_mx_cache_load)>("dllava_mx_cache_load"),
    kind<decltype(&dllava_mx_decode_attn_append)>("dllava_mx_decode_attn_append"),
    kind<decltype(&dllava_group_prefill_attn)>("dllava_group_prefill_attn"),
};

// ---- the callable -----------------------------------------------------------------------------------------------------------
// the Python function would call the C function of this callable
bool same_library(const Call& c) {
  PyObject* const lib = PyDict_GetItemWithError(c.globals, g_lib_name);
  PyObject* const f = lib ? PyObject_GetAttr(lib, c.name) : nullptr;
  Py_XDECREF(f);  // compared only
  if (!f) PyErr_Clear();
  return f == c.c_function;
}

PyObject* call_vector(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* kwnames) {
  Call* c = reinterpret_cast<Call*>(self);
  const size_t n = PyVectorcall_NARGS(nargsf), want = c->kind->n_args, nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
  PyObject* all[kMaxArgs];
  bool ok = n <= want && !at::impl::PythonTorchFunctionTLS::stack_len() && same_library(*c);
  if (ok) {
    memcpy(all, args, n * sizeof(PyObject*));
    for (size_t i = n; i < want; ++i) all[i] = nullptr;
    for (size_t k = 0; ok && k < nkw; ++k) {
      PyObject* name = PyTuple_GET_ITEM(kwnames, k);
      size_t i = n;
      while (i < want && PyTuple_GET_ITEM(c->names, i) != name && PyUnicode_Compare(PyTuple_GET_ITEM(c->names, i), name) != 0) ++i;
      ok = i < want && !all[i];
      if (ok) all[i] = args[n + k];
    }
    if (!all[want - 1]) all[want - 1] = Py_None;
    for (size_t i = n; ok && i < want; ++i) ok = all[i] != nullptr;
  }
  if (ok) {
    int rc = 0;
    Outcome o = Outcome::kFallback;
    try {
      o = c->kind->call(*c, all, c->kind->no_cache, rc);
    } catch (const std::exception&) {  // a tensor without memory of its own: torch's own message comes from the Python function
    }
    if (o == Outcome::kDone) {
      if (__builtin_expect(rc != 0, 0)) {
        PyObject* code = PyLong_FromLong(rc);
        if (!code) return nullptr;
        PyObject* const check = PyDict_GetItemWithError(c->globals, g_check_name);
        PyObject* r = PyObject_CallOneArg(check ? check : g_check, code);  // raises
        Py_DECREF(code);
        return r;
      }
      Py_RETURN_NONE;
    }
    PyErr_Clear();
  }
  return PyObject_Vectorcall(c->python, args, nargsf, kwnames);
}

int call_traverse(PyObject* self, visitproc visit, void* arg) {
  Call* c = reinterpret_cast<Call*>(self);
  for (PyObject* o : {c->python, c->names, c->name, c->globals, c->c_function, c->stream, c->dict}) Py_VISIT(o);
  return 0;
}
int call_clear(PyObject* self) {
  Call* c = reinterpret_cast<Call*>(self);
  for (PyObject** o : {&c->python, &c->names, &c->name, &c->globals, &c->c_function, &c->stream, &c->dict}) Py_CLEAR(*o);
  return 0;
}
void call_dealloc(PyObject* self) {
  PyObject_GC_UnTrack(self);
  if (reinterpret_cast<Call*>(self)->weak_references) PyObject_ClearWeakRefs(self);
  call_clear(self);
  Py_TYPE(self)->tp_free(self);
}
PyObject* call_repr(PyObject* self) { return PyUnicode_FromFormat("<call %s>", reinterpret_cast<Call*>(self)->kind->name); }
// in a class it is a method, as a function is
PyObject* call_get(PyObject* self, PyObject* object, PyObject*) {
  if (object && object != Py_None) return PyMethod_New(self, object);
  Py_INCREF(self);
  return self;
}
PyObject* call_reduce(PyObject* self, PyObject*) { return PyUnicode_FromString(reinterpret_cast<Call*>(self)->kind->name); }

PyMethodDef call_methods[] = {{"__reduce__", call_reduce, METH_NOARGS, "pickled by name"}, {}};
PyGetSetDef call_getset[] = {{"__dict__", PyObject_GenericGetDict, PyObject_GenericSetDict, nullptr, nullptr}, {}};

PyTypeObject CallType = {PyVarObject_HEAD_INIT(nullptr, 0)};

// bind(name, python function, its parameter names, the ctypes function it calls, that function's address) -> callable
PyObject* bind(PyObject*, PyObject* args) {
  const char* name;
  PyObject *python, *names, *c_function;
  unsigned long long address;
  if (!PyArg_ParseTuple(args, "sO!O!OK", &name, &PyFunction_Type, &python, &PyTuple_Type, &names, &c_function, &address)) return nullptr;
  PyObject* const globals = PyFunction_GetGlobals(python);
  PyObject* const stream = PyDict_GetItemWithError(globals, g_stream_name);
  if (!stream) return PyErr_Format(PyExc_KeyError, "_stream");
  for (const Kind& k : kKinds)
    if (!strcmp(k.name, name)) {
      if (static_cast<size_t>(PyTuple_GET_SIZE(names)) != k.n_args)
        return PyErr_Format(PyExc_TypeError, "%s takes %zu arguments, its Python function %zd", name, k.n_args, PyTuple_GET_SIZE(names));
      PyObject* const interned = PyUnicode_InternFromString(name);
      Call* c = interned ? PyObject_GC_New(Call, &CallType) : nullptr;
      if (!c) {
        Py_XDECREF(interned);
        return nullptr;
      }
      c->vectorcall = call_vector;
      c->kind = &k;
      c->python = python, c->names = names, c->name = interned, c->globals = globals, c->c_function = c_function, c->stream = stream;
      c->address = reinterpret_cast<void (*)()>(address);
      c->dict = c->weak_references = nullptr;
      for (PyObject* o : {python, names, globals, c_function, stream}) Py_INCREF(o);
      PyObject_GC_Track(c);
      return reinterpret_cast<PyObject*>(c);
    }
  return PyErr_Format(PyExc_KeyError, "%s", name);
}

// init(cache class, predictor class, error check, torch.cuda.current_device, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
PyObject* init(PyObject*, PyObject* args) {
  PyObject* o[6];
  if (!PyArg_ParseTuple(args, "OOOOOO", &o[0], &o[1], &o[2], &o[3], &o[4], &o[5])) return nullptr;
  PyObject** const to[6] = {&g_cache_type, &g_predictor_type, &g_check, &g_current_device, &g_get_device, &g_raw_stream};
  for (int i = 0; i < 6; ++i) {
    Py_INCREF(o[i]);
    Py_XSETREF(*to[i], o[i]);
  }
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, "bind(name, function, parameter names, C function, its address): the native call of that name"},
                         {"init", init, METH_VARARGS, "init(classes and functions of the binding and of torch)"},
                         {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Native marshalling of the library's calls.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  CallType.tp_name = "paper_2412_00876_amd._calls.Call";
  CallType.tp_basicsize = sizeof(Call);
  CallType.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_GC | Py_TPFLAGS_HAVE_VECTORCALL;
  CallType.tp_vectorcall_offset = offsetof(Call, vectorcall);
  CallType.tp_dictoffset = offsetof(Call, dict);
  CallType.tp_weaklistoffset = offsetof(Call, weak_references);
  CallType.tp_descr_get = call_get;
  CallType.tp_call = PyVectorcall_Call;
  CallType.tp_traverse = call_traverse;
  CallType.tp_clear = call_clear;
  CallType.tp_dealloc = call_dealloc;
  CallType.tp_repr = call_repr;
  CallType.tp_methods = call_methods;
  CallType.tp_getset = call_getset;
  if (PyType_Ready(&CallType) < 0) return nullptr;
  if (!(g_c = PyUnicode_InternFromString("c")) || !(g_lib_name = PyUnicode_InternFromString("_lib")) ||
      !(g_stream_name = PyUnicode_InternFromString("_stream")) || !(g_check_name = PyUnicode_InternFromString("_check")))
    return nullptr;
  // in a forked child torch refuses the device: ask it again there
  pthread_atfork(nullptr, nullptr, [] { g_device_ready = false; });
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", DLLAVA_TORCH_VERSION) < 0) Py_CLEAR(m);
  return m;
}
