// The calls that a program makes for every block and every token, from Python tensors to the library's C functions in
// one native step.  A small decode step takes 5 to 7 us on the GPU; checking and marshalling its arguments in Python took
// 3.4 us of the 7.1 us that a step took on the host (the C call with its launch 2.7, ctypes 1.0).
//
// The functions return the library's status code (those of packed caches that make their outputs: the outputs, where it is 0), or
// None where an argument is not what they handle (a tensor subclass, a stream object, an index that is not an int): binding.py and
// packed.py then take their own, general way.  The checks are that way's checks and fail like them, with AssertionError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

typedef int32_t (*DecodeFn)(void*, int32_t, int32_t, int32_t, const void*, const void*, const void*, void*, int32_t, void*);
typedef int32_t (*PrefillFn)(void*, int32_t, int32_t, int32_t, const void*, const void*, const void*, int32_t, int32_t, void*,
                             int32_t, void*);

// int arguments args[0 .. n): false where one is no plain int of 32 bits
bool ints(PyObject* const* args, int n, int32_t* out) {
  for (int i = 0; i < n; ++i) {
    if (!PyLong_CheckExact(args[i])) return false;
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(args[i], &overflow);
    if (overflow != 0 || v < INT32_MIN || v > INT32_MAX) return false;
    out[i] = (int32_t)v;
  }
  return true;
}

// q, k, v, out: exact torch.Tensor objects with storage
bool tensors(PyObject* const* args, const at::Tensor** t) {
  for (int i = 0; i < 4; ++i) {
    if (!THPVariable_CheckExact(args[i])) return false;
    t[i] = &THPVariable_Unpack(args[i]);
    if (!t[i]->has_storage()) return false;
  }
  return true;
}

bool layouts_ok(const at::Tensor* const* t, bool bf16) {
  const at::ScalarType want = bf16 ? at::kBFloat16 : at::kFloat;
  if (!t[0]->is_contiguous() || !t[1]->is_contiguous() || !t[2]->is_contiguous() || t[0]->scalar_type() != want) {
    PyErr_SetNone(PyExc_AssertionError);
    return false;
  }
  if (!t[3]->is_contiguous() || t[3]->scalar_type() != want || !t[3]->sizes().equals(t[0]->sizes())) {
    PyErr_SetString(PyExc_AssertionError, "out must be a contiguous tensor of q's shape and dtype");
    return false;
  }
  return true;
}

// (function address, handle, bf16, q, k, v, out, layer, sample0, evict_to)
PyObject* decode(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int32_t x[3];
  const at::Tensor* t[4];
  if (n != 10 || !tensors(args + 3, t) || !ints(args + 7, 3, x) || t[0]->dim() < 1) Py_RETURN_NONE;
  void* fn = PyLong_AsVoidPtr(args[0]);
  void* h = PyLong_AsVoidPtr(args[1]);
  if (PyErr_Occurred() || !layouts_ok(t, args[2] == Py_True)) return nullptr;
  const void *q = t[0]->data_ptr(), *k = t[1]->data_ptr(), *v = t[2]->data_ptr();
  void* out = t[3]->data_ptr();
  const int32_t ns = (int32_t)t[0]->size(0);
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<DecodeFn>(fn)(h, x[0], x[1], ns, q, k, v, out, x[2], stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// (function address, handle, bf16, q, k, v, out, layer, sample0, evict_to, pos0)
PyObject* prefill(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int32_t x[4];
  const at::Tensor* t[4];
  if (n != 11 || !tensors(args + 3, t) || !ints(args + 7, 4, x) || t[0]->dim() < 2) Py_RETURN_NONE;
  void* fn = PyLong_AsVoidPtr(args[0]);
  void* h = PyLong_AsVoidPtr(args[1]);
  if (PyErr_Occurred() || !layouts_ok(t, args[2] == Py_True)) return nullptr;
  const void *q = t[0]->data_ptr(), *k = t[1]->data_ptr(), *v = t[2]->data_ptr();
  void* out = t[3]->data_ptr();
  const int32_t ns = (int32_t)t[0]->size(0), I = (int32_t)t[0]->size(1);
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<PrefillFn>(fn)(h, x[0], x[1], ns, q, k, v, I, x[3], out, x[2], stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// ---- packed caches ---------------------------------------------------------------------------------------------------
typedef int32_t (*PackedWriteFn)(void*, int32_t, int32_t, int32_t, const void*, const void*, const int64_t*, int32_t, const int32_t*,
                                 const int32_t*, void*);
typedef int32_t (*PackedReadFn)(void*, int32_t, int32_t, int32_t, int32_t, int32_t, const int32_t*, void*, void*, void*);
typedef int32_t (*PackedAttendFn)(void*, int32_t, int32_t, int32_t, const void*, const int64_t*, int32_t, const int32_t*, const int32_t*,
                                  int32_t, void*, void*, size_t, void*);

// (handle, bf16, device, q heads, kv heads, head_dim): what a handle's calls begin with, after the function's address
struct Packed {
  void* fn;
  void* handle;
  at::ScalarType type;
  int device;
  int64_t q_heads, kv_heads, d;
};
constexpr int kPackedArgs = 7;

bool packed(PyObject* const* args, Packed* p) {
  int32_t x[4];
  if (!ints(args + 3, 4, x)) return false;
  p->fn = PyLong_AsVoidPtr(args[0]);
  p->handle = PyLong_AsVoidPtr(args[1]);
  p->type = args[2] == Py_True ? at::kBFloat16 : at::kFloat;
  p->device = x[0];
  p->q_heads = x[1];
  p->kv_heads = x[2];
  p->d = x[3];
  return !PyErr_Occurred() && p->handle != nullptr;
}

// an exact torch.Tensor with storage, or (optional) None
bool tensor(PyObject* arg, bool optional, const at::Tensor** t) {
  *t = nullptr;
  if (arg == Py_None) return optional;
  if (!THPVariable_CheckExact(arg)) return false;
  *t = &THPVariable_Unpack(arg);
  return (*t)->has_storage();
}

bool fail(const char* text) {
  PyErr_SetString(PyExc_AssertionError, text);
  return false;
}

bool on_device(const at::Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }

// (nsamples, I, heads, d): a token's heads lie together, samples and tokens may be strided
bool rows_ok(const at::Tensor& t, int64_t heads, const Packed& p, int64_t* strides) {
  if (t.dim() != 4 || t.size(2) != heads || t.size(3) != p.d || t.size(0) < 1 || t.size(1) < 1 || t.scalar_type() != p.type ||
      !on_device(t, p.device))
    return fail("rows must be (nsamples, I, heads, head_dim) tensors of the handle's dtype on its device");
  if (t.stride(3) != 1 || (t.stride(2) != p.d && heads != 1)) return fail("a token's heads must lie together");
  strides[0] = t.size(0) > 1 ? t.stride(0) : 0;
  strides[1] = t.size(1) > 1 ? t.stride(1) : 0;
  return true;
}

bool index_ok(const at::Tensor* t, int64_t n, const Packed& p, const int32_t** out) {
  *out = nullptr;
  if (t == nullptr) return true;
  if (t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != n || !t->is_contiguous() || !on_device(*t, p.device))
    return fail("lengths and rows must be contiguous int32 tensors of one entry per sample on the handle's device");
  *out = static_cast<const int32_t*>(t->data_ptr());
  return true;
}

// a new tensor, straight from the allocator (through the dispatcher 0.5 us more)
at::Tensor make(at::IntArrayRef sizes, const Packed& p) {
  return at::detail::empty_cuda(sizes, p.type, c10::Device(c10::kCUDA, (c10::DeviceIndex)p.device), std::nullopt);
}

bool fits(int64_t x) { return x <= INT32_MAX; }

// (Packed ..., k, v, start, counts, layer, sample0)
PyObject* packed_write(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Packed p;
  const at::Tensor *k, *v, *start, *counts;
  int32_t x[2];
  PyObject* const* a = args + kPackedArgs;
  if (n != kPackedArgs + 6 || !tensor(a[0], false, &k) || !tensor(a[1], false, &v) || !tensor(a[2], true, &start) ||
      !tensor(a[3], true, &counts) || !ints(a + 4, 2, x))
    Py_RETURN_NONE;
  if (!packed(args, &p)) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  int64_t strides[4];
  const int32_t *rows, *limits;
  if (!v->sizes().equals(k->sizes())) return fail("k and v must have one shape"), nullptr;
  if (!rows_ok(*k, p.kv_heads, p, strides) || !rows_ok(*v, p.kv_heads, p, strides + 2) || !index_ok(start, k->size(0), p, &rows) ||
      !index_ok(counts, k->size(0), p, &limits))
    return nullptr;
  if (!fits(k->size(0)) || !fits(k->size(1))) Py_RETURN_NONE;
  void* stream = c10::cuda::getCurrentCUDAStream(p.device).stream();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<PackedWriteFn>(p.fn)(p.handle, x[0], x[1], (int32_t)k->size(0), k->data_ptr(), v->data_ptr(), strides,
                                                           (int32_t)k->size(1), rows, limits,
                                                           stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// (Packed ..., row0, rows, layer, sample0, nsamples, lens): (k, v), or the status code that is not 0
PyObject* packed_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Packed p;
  const at::Tensor* lens;
  int32_t x[5];
  PyObject* const* a = args + kPackedArgs;
  if (n != kPackedArgs + 6 || !ints(a, 5, x) || !tensor(a[5], true, &lens) || x[1] < 1 || x[4] < 1) Py_RETURN_NONE;
  if (!packed(args, &p)) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  const int32_t* limits;
  if (!index_ok(lens, x[4], p, &limits)) return nullptr;
  at::Tensor k = make({x[4], x[1], p.kv_heads, p.d}, p), v = make({x[4], x[1], p.kv_heads, p.d}, p);
  void* stream = c10::cuda::getCurrentCUDAStream(p.device).stream();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<PackedReadFn>(p.fn)(p.handle, x[2], x[3], x[4], x[0], x[1], limits, k.data_ptr(), v.data_ptr(),
                                                          stream);
  Py_END_ALLOW_THREADS
  if (rc != 0) return PyLong_FromLong(rc);
  PyObject* both = PyTuple_New(2);
  if (both == nullptr) return nullptr;
  PyTuple_SET_ITEM(both, 0, THPVariable_Wrap(std::move(k)));
  PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(std::move(v)));
  return both;
  END_HANDLE_TH_ERRORS
}

// (Packed ..., q, lens, first, out, workspace, max_len, layer, sample0): out, or the status code that is not 0
PyObject* packed_attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Packed p;
  const at::Tensor *q, *lens, *first, *out, *workspace;
  int32_t x[3];
  PyObject* const* a = args + kPackedArgs;
  if (n != kPackedArgs + 8 || !tensor(a[0], false, &q) || !tensor(a[1], false, &lens) || !tensor(a[2], true, &first) ||
      !tensor(a[3], true, &out) || !tensor(a[4], false, &workspace) || !ints(a + 5, 3, x))
    Py_RETURN_NONE;
  if (!packed(args, &p)) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  int64_t strides[2];
  const int32_t *lengths, *firsts;
  if (!rows_ok(*q, p.q_heads, p, strides) || !index_ok(lens, q->size(0), p, &lengths) || !index_ok(first, q->size(0), p, &firsts))
    return nullptr;
  if (out != nullptr && (!out->is_contiguous() || out->scalar_type() != p.type || !out->sizes().equals(q->sizes()) || !on_device(*out, p.device)))
    return fail("out must be a contiguous tensor of q's shape and dtype"), nullptr;
  if (workspace->scalar_type() != at::kByte || !workspace->is_contiguous() || !on_device(*workspace, p.device))
    return fail("arena and workspace must be contiguous uint8 tensors on the handle's device"), nullptr;
  if (!fits(q->size(0)) || !fits(q->size(1))) Py_RETURN_NONE;
  at::Tensor made;
  if (out == nullptr) {
    made = make(q->sizes(), p);
    out = &made;
  }
  void* stream = c10::cuda::getCurrentCUDAStream(p.device).stream();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = reinterpret_cast<PackedAttendFn>(p.fn)(p.handle, x[1], x[2], (int32_t)q->size(0), q->data_ptr(), strides,
                                                            (int32_t)q->size(1), lengths, firsts, x[0], out->data_ptr(),
                                                            workspace->data_ptr(), (size_t)workspace->numel(),
                                                            stream);
  Py_END_ALLOW_THREADS
  if (rc != 0) return PyLong_FromLong(rc);
  if (made.defined()) return THPVariable_Wrap(std::move(made));
  Py_INCREF(a[3]);
  return a[3];
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode)), METH_FASTCALL, nullptr},
    {"prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prefill)), METH_FASTCALL, nullptr},
    {"packed_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(packed_write)), METH_FASTCALL, nullptr},
    {"packed_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(packed_read)), METH_FASTCALL, nullptr},
    {"packed_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(packed_attend)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
