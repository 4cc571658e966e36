// _marshal_torch_<version>: the part of the Python binding that runs several times per argument of every operator call. It looks at
// what the library cannot see of a tensor (type, device, shape, layout) and puts its address and strides where the C ABI
// wants them. A tensor that is not as it should be goes to the binding's own Python functions, which say what is wrong with
// it or accept it (subclasses of Tensor). One token through the norm operator, 8 tensors: 10.8 us a call with these checks
// in Python, 9.6 in C through the tensors' Python attributes, 6.5 as here.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAStream.h>

static PyObject *careful_flat, *careful_heads, *careful_rows, *careful_tensor; // set by setup()
static thread_local int device = 0;            // of the call whose argument block was asked for last

typedef struct { // slidedp_heads
  uint64_t data;
  int64_t stride_token, stride_head;
} heads_view;

typedef struct { // slidedp_rows
  uint64_t data;
  int64_t stride;
} rows_view;

typedef struct { // slidedp_tensor
  uint64_t data;
  int64_t count;
  int32_t dtype, reserved;
} tensor_view;

// Whether x is a Tensor or Parameter of this dtype and shape (a tuple, or None) on the call's GPU.
static bool plain(PyObject* x, PyObject* dtype, PyObject* shape) {
  if (!THPVariable_CheckExact(x) || !THPDtype_Check(dtype)) return false;
  const at::Tensor& t = THPVariable_Unpack(x);
  if (t.scalar_type() != reinterpret_cast<THPDtype*>(dtype)->scalar_type || !t.is_cuda() || t.get_device() != device) return false;
  if (shape == Py_None) return true;
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != t.dim()) return false;
  for (int64_t i = 0; i < t.dim(); ++i) {
    if (PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)) == t.size(i)) continue;
    PyErr_Clear();
    return false;
  }
  return true;
}

// flat(x, what, dtype, shape or None): address of a contiguous tensor
static PyObject* flat(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3 && n != 4) return PyErr_Format(PyExc_TypeError, "flat takes 3 or 4 arguments");
  PyObject *x = args[0], *shape = n == 4 ? args[3] : Py_None;
  if (plain(x, args[2], shape) && THPVariable_Unpack(x).is_contiguous()) return PyLong_FromVoidPtr(THPVariable_Unpack(x).data_ptr());
  return PyObject_CallFunctionObjArgs(careful_flat, x, args[1], args[2], shape, NULL);
}

static bool view_of(PyObject* x, PyObject* what, PyObject* dtype, PyObject* shape, heads_view* v) {
  if (plain(x, dtype, shape)) {
    const at::Tensor& t = THPVariable_Unpack(x);
    if (t.dim() == 3 && t.stride(2) == 1) {
      *v = heads_view{reinterpret_cast<uint64_t>(t.data_ptr()), t.stride(0), t.stride(1)};
      return true;
    }
  }
  PyObject* r = PyObject_CallFunctionObjArgs(careful_heads, x, what, dtype, shape, NULL);
  if (!r) return false;
  unsigned long long data;
  long long a, b;
  const bool got = PyArg_ParseTuple(r, "KLL", &data, &a, &b);
  Py_DECREF(r);
  if (got) *v = heads_view{data, a, b};
  return got;
}

// heads(at, dtype, shape, x0, what0, x1, what1, ..): the tensors' views, one after the other from address `at` on
static PyObject* heads(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 3 || n % 2 == 0) return PyErr_Format(PyExc_TypeError, "heads takes an address, a dtype, a shape and pairs");
  heads_view* out = static_cast<heads_view*>(PyLong_AsVoidPtr(args[0]));
  if (PyErr_Occurred()) return NULL;
  for (Py_ssize_t i = 3; i < n; i += 2)
    if (!view_of(args[i], args[i + 1], args[1], args[2], out++)) return NULL;
  Py_RETURN_NONE;
}

static bool rows_of(PyObject* x, PyObject* what, PyObject* dtype, PyObject* shape, rows_view* v) {
  if (x == Py_None) {
    *v = rows_view{0, 0};
    return true;
  }
  if (plain(x, dtype, shape)) {
    const at::Tensor& t = THPVariable_Unpack(x);
    if (t.dim() == 2 && t.stride(1) == 1) {
      *v = rows_view{reinterpret_cast<uint64_t>(t.data_ptr()), t.stride(0)};
      return true;
    }
  }
  PyObject* r = PyObject_CallFunctionObjArgs(careful_rows, x, what, dtype, shape, NULL);
  if (!r) return false;
  unsigned long long data;
  long long a;
  const bool got = PyArg_ParseTuple(r, "KL", &data, &a);
  Py_DECREF(r);
  if (got) *v = rows_view{data, a};
  return got;
}

// rows(at, dtype, shape, x0, what0, x1, what1, ..): the matrices' views, one after the other from address `at` on; None: no data
static PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 3 || n % 2 == 0) return PyErr_Format(PyExc_TypeError, "rows takes an address, a dtype, a shape and pairs");
  rows_view* out = static_cast<rows_view*>(PyLong_AsVoidPtr(args[0]));
  if (PyErr_Occurred()) return NULL;
  for (Py_ssize_t i = 3; i < n; i += 2)
    if (!rows_of(args[i], args[i + 1], args[1], args[2], out++)) return NULL;
  Py_RETURN_NONE;
}

// tensors(sequence, what): the bytes of an array of slidedp_tensor
static PyObject* tensors(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) return PyErr_Format(PyExc_TypeError, "tensors takes a sequence and its name");
  PyObject* all = PySequence_Fast(args[0], "tensors must come as a sequence");
  if (!all) return NULL;
  const Py_ssize_t count = PySequence_Fast_GET_SIZE(all);
  PyObject* bytes = PyBytes_FromStringAndSize(NULL, count * (Py_ssize_t)sizeof(tensor_view));
  tensor_view* out = bytes ? reinterpret_cast<tensor_view*>(PyBytes_AS_STRING(bytes)) : NULL;
  for (Py_ssize_t i = 0; bytes && i < count; ++i) {
    PyObject* x = PySequence_Fast_GET_ITEM(all, i);
    if (THPVariable_CheckExact(x)) {
      const at::Tensor& t = THPVariable_Unpack(x);
      const bool f32 = t.scalar_type() == at::kFloat;
      if ((f32 || t.scalar_type() == at::kBFloat16) && t.is_cuda() && t.get_device() == device && t.is_contiguous()) {
        out[i] = tensor_view{reinterpret_cast<uint64_t>(t.data_ptr()), t.numel(), f32 ? 1 : 0, 0};
        continue;
      }
    }
    PyObject* r = PyObject_CallFunctionObjArgs(careful_tensor, x, args[1], NULL);
    unsigned long long data;
    long long numel;
    int dtype;
    if (r && PyArg_ParseTuple(r, "KLi", &data, &numel, &dtype)) out[i] = tensor_view{data, numel, dtype, 0};
    else Py_CLEAR(bytes);
    Py_XDECREF(r);
  }
  Py_DECREF(all);
  return bytes;
}

// block(device): address of this thread's argument block, free for use until its next call; tensors are to be on that GPU
static PyObject* block(PyObject*, PyObject* on) {
  static thread_local uint64_t bytes[64];
  const long d = PyLong_AsLong(on);
  if (d == -1 && PyErr_Occurred()) return NULL;
  device = (int)d;
  return PyLong_FromVoidPtr(bytes);
}

// device(): the one given to block
static PyObject* expected_device(PyObject*, PyObject*) { return PyLong_FromLong(device); }

// current_stream(device): the handle of torch's current stream there; -1: on the current device
static PyObject* current_stream(PyObject*, PyObject* on) {
  const long d = PyLong_AsLong(on);
  if (d == -1 && PyErr_Occurred()) return NULL;
  return PyLong_FromVoidPtr(c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)d).stream());
}

// setup(functions for flat, heads, rows and the members of tensors)
static PyObject* setup(PyObject*, PyObject* args) {
  PyObject* f[4];
  if (!PyArg_ParseTuple(args, "OOOO", &f[0], &f[1], &f[2], &f[3])) return NULL;
  PyObject** const to[4] = {&careful_flat, &careful_heads, &careful_rows, &careful_tensor};
  for (int i = 0; i < 4; ++i) {
    Py_INCREF(f[i]);
    Py_XSETREF(*to[i], f[i]);
  }
  Py_RETURN_NONE;
}

// No C++ exception leaves a function called by the interpreter.
template <typename F>
static PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return PyErr_Format(PyExc_RuntimeError, "%s", e.what());
  }
}
static PyObject* py_flat(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  return guarded([&] { return flat(self, args, n); });
}
static PyObject* py_heads(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  return guarded([&] { return heads(self, args, n); });
}
static PyObject* py_rows(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  return guarded([&] { return rows(self, args, n); });
}
static PyObject* py_tensors(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  return guarded([&] { return tensors(self, args, n); });
}
static PyObject* py_current_stream(PyObject* self, PyObject* on) {
  return guarded([&] { return current_stream(self, on); });
}

static PyMethodDef methods[] = {{"flat", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_flat)), METH_FASTCALL, NULL},
                                {"heads", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_heads)), METH_FASTCALL, NULL},
                                {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_rows)), METH_FASTCALL, NULL},
                                {"tensors", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_tensors)), METH_FASTCALL, NULL},
                                {"block", block, METH_O, NULL},
                                {"device", expected_device, METH_NOARGS, NULL},
                                {"current_stream", py_current_stream, METH_O, NULL},
                                {"setup", setup, METH_VARARGS, NULL},
                                {NULL, NULL, 0, NULL}};
#define MARSHAL_TEXT2(x) #x
#define MARSHAL_TEXT(x) MARSHAL_TEXT2(x)
#define MARSHAL_INIT2(x) PyInit_##x
#define MARSHAL_INIT(x) MARSHAL_INIT2(x)
static PyModuleDef module = {PyModuleDef_HEAD_INIT, MARSHAL_TEXT(MARSHAL_NAME), NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC MARSHAL_INIT(MARSHAL_NAME)(void) { return PyModule_Create(&module); }
