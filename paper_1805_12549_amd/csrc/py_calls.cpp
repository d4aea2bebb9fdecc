// The calls a program makes per forward pass, as a Python extension: what binding.py does with ctypes, without the interpreter's part of it.
//
// One image through ResNet-18 was 22 launches of 3 to 9 us each (19 now); with tensors, workspace and arguments handled in Python a call took 5.0 us of host time
// (7.8 where it allocates its output, 11.6 with bitmap and counts too) beside the 2.7 us of a launch, and the GPU waited for the host.
//
// Only what a plain call needs is here.  A call with anything else - a tensor subclass, an active __torch_function__ mode, symbolic sizes, an argument
// that is no tensor - returns None, and binding.py takes it.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/HIPContextLight.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cg_calls.h"
#include "cg_conv.h"

namespace {

// A layer as its calls see it; the handle is binding.py's, which drops this object before it destroys the handle.
struct Layer {
  PyObject_HEAD
  cg_conv* handle;
  int64_t ho, wo, c_out, words;
  at::ScalarType y_type;
};

// memory of the caching allocator that belongs to one stream, given back at the end of the call: it then serves later work of the same stream only, and
// under capture it is the graph's own
struct Scratch {
  void* ptr = nullptr;
  Scratch(size_t bytes, hipStream_t stream) {
    if (bytes) ptr = c10::hip::HIPCachingAllocator::raw_alloc_with_stream(bytes, stream);
  }
  ~Scratch() {
    if (ptr) c10::hip::HIPCachingAllocator::raw_delete(ptr);
  }
};

struct WithoutGil {
  PyThreadState* state = PyEval_SaveThread();
  ~WithoutGil() { PyEval_RestoreThread(state); }
};

extern PyTypeObject layer_type;

bool plain_tensor(PyObject* o) { return THPVariable_CheckExact(o); }

// an output argument: True (allocate), False / None (leave out), a tensor; anything else: false
bool wanted(PyObject* o, bool& make, at::Tensor& given) {
  if (o == Py_True) {
    make = true;
  } else if (o != Py_False && o != Py_None) {
    if (!plain_tensor(o)) return false;
    given = THPVariable_Unpack(o);
  }
  return true;
}

// forward(layer, stream, x, residual, y, bitmap, counts): (y, bitmap, counts); an error code; None: not a plain call
PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 7) {
    PyErr_SetString(PyExc_TypeError, "forward takes seven arguments");
    return nullptr;
  }
  if (Py_TYPE(args[0]) != &layer_type) {
    PyErr_SetString(PyExc_TypeError, "forward's first argument is a Layer");
    return nullptr;
  }
  const Layer* const l = (const Layer*)args[0];
  PyObject *const stream_arg = args[1], *const residual_arg = args[3], *const y_arg = args[4];
  if (at::impl::torch_function_mode_enabled() || !plain_tensor(args[2])) Py_RETURN_NONE;
  if (residual_arg != Py_None && !plain_tensor(residual_arg)) Py_RETURN_NONE;
  if (y_arg != Py_None && !plain_tensor(y_arg)) Py_RETURN_NONE;
  bool make_bitmap = false, make_counts = false;
  at::Tensor residual, y, bitmap, counts;
  if (!wanted(args[5], make_bitmap, bitmap) || !wanted(args[6], make_counts, counts)) Py_RETURN_NONE;
  const at::Tensor& x = THPVariable_Unpack(args[2]);
  if (x.unsafeGetTensorImpl()->has_symbolic_sizes_strides() || x.dim() == 0) Py_RETURN_NONE;
  if (residual_arg != Py_None) residual = THPVariable_Unpack(residual_arg);
  if (y_arg != Py_None) y = THPVariable_Unpack(y_arg);
  hipStream_t stream;
  if (stream_arg == Py_None) {
    stream = c10::hip::getCurrentHIPStream().stream();
  } else {
    PyObject* const address = PyObject_GetAttrString(stream_arg, "cuda_stream");
    if (!address) return nullptr;
    stream = (hipStream_t)PyLong_AsVoidPtr(address);
    Py_DECREF(address);
    if (PyErr_Occurred()) return nullptr;
  }
  int rc;
  {
    const WithoutGil released;
    const int64_t n = x.size(0), ho = l->ho, wo = l->wo, c = l->c_out;
    const at::TensorOptions here = at::TensorOptions().device(x.device());
    if (!y.defined()) y = at::empty_strided({n, ho, wo, c}, {ho * wo * c, wo * c, c, 1}, here.dtype(l->y_type));
    if (make_bitmap) bitmap = at::empty_strided({n * ho * wo, l->words}, {l->words, 1}, here.dtype(at::kInt));
    if (make_counts) counts = at::empty({2 + n * c}, here.dtype(at::kInt));
    const size_t need = cg_conv_call_scratch_bytes(l->handle, (int32_t)n, bitmap.defined(), counts.defined());
    const Scratch scratch(need, stream);
    rc = cg_conv_call(l->handle, (int32_t)n, x.data_ptr(), residual.defined() ? residual.data_ptr() : nullptr, y.data_ptr(),
                      bitmap.defined() ? (uint32_t*)bitmap.data_ptr() : nullptr, counts.defined() ? (uint32_t*)counts.data_ptr() : nullptr,
                      scratch.ptr, need, stream);
  }
  if (rc != CG_OK) return PyLong_FromLong(rc);
  PyObject* const out = PyTuple_New(3);
  if (!out) return nullptr;
  const auto put = [&](int at, PyObject* given, bool made, const at::Tensor& t) {
    PyObject* o = made ? THPVariable_Wrap(t) : t.defined() ? given : Py_None;
    if (!made) Py_INCREF(o);
    PyTuple_SET_ITEM(out, at, o);
  };
  put(0, y_arg, y_arg == Py_None, y);
  put(1, args[5], make_bitmap, bitmap);
  put(2, args[6], make_counts, counts);
  return out;
  END_HANDLE_TH_ERRORS
}

// empty_bf16(like, sizes ...): a contiguous bf16 tensor on the device of `like`; None: not a plain tensor
PyObject* empty_bf16(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args < 2 || n_args > 5) {
    PyErr_SetString(PyExc_TypeError, "empty_bf16 takes a tensor and one to four sizes");
    return nullptr;
  }
  if (at::impl::torch_function_mode_enabled() || !plain_tensor(args[0])) Py_RETURN_NONE;
  const at::Tensor& like = THPVariable_Unpack(args[0]);
  int64_t sizes[4];
  for (Py_ssize_t i = 1; i < n_args; ++i) {
    sizes[i - 1] = PyLong_AsLongLong(args[i]);
    if (sizes[i - 1] == -1 && PyErr_Occurred()) return nullptr;
  }
  at::Tensor t;
  {
    const WithoutGil released;
    t = at::empty(at::IntArrayRef(sizes, n_args - 1), at::TensorOptions().device(like.device()).dtype(at::kBFloat16));
  }
  return THPVariable_Wrap(t);
  END_HANDLE_TH_ERRORS
}

// What the operators behind the classifier are given, as binding.py checks it; false: something that it has to look at (and to refuse, as a rule)
struct Logits {
  const at::Tensor* t = nullptr;
  int32_t dtype = 0;
  int64_t rows = 0, classes = 0, stride = 0;
  bool take(PyObject* o) {
    if (!plain_tensor(o)) return false;
    t = &THPVariable_Unpack(o);
    if (t->unsafeGetTensorImpl()->has_symbolic_sizes_strides() || t->dim() != 2 || !t->is_cuda() || t->get_device() != c10::hip::current_device()) return false;
    if (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16) return false;
    dtype = t->scalar_type() == at::kFloat ? CG_F32 : CG_BF16;
    rows = t->size(0), classes = t->size(1), stride = t->stride(0);
    return classes > 0 && classes <= INT32_MAX && (classes == 1 || t->stride(1) == 1);
  }
  // A contiguous tensor on the current device, where the logits are, in memory of its own: it is kept and saved without the call's others.  From torch's
  // allocator directly: the way through the dispatcher costs each 0.2 us more of host time (one image's answer of four tensors 5.4 us, by at::empty 6.2).
  at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type) const {
    return at::detail::empty_generic(sizes, at::cuda::getCUDADeviceAllocator(), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
  }
  // a contiguous tensor of that type beside the logits, or None
  bool beside(PyObject* o, at::ScalarType type, at::IntArrayRef sizes, const void*& ptr) const {
    if (o == Py_None) return true;
    if (!plain_tensor(o)) return false;
    const at::Tensor& b = THPVariable_Unpack(o);
    if (b.unsafeGetTensorImpl()->has_symbolic_sizes_strides() || b.scalar_type() != type || b.device() != t->device() || b.sizes() != sizes ||
        !b.is_contiguous())
      return false;
    ptr = b.data_ptr();
    return true;
  }
  // where the gradient goes: None or True (a new tensor, each of whose rows is aligned to 16 bytes as the logits' row is) or a tensor
  bool gradient(PyObject* o, at::Tensor& grad) const {
    if (o == Py_None || o == Py_True) {
      const int64_t size = dtype == CG_F32 ? 4 : 2, per = 16 / size, step = classes + ((stride - classes) % per + per) % per;
      const int64_t phase = rows ? (int64_t)((uintptr_t)t->data_ptr() % 16) / size : 0;
      grad = fresh({rows ? phase + (rows - 1) * step + classes : 0}, t->scalar_type());
      grad.unsafeGetTensorImpl()->set_sizes_and_strides(t->sizes(), at::IntArrayRef{step, 1}, phase);
      return true;
    }
    if (!plain_tensor(o)) return false;
    grad = THPVariable_Unpack(o);
    return !grad.unsafeGetTensorImpl()->has_symbolic_sizes_strides() && grad.scalar_type() == t->scalar_type() && grad.sizes() == t->sizes() &&
           grad.device() == t->device() && (classes == 1 || grad.stride(1) == 1);
  }
};

// a Python float or int, as binding.py passes it to ctypes
bool number(PyObject* o, float& v) {
  if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
  const double d = PyFloat_AsDouble(o);
  if (d == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  v = (float)d;
  return true;
}

// logprobs(logits, labels, top, temperature, entropy): (logprob, entropy, top_ids, top_logprobs); an error code; None: not a plain call
PyObject* logprobs(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 5) {
    PyErr_SetString(PyExc_TypeError, "logprobs takes five arguments");
    return nullptr;
  }
  Logits z;
  float temperature;
  if (at::impl::torch_function_mode_enabled() || !z.take(args[0]) || !PyLong_CheckExact(args[2]) || !number(args[3], temperature)) Py_RETURN_NONE;
  const long long top = PyLong_AsLongLong(args[2]);
  if (top < 0 || top > z.classes || top > CG_TOP_MAX) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  const int entropy_wanted = PyObject_IsTrue(args[4]);
  if (entropy_wanted < 0) return nullptr;
  const void* labels_ptr = nullptr;
  const at::Tensor* labels = nullptr;
  int64_t given = 0;
  if (args[1] != Py_None) {
    if (!plain_tensor(args[1])) Py_RETURN_NONE;
    labels = &THPVariable_Unpack(args[1]);
    if (labels->dim() < 1 || labels->dim() > 2 || labels->size(0) != z.rows || !z.beside(args[1], at::kLong, labels->sizes(), labels_ptr)) Py_RETURN_NONE;
    given = labels->dim() == 1 ? 1 : labels->size(1);
    if (given > INT32_MAX) Py_RETURN_NONE;
  }
  at::Tensor logprob, entropy, top_ids, top_logprobs;
  int rc;
  {
    const WithoutGil released;
    const hipStream_t stream = c10::hip::getCurrentHIPStream().stream();
    if (labels) logprob = z.fresh(labels->sizes(), at::kFloat);
    if (entropy_wanted) entropy = z.fresh({z.rows}, at::kFloat);
    if (top) {
      top_ids = z.fresh({z.rows, top}, at::kLong);
      top_logprobs = z.fresh({z.rows, top}, at::kFloat);
    }
    const size_t need = cg_logprobs_workspace_bytes(z.rows, (int32_t)z.classes, (int32_t)top);
    const Scratch scratch(need, stream);
    const auto at = [](const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
    rc = cg_logprobs(z.t->data_ptr(), z.dtype, z.rows, (int32_t)z.classes, z.stride, temperature, (const int64_t*)labels_ptr, (int32_t)given, (int32_t)top,
                     (float*)at(logprob), (float*)at(entropy), (int64_t*)at(top_ids), (float*)at(top_logprobs), scratch.ptr, need, stream);
  }
  if (rc != CG_OK) return PyLong_FromLong(rc);
  PyObject* const out = PyTuple_New(4);
  if (!out) return nullptr;
  const at::Tensor* const made[4] = {&logprob, &entropy, &top_ids, &top_logprobs};
  for (int i = 0; i < 4; ++i) {
    PyObject* o = Py_None;
    if (made[i]->defined())
      o = THPVariable_Wrap(*made[i]);
    else
      Py_INCREF(o);
    PyTuple_SET_ITEM(out, i, o);
  }
  return out;
  END_HANDLE_TH_ERRORS
}

// distill(logits, stats, top_ids, top_logits, labels, teacher_weight, label_weight, temperature, grad, grad_loss): (loss, stats, grad), or with stats
// given the gradient alone; an error code; None: not a plain call
PyObject* distill(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 10) {
    PyErr_SetString(PyExc_TypeError, "distill takes ten arguments");
    return nullptr;
  }
  Logits z;
  float w_teacher, w_label, temperature;
  if (at::impl::torch_function_mode_enabled() || !z.take(args[0]) || !number(args[5], w_teacher) || !number(args[6], w_label) ||
      !number(args[7], temperature))
    Py_RETURN_NONE;
  int64_t top = 0;
  if ((args[2] == Py_None) != (args[3] == Py_None)) Py_RETURN_NONE;
  if (args[2] != Py_None) {
    if (!plain_tensor(args[2]) || THPVariable_Unpack(args[2]).dim() != 2) Py_RETURN_NONE;
    top = THPVariable_Unpack(args[2]).size(1);
    if (top > CG_TOP_MAX) Py_RETURN_NONE;
  }
  const void *ids = nullptr, *top_logits = nullptr, *labels = nullptr, *up = nullptr, *given_stats = nullptr;
  if (!z.beside(args[2], at::kLong, {z.rows, top}, ids) || !z.beside(args[3], at::kFloat, {z.rows, top}, top_logits) ||
      !z.beside(args[4], at::kLong, {z.rows}, labels) || !z.beside(args[9], at::kFloat, {z.rows}, up) || !z.beside(args[1], at::kFloat, {z.rows, 3}, given_stats))
    Py_RETURN_NONE;
  const bool backward = args[1] != Py_None, want = backward || (args[8] != Py_None && args[8] != Py_False);
  at::Tensor grad, loss, stats;
  if (want && !z.gradient(args[8], grad)) Py_RETURN_NONE;
  int rc;
  {
    const WithoutGil released;
    const hipStream_t stream = c10::hip::getCurrentHIPStream().stream();
    if (backward) {
      rc = cg_distill_backward(z.t->data_ptr(), z.dtype, z.rows, (int32_t)z.classes, z.stride, temperature, (const int64_t*)ids, (const float*)top_logits,
                               (int32_t)top, (const int64_t*)labels, w_teacher, w_label, (const float*)given_stats, (const float*)up, grad.data_ptr(),
                               grad.stride(0), stream);
    } else {
      loss = z.fresh({z.rows}, at::kFloat);
      stats = z.fresh({z.rows, 3}, at::kFloat);
      const size_t need = cg_distill_workspace_bytes(z.rows, (int32_t)z.classes);
      const Scratch scratch(need, stream);
      rc = cg_distill_forward(z.t->data_ptr(), z.dtype, z.rows, (int32_t)z.classes, z.stride, temperature, (const int64_t*)ids, (const float*)top_logits,
                              (int32_t)top, (const int64_t*)labels, w_teacher, w_label, (float*)loss.data_ptr(), (float*)stats.data_ptr(),
                              (const float*)up, want ? grad.data_ptr() : nullptr, want ? grad.stride(0) : 0, scratch.ptr, need, stream);
    }
  }
  if (rc != CG_OK) return PyLong_FromLong(rc);
  PyObject* g = want && plain_tensor(args[8]) ? args[8] : Py_None;
  if (want && g == Py_None)
    g = THPVariable_Wrap(grad);
  else
    Py_INCREF(g);
  if (backward) return g;
  PyObject* const out = PyTuple_New(3);
  if (!out) {
    Py_DECREF(g);
    return nullptr;
  }
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(loss));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(stats));
  PyTuple_SET_ITEM(out, 2, g);
  return out;
  END_HANDLE_TH_ERRORS
}

int layer_init(PyObject* self, PyObject* args, PyObject*) {
  Layer* const l = (Layer*)self;
  unsigned long long handle;
  long long ho, wo, c_out;
  int out_dtype;
  if (!PyArg_ParseTuple(args, "KLLLi", &handle, &ho, &wo, &c_out, &out_dtype)) return -1;
  l->handle = (cg_conv*)handle;
  l->ho = ho;
  l->wo = wo;
  l->c_out = c_out;
  l->words = (c_out + 31) / 32;
  l->y_type = out_dtype == CG_F32 ? at::kFloat : out_dtype == CG_BF16 ? at::kBFloat16 : out_dtype == CG_I8 ? at::kChar : at::kInt;
  return 0;
}

PyTypeObject layer_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyMethodDef methods[] = {
    {"forward", (PyCFunction)(void (*)(void))forward, METH_FASTCALL, "forward(layer, stream, x, residual, y, bitmap, counts)"},
    {"empty_bf16", (PyCFunction)(void (*)(void))empty_bf16, METH_FASTCALL, "empty_bf16(like, *sizes)"},
    {"logprobs", (PyCFunction)(void (*)(void))logprobs, METH_FASTCALL, "logprobs(logits, labels, top, temperature, entropy)"},
    {"distill", (PyCFunction)(void (*)(void))distill, METH_FASTCALL,
     "distill(logits, stats, top_ids, top_logits, labels, teacher_weight, label_weight, temperature, grad, grad_loss)"},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Forward calls without the interpreter's part of them.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
  layer_type.tp_name = "_calls.Layer";
  layer_type.tp_basicsize = sizeof(Layer);
  layer_type.tp_flags = Py_TPFLAGS_DEFAULT;
  layer_type.tp_doc = "Layer(handle, ho, wo, c_out, out_dtype)";
  layer_type.tp_new = PyType_GenericNew;
  layer_type.tp_init = layer_init;
  if (PyType_Ready(&layer_type) < 0) return nullptr;
  PyObject* const m = PyModule_Create(&module);
  if (!m) return nullptr;
  // (torch's objects are read as this version lays them out)
  if (PyModule_AddStringConstant(m, "torch_version", CG_TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  Py_INCREF(&layer_type);
  if (PyModule_AddObject(m, "Layer", (PyObject*)&layer_type) < 0) {
    Py_DECREF(&layer_type);
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
