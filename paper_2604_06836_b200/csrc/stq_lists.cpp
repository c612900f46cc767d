// What a call over a list of tensors has to know of each, gathered in one pass of C++ over the list (through the interpreter every
// question costs 0.1 us a tensor, and a model has hundreds).  A Python module, STQ_LISTS, named after the torch that it was built for;
// libstq itself does not know torch.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "../../include/stq.h"

namespace {

// Type code of a gradient, or -1.
int code_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return STQ_GRAD_F32;
    case at::kBFloat16: return STQ_GRAD_BF16;
    case at::kHalf: return STQ_GRAD_F16;
    default: return -1;
  }
}

bool refuse(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  return false;
}

// The tensor that a list's entry is, or null where a call does not take it.  (A pointer into the entry, which the list holds: one more
// owner of a tensor, for a moment, costs 65 ns, all the rest of a tensor 30.)
const at::Tensor* take(PyObject* o, const char* name, long dev, bool dense) {
  if (!THPVariable_Check(o)) return refuse(std::string(name) + " are tensors"), nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.get_device() != dev) return refuse(std::string(name) + " live on the handle's device"), nullptr;
  if (t.layout() != at::kStrided || code_of(t) < 0)
    return refuse(std::string(name) + " are float32, bfloat16 or float16, not " + c10::toString(t.scalar_type())), nullptr;
  if (dense && !t.is_non_overlapping_and_dense()) return refuse(std::string(name) + " are dense: no gaps, no overlap"), nullptr;
  return &t;
}

// rows(grads, out or None, device) -> (stq_grad rows as bytes, how many): without the gradients that are None.
PyObject* rows(PyObject*, PyObject* args) {
  PyObject *grads, *out;
  long dev;
  if (!PyArg_ParseTuple(args, "OOl", &grads, &out, &dev)) return nullptr;
  PyObject* g = PySequence_Fast(grads, "gradients are a sequence");
  if (!g) return nullptr;
  PyObject* o = out == Py_None ? nullptr : PySequence_Fast(out, "out is a sequence");
  if (out != Py_None && !o) {
    Py_DECREF(g);
    return nullptr;
  }
  PyObject* result = nullptr;
  try {
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(g);
    bool ok = !o || PySequence_Fast_GET_SIZE(o) == n || refuse("out has a tensor for each gradient");
    std::vector<stq_grad> r;
    r.reserve(n);
    for (Py_ssize_t i = 0; ok && i < n; ++i) {
      PyObject* item = PySequence_Fast_GET_ITEM(g, i);
      if (item == Py_None) continue;
      const at::Tensor* t = take(item, "gradients", dev, true);
      if (!(ok = t)) break;
      stq_grad row = {t->const_data_ptr(), nullptr, (uint64_t)t->numel(), code_of(*t), code_of(*t)};
      row.out = const_cast<void*>(row.grad);
      if (o) {
        const at::Tensor* u = take(PySequence_Fast_GET_ITEM(o, i), "results", dev, false);
        if (!(ok = u)) break;
        if (u->sizes() != t->sizes() || !(u->strides() == t->strides() || (u->is_contiguous() && t->is_contiguous()))) {
          ok = refuse("a result has the shape and layout of its gradient");
          break;
        }
        row.out = u->data_ptr();
        row.out_dtype = code_of(*u);
        if (row.out_dtype != row.dtype && row.out_dtype != STQ_GRAD_F32) {
          ok = refuse("a result has the type of its gradient or float32");
          break;
        }
      }
      r.push_back(row);
    }
    if (ok)
      result = Py_BuildValue("(y#n)", reinterpret_cast<const char*>(r.data()), (Py_ssize_t)(r.size() * sizeof(stq_grad)), (Py_ssize_t)r.size());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  Py_DECREF(g);
  Py_XDECREF(o);
  return result;
}

// written(tensors): they have been changed behind torch's back.
PyObject* written(PyObject*, PyObject* list) {
  PyObject* g = PySequence_Fast(list, "a sequence of tensors");
  if (!g) return nullptr;
  bool ok = true;
  try {
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(g); ++i) {
      PyObject* item = PySequence_Fast_GET_ITEM(g, i);
      if (!THPVariable_Check(item)) continue;
      const at::Tensor& t = THPVariable_Unpack(item);
      if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    ok = false;
  }
  Py_DECREF(g);
  if (!ok) return nullptr;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"rows", rows, METH_VARARGS, nullptr}, {"written", written, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "lists", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#define STQ_INIT_OF(name) PyInit_##name
#define STQ_INIT(name) STQ_INIT_OF(name)
PyMODINIT_FUNC STQ_INIT(STQ_LISTS)() { return PyModule_Create(&module); }
