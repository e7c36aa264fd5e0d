// Python module `_tensors`: the addresses of a call's tensors, once they are what its description says.  The checks are those of binding.py, which says what is
// wrong where one fails; ten tensors take 7 us there, 0.5 here, of a call whose launch takes 3.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// Whether the tuple holds these numbers.
bool same(PyObject *tuple, at::IntArrayRef x) {
    if (PyTuple_GET_SIZE(tuple) != (Py_ssize_t)x.size()) return false;
    for (size_t i = 0; i < x.size(); ++i)
        if (PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i)) != x[i]) return false;
    return true;
}

// As described: (name, element type, number of elements or None, shape, strides).
bool fits(PyObject *what, const at::Tensor &t, long device) {
    PyObject *dtype = PyTuple_GET_ITEM(what, 1), *n = PyTuple_GET_ITEM(what, 2), *shape = PyTuple_GET_ITEM(what, 3), *stride = PyTuple_GET_ITEM(what, 4);
    if (!THPDtype_Check(dtype) || t.scalar_type() != ((THPDtype *)dtype)->scalar_type || t.get_device() != device) return false;
    if (shape == Py_None) return t.numel() == PyLong_AsLongLong(n) && t.is_contiguous();
    return PyTuple_Check(shape) && PyTuple_Check(stride) && same(shape, t.sizes()) && same(stride, t.strides());
}

// pointers(described, given, device): a list of addresses and None's, or None if a tensor is not as described.
PyObject *pointers(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    if (n_args != 3 || !PyTuple_Check(args[0]) || !PyTuple_Check(args[1]) || !PyLong_Check(args[2])) Py_RETURN_NONE;
    const Py_ssize_t n = PyTuple_GET_SIZE(args[0]);
    if (PyTuple_GET_SIZE(args[1]) != n) Py_RETURN_NONE;
    const long device = PyLong_AsLong(args[2]);
    PyObject *out = PyList_New(n);
    if (!out) return nullptr;
    bool ok = true;
    try {
        for (Py_ssize_t i = 0; i < n && ok; ++i) {
            PyObject *what = PyTuple_GET_ITEM(args[0], i), *given = PyTuple_GET_ITEM(args[1], i), *at = Py_None;
            if (given == Py_None) {
                Py_INCREF(at);
            } else {
                ok = PyTuple_Check(what) && PyTuple_GET_SIZE(what) == 5 && THPVariable_Check(given) && fits(what, THPVariable_Unpack(given), device);
                if (!ok) break;
                at = PyLong_FromVoidPtr(THPVariable_Unpack(given).data_ptr());
                if (!at) ok = false;
            }
            if (at) PyList_SET_ITEM(out, i, at);
        }
    } catch (...) {  // (a tensor without strides or storage, for one)
        ok = false;
    }
    if (ok && !PyErr_Occurred()) return out;
    PyErr_Clear();
    Py_DECREF(out);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"pointers", (PyCFunction)(void (*)(void))pointers, METH_FASTCALL, "Addresses of tensors that are as described, else None."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
