// Addresses of tensors for the ctypes binding (_lib.py): the checks of one argument in C++ (a tenth of a microsecond
// against the same checks as Python attribute reads, 0.4, of a launch's 3). An extension module of one
// function; the binding has the same checks in Python and uses those where this is not built.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

namespace {

PyObject* g_slow = nullptr;  // the binding's own check: says what is wrong with a tensor

// addr(fn, name, tensor | int | None, kind, n): the address of a dense GPU tensor of n elements of `kind`
// (0 fp32, 1 bf16, 2 int32, 3 int8); an int or None as it is.
PyObject* addr(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 5) {
        PyErr_SetString(PyExc_TypeError, "addr takes fn, name, tensor, kind, n");
        return nullptr;
    }
    PyObject* t = args[2];
    if (t == Py_None || PyLong_CheckExact(t)) {
        Py_INCREF(t);
        return t;
    }
    if (THPVariable_Check(t)) {
        static const at::ScalarType kinds[4] = {at::kFloat, at::kBFloat16, at::kInt, at::kChar};
        const long kind = PyLong_AsLong(args[3]);
        const long long n = PyLong_AsLongLong(args[4]);
        if ((kind == -1 || n == -1) && PyErr_Occurred()) return nullptr;
        const void* p = nullptr;
        try {
            const at::Tensor& v = THPVariable_Unpack(t);
            if (kind >= 0 && kind < 4 && v.layout() == at::kStrided && v.is_cuda() && v.scalar_type() == kinds[kind] && v.numel() == n &&
        v.is_contiguous()) {
                p = v.data_ptr();
                if (!p) return PyLong_FromLong(0);
            }
        } catch (const std::exception&) {  // (a tensor without storage, say: the slow check says so)
        }
        if (p) return PyLong_FromVoidPtr(const_cast<void*>(p));
    }
    if (!g_slow) {
        PyErr_SetString(PyExc_TypeError, "not a dense GPU tensor of the call's type and size");
        return nullptr;
    }
    return PyObject_Vectorcall(g_slow, args, (size_t)nargs, nullptr);
}

PyObject* set_slow(PyObject*, PyObject* f) {
    Py_INCREF(f);
    Py_XSETREF(g_slow, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"addr", (PyCFunction)(void (*)(void))addr, METH_FASTCALL, "address of a tensor argument"},
    {"set_slow", set_slow, METH_O, "the check to call where a tensor does not fit"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module);
    if (m) PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION);  // whose objects this reads
    return m;
}
