// Arguments of the Python binding: the tensors of a call looked over and turned into addresses, in one call.
//
// A property of a tensor that Python asks for takes 0.04 us, so device, type, layout and address of a plan's 13 arrays are 2.2 us.  The plan of a small
// batch, which the GPU is done with in 4.6, takes 4.8 a call with all of them read here; with device and address read from Python it took 6.1.
//
// addresses(device, kinds, names, *arguments): an address for each argument, which may be a tensor, an address or None.  kinds has a letter for each:
//   i, f   int32 / float32, contiguous (the call has no stride for it)
//   h, s   float16 / float32 in rows: the call states the row stride, the columns lie side by side
//   b, r   of any type, contiguous / in rows
#include <torch/csrc/autograd/python_variable.h>

namespace {

bool type_fits(char kind, c10::ScalarType t) {
    switch (kind) {
        case 'i': return t == c10::ScalarType::Int;
        case 'f': case 's': return t == c10::ScalarType::Float;
        case 'h': return t == c10::ScalarType::Half;
        default: return true;
    }
}
const char* type_name(char kind) { return kind == 'i' ? "torch.int32" : kind == 'h' ? "torch.float16" : "torch.float32"; }

// an exception, with what the tensor's attribute says
PyObject* refuse(PyObject* error, PyObject* name, const char* must, PyObject* tensor, const char* attribute) {
    PyObject* is = PyObject_GetAttrString(tensor, attribute);
    if (is) PyErr_Format(error, "%U must be %s, got %S", name, must, is);
    Py_XDECREF(is);
    return nullptr;
}

PyObject* address_of(PyObject* arg, char kind, PyObject* name, long device) {
    if (arg == Py_None || PyLong_Check(arg)) {
        Py_INCREF(arg);
        return arg;
    }
    if (!THPVariable_Check(arg)) {
        PyErr_Format(PyExc_TypeError, "%U must be a tensor, an address or None, got %s", name, Py_TYPE(arg)->tp_name);
        return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(arg);
    if (!type_fits(kind, t.scalar_type())) return refuse(PyExc_TypeError, name, type_name(kind), arg, "dtype");
    if (kind == 'i' || kind == 'f' || kind == 'b') {
        if (!t.is_contiguous()) return PyErr_Format(PyExc_ValueError, "%U must be contiguous", name);
    } else if (t.dim() > 0 && t.size(-1) > 1 && t.stride(-1) != 1) {
        return PyErr_Format(PyExc_ValueError, "the columns of %U must lie side by side", name);
    }
    if (!t.device().is_cuda() || t.device().index() != device) {
        char must[64];
        snprintf(must, sizeof must, "on the current device cuda:%ld", device);
        return refuse(PyExc_ValueError, name, must, arg, "device");
    }
    return PyLong_FromVoidPtr(t.data_ptr());
}

PyObject* addresses(PyObject*, PyObject* const* args, Py_ssize_t n) {
    const char* kinds = n >= 3 && PyUnicode_Check(args[1]) ? PyUnicode_AsUTF8(args[1]) : nullptr;
    const long device = n >= 3 ? PyLong_AsLong(args[0]) : -1;
    if (PyErr_Occurred()) return nullptr;
    if (!kinds || !PyTuple_Check(args[2]) || (Py_ssize_t)strlen(kinds) != n - 3 || PyTuple_GET_SIZE(args[2]) != n - 3) {
        PyErr_SetString(PyExc_TypeError, "addresses(device, kinds, names, *arguments): a kind and a name for each argument");
        return nullptr;
    }
    PyObject* out = PyList_New(n - 3);
    for (Py_ssize_t i = 0; out && i < n - 3; ++i) {
        PyObject* a = nullptr;
        try {
            a = address_of(args[3 + i], kinds[i], PyTuple_GET_ITEM(args[2], i), device);
        } catch (const std::exception& e) {                 // a tensor without strides or memory of its own
            PyErr_SetString(PyExc_RuntimeError, e.what());
        }
        if (a) PyList_SET_ITEM(out, i, a);
        else Py_CLEAR(out);
    }
    return out;
}

PyMethodDef methods[] = {{"addresses", (PyCFunction)(void*)addresses, METH_FASTCALL, "addresses(device, kinds, names, *arguments) -> list"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_args() { return PyModule_Create(&module); }
