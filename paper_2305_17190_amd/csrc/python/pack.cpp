// Reads the tensors of a call for attention.py: what a call's argument checks
// depend on, as one hashable key, and the addresses, as the bytes its argument
// structure begins with.  (In Python, type, shape, strides, device and address of
// append_kv's eleven tensors took 5 of its 10 us of host time.)

#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

constexpr int kMostTensors = 16;
constexpr int kMostDims = 8;
constexpr int kPerTensor = 1 + 2 * kMostDims;

// pack(tensor or None, ...) -> (key, addresses), or None where an argument is
// something else: the caller's checks then say what.
PyObject *pack(PyObject *, PyObject *const *args, Py_ssize_t count) {
    int64_t key[kMostTensors * kPerTensor], address[kMostTensors];
    Py_ssize_t used = 0;
    if (count > kMostTensors)
        Py_RETURN_NONE;
    for (Py_ssize_t i = 0; i < count; ++i) {
        address[i] = 0;
        if (args[i] == Py_None) {
            key[used++] = -1;
            continue;
        }
        if (!THPVariable_Check(args[i]))
            Py_RETURN_NONE;
        try {
            const at::Tensor &t = THPVariable_Unpack(args[i]);
            const int64_t dims = t.dim();
            if (t.layout() != at::kStrided || dims > kMostDims)
                Py_RETURN_NONE;
            const c10::Device device = t.device();
            key[used++] = (int64_t)t.scalar_type() | (int64_t)device.type() << 8 | (int64_t)(uint8_t)device.index() << 16 |
                          dims << 24;
            for (int64_t d = 0; d < dims; ++d) {
                key[used++] = t.size(d);
                key[used++] = t.stride(d);
            }
            address[i] = (int64_t)t.data_ptr();
        } catch (...) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
    }
    return Py_BuildValue("(y#y#)", (const char *)key, (Py_ssize_t)(used * sizeof(int64_t)), (const char *)address,
                         (Py_ssize_t)(count * sizeof(int64_t)));
}

PyMethodDef methods[] = {{"pack", (PyCFunction)(void *)pack, METH_FASTCALL, "pack(tensor or None, ...) -> (key, addresses)"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pack", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pack(void) { return PyModule_Create(&module); }
