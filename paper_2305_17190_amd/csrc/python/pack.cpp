// The tensors of a call for attention.py.  pack reads the inputs: what a call's
// argument checks depend on, as one hashable key, and the addresses, as the bytes
// its argument structure begins with.  (In Python, type, shape, strides, device
// and address of append_kv's eleven tensors took 5 of its 10 us of host time.)
// make allocates the results and the workspace, and like torch.empty lets other
// threads run meanwhile: an allocation may wait for the device.  (torch.empty takes
// 1.5 us a tensor; the gradient of norm and rotation makes five.)

#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <pybind11/pybind11.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <memory>

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

// make(type, bytes, tensor or None, ...) -> (result or None, ..., workspace or
// None, addresses): a contiguous tensor like each given one, of float32 (type 0),
// bfloat16 (1) or its own type (-1), and where bytes > 0 a workspace of as many
// on the device of the first tensor given; the addresses of all.
PyObject *make(PyObject *, PyObject *const *args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count < 3 || count > kMostTensors) {
        PyErr_SetString(PyExc_TypeError, "make takes a type, a number of bytes and tensors");
        return nullptr;
    }
    const long type = PyLong_AsLong(args[0]);
    const long long bytes = PyLong_AsLongLong(args[1]);
    if (PyErr_Occurred())
        return nullptr;
    // Of the tensors, then the workspace; the results end with the addresses.
    const Py_ssize_t last = count - 2;
    at::Tensor like[kMostTensors], made[kMostTensors];
    const at::Tensor *first = nullptr;
    for (Py_ssize_t i = 0; i < last; ++i) {
        if (args[i + 2] == Py_None)
            continue;
        if (!THPVariable_Check(args[i + 2])) {
            PyErr_SetString(PyExc_TypeError, "make takes tensors");
            return nullptr;
        }
        like[i] = THPVariable_Unpack(args[i + 2]);
        if (first == nullptr)
            first = &like[i];
    }
    {
        pybind11::gil_scoped_release others;
        for (Py_ssize_t i = 0; i < last; ++i)
            if (like[i].defined())
                made[i] = at::empty(like[i].sizes(), like[i].options().dtype(type < 0    ? like[i].scalar_type()
                                                                             : type == 0 ? at::kFloat
                                                                                         : at::kBFloat16));
        if (bytes > 0 && first != nullptr)
            made[last] = at::empty({(int64_t)bytes}, first->options().dtype(at::kByte));
    }
    int64_t address[kMostTensors];
    std::unique_ptr<PyObject, void (*)(PyObject *)> results(PyTuple_New(count), Py_DecRef);
    if (!results)
        return nullptr;
    for (Py_ssize_t i = 0; i <= last; ++i) {
        address[i] = made[i].defined() ? (int64_t)made[i].data_ptr() : 0;
        PyObject *item = THPVariable_Wrap(made[i]);   // None where none was made
        if (item == nullptr)
            return nullptr;
        PyTuple_SET_ITEM(results.get(), i, item);
    }
    PyObject *addresses = PyBytes_FromStringAndSize((const char *)address, (Py_ssize_t)((last + 1) * sizeof(int64_t)));
    if (addresses == nullptr)
        return nullptr;
    PyTuple_SET_ITEM(results.get(), count - 1, addresses);
    return results.release();
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"make", (PyCFunction)(void *)make, METH_FASTCALL,
                          "make(type, bytes, tensor or None, ...) -> (result, ..., workspace, addresses)"},
                         {"pack", (PyCFunction)(void *)pack, METH_FASTCALL, "pack(tensor or None, ...) -> (key, addresses)"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pack", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pack(void) { return PyModule_Create(&module); }
