// The tensors of a call for attention.py and training.py.  pack reads the inputs: what a call's
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
#include <vector>

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

// matrices(tensor, bytes, type, rows, columns, type, rows, columns) -> (matrix or
// None, matrix or None, workspace or None, addresses): contiguous matrices of
// float32 (type 0) or bfloat16 (1; -1: none) on the tensor's device, vectors where
// rows == -1, a single value without dimensions where rows == -2, and a workspace
// of so many bytes.
PyObject *matrices(PyObject *, PyObject *const *args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != 8 || !THPVariable_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "matrices takes a tensor, a number of bytes and two matrices' types and sizes");
        return nullptr;
    }
    long long number[8];
    for (int i = 1; i < 8; ++i)
        number[i] = PyLong_AsLongLong(args[i]);
    if (PyErr_Occurred())
        return nullptr;
    const at::TensorOptions options = THPVariable_Unpack(args[0]).options();
    at::Tensor made[3];
    {
        pybind11::gil_scoped_release others;
        for (int i = 0; i < 2; ++i) {
            const long long *want = number + 2 + 3 * i;
            if (want[0] < 0)
                continue;
            const at::TensorOptions typed = options.dtype(want[0] == 0 ? at::kFloat : at::kBFloat16);
            made[i] = want[1] >= 0 ? at::empty({(int64_t)want[1], (int64_t)want[2]}, typed)
                      : want[1] == -1 ? at::empty({(int64_t)want[2]}, typed)
                                      : at::empty({}, typed);
        }
        if (number[1] > 0)
            made[2] = at::empty({(int64_t)number[1]}, options.dtype(at::kByte));
    }
    int64_t address[3];
    std::unique_ptr<PyObject, void (*)(PyObject *)> results(PyTuple_New(4), Py_DecRef);
    if (!results)
        return nullptr;
    for (int i = 0; i < 3; ++i) {
        address[i] = made[i].defined() ? (int64_t)made[i].data_ptr() : 0;
        PyObject *item = THPVariable_Wrap(made[i]);
        if (item == nullptr)
            return nullptr;
        PyTuple_SET_ITEM(results.get(), i, item);
    }
    PyObject *addresses = PyBytes_FromStringAndSize((const char *)address, (Py_ssize_t)sizeof address);
    if (addresses == nullptr)
        return nullptr;
    PyTuple_SET_ITEM(results.get(), 3, addresses);
    return results.release();
    END_HANDLE_TH_ERRORS
}

// step(params, grads, avgs, sqs, avg_scales, sq_scales, copies) -> (count, the
// array of pam_step_tensor_t, whether the gradients are bfloat16, whether the
// states are bytes, the first gradient or None), or None where the lists are not
// what the call takes: the caller's checks then say why.  Each is a list or tuple
// of tensors or, but for the gradients, None.  What the call writes counts as
// changed in place.
PyObject *step(PyObject *, PyObject *const *args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    constexpr int kLists = 7, kGrads = 1;
    constexpr int64_t kBlock = 256;
    if (count != kLists)
        Py_RETURN_NONE;
    PyObject *const *items[kLists] = {};
    Py_ssize_t n = -1;
    for (int l = 0; l < kLists; ++l) {
        if (args[l] == Py_None)
            continue;
        if (!PyList_Check(args[l]) && !PyTuple_Check(args[l]))
            Py_RETURN_NONE;
        const Py_ssize_t have = PySequence_Fast_GET_SIZE(args[l]);
        if (n >= 0 && have != n)
            Py_RETURN_NONE;
        n = have;
        items[l] = PySequence_Fast_ITEMS(args[l]);
    }
    const bool whole = args[0] != Py_None;   // a step, not the norm alone
    if (args[kGrads] == Py_None || (whole && (args[2] == Py_None || args[3] == Py_None)) ||
        (args[4] == Py_None) != (args[5] == Py_None))
        Py_RETURN_NONE;
    const bool scales = args[4] != Py_None;
    const at::ScalarType held = scales ? at::kByte : at::kFloat;
    at::ScalarType grad = at::kFloat;
    c10::Device device(c10::kCPU);
    std::vector<int64_t> array((size_t)n * 8);
    for (Py_ssize_t j = 0; j < n; ++j) {
        int64_t *one = array.data() + j * 8;
        if (!THPVariable_Check(items[kGrads][j]))
            Py_RETURN_NONE;
        const at::Tensor &g = THPVariable_Unpack(items[kGrads][j]);
        if (j == 0) {
            grad = g.scalar_type();
            device = g.device();
            if ((grad != at::kFloat && grad != at::kBFloat16) || !device.is_cuda())
                Py_RETURN_NONE;
        }
        const int64_t values = g.numel();
        const at::ScalarType types[kLists] = {at::kFloat, grad, held, held, at::kFloat, at::kFloat, at::kBFloat16};
        for (int l = 0; l < kLists; ++l) {
            if (args[l] == Py_None)
                continue;
            if (!THPVariable_Check(items[l][j]))
                Py_RETURN_NONE;
            const at::Tensor &t = THPVariable_Unpack(items[l][j]);
            const bool scale = l == 4 || l == 5;
            if (t.layout() != at::kStrided || t.scalar_type() != types[l] || t.device() != device ||
                !t.is_contiguous() || t.numel() != (scale ? (values + kBlock - 1) / kBlock : values))
                Py_RETURN_NONE;
            one[l] = (int64_t)t.data_ptr();
        }
        one[7] = values;
    }
    for (int l = 0; l < kLists; ++l)
        for (Py_ssize_t j = 0; j < n && l != kGrads && args[l] != Py_None; ++j) {
            const at::Tensor &t = THPVariable_Unpack(items[l][j]);
            if (!t.is_inference())
                t.unsafeGetTensorImpl()->bump_version();
        }
    return Py_BuildValue("(ny#iiO)", n, (const char *)array.data(), (Py_ssize_t)(array.size() * sizeof(int64_t)),
                         (int)(grad == at::kBFloat16), (int)scales, n > 0 ? items[kGrads][0] : Py_None);
    END_HANDLE_TH_ERRORS
}

// call(function, argument, ..., stream) -> status of the library's C function at
// that address, on integers and the bytes of structures; other threads run
// meanwhile.  (Through ctypes a call takes 0.7 us more.)
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t count) {
    constexpr Py_ssize_t kMost = 7;
    if (count < 2 || count > 1 + kMost) {
        PyErr_SetString(PyExc_TypeError, "call takes a function and one to seven arguments");
        return nullptr;
    }
    // Integers and pointers alike go in the C convention's integer registers, and
    // then on the stack.
    int64_t a[kMost] = {};
    for (Py_ssize_t i = 0; i + 1 < count; ++i)
        a[i] = PyBytes_Check(args[i + 1]) ? (int64_t)PyBytes_AS_STRING(args[i + 1]) : PyLong_AsLongLong(args[i + 1]);
    void *const function = PyLong_AsVoidPtr(args[0]);
    if (PyErr_Occurred())
        return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = ((int (*)(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t))function)(a[0], a[1], a[2], a[3], a[4],
                                                                                       a[5], a[6]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

PyMethodDef methods[] = {{"make", (PyCFunction)(void *)make, METH_FASTCALL,
                          "make(type, bytes, tensor or None, ...) -> (result, ..., workspace, addresses)"},
                         {"call", (PyCFunction)(void *)call, METH_FASTCALL, "call(function, argument, ..., stream) -> status"},
                         {"matrices", (PyCFunction)(void *)matrices, METH_FASTCALL,
                          "matrices(tensor, bytes, type, rows, columns, type, rows, columns)"},
                         {"step", (PyCFunction)(void *)step, METH_FASTCALL,
                          "step(params, grads, avgs, sqs, avg_scales, sq_scales, copies)"},
                         {"pack", (PyCFunction)(void *)pack, METH_FASTCALL, "pack(tensor or None, ...) -> (key, addresses)"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pack", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pack(void) { return PyModule_Create(&module); }
