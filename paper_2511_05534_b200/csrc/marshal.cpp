// Argument marshalling of the paged caches' calls and of rotary positions for Python: looks at the tensors of a call (shapes, types, devices, strides) and
// passes their addresses on.  The same in Python took longer than the kernels of a decode step: ten tensors' attributes 4 us.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>
#include <string>
#include <vector>

#include "flowmm.h"

namespace {

union Params {
    flowmm_cache_params cache;
    flowmm_rotary_params rotary;
    char bytes[1];
};

struct Argument {
    std::string name;
    std::vector<int64_t> shape;              // -1: any size
    std::vector<c10::ScalarType> types;
    int dense;                               // where in the params the strides of a tensor of rows are, in bytes; else 0: contiguous
    bool optional;                           // may be None
    bool no_middle;                          // the middle one of three sizes, 1, may be left out
};
// One entry point with one set of params: what its tensors have to look like, in the order of its pointers; should it have a workspace, that is the last one.
struct Call {
    std::string what;
    void *function;
    Params params;
    bool workspace;
    std::vector<Argument> arguments;
};

constexpr const char *kCapsule = "flowmm_call";
constexpr size_t kFewestPointers = 6, kMostPointers = 9;

void drop(PyObject *capsule) { delete static_cast<Call *>(PyCapsule_GetPointer(capsule, kCapsule)); }

// make(what, function's address, params' address and size, workspace, ((name, shape, types, dense, optional[, no_middle]), ...)) -> the call's handle
PyObject *make(PyObject *, PyObject *args) {
    const char *what;
    unsigned long long function, params;
    Py_ssize_t size;
    int workspace;
    PyObject *list;
    if (!PyArg_ParseTuple(args, "sKKnpO!", &what, &function, &params, &size, &workspace, &PyTuple_Type, &list)) return nullptr;
    if (size < 0 || (size_t)size > sizeof(Params)) { PyErr_SetString(PyExc_ValueError, "unknown params"); return nullptr; }
    try {
        Call *call = new Call{what, reinterpret_cast<void *>(function), {}, workspace != 0, {}};
        std::memcpy(call->params.bytes, reinterpret_cast<const void *>(params), (size_t)size);
        PyObject *capsule = PyCapsule_New(call, kCapsule, drop);
        if (!capsule) { delete call; return nullptr; }
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(list); ++i) {
            const char *name;
            PyObject *shape, *types;
            int dense, optional, no_middle = 0;
            if (!PyArg_ParseTuple(PyTuple_GET_ITEM(list, i), "sO!O!ip|p", &name, &PyTuple_Type, &shape, &PyTuple_Type, &types, &dense, &optional, &no_middle)) {
                Py_DECREF(capsule);
                return nullptr;
            }
            Argument a{name, {}, {}, dense, optional != 0, no_middle != 0};
            for (Py_ssize_t j = 0; j < PyTuple_GET_SIZE(shape); ++j) a.shape.push_back(PyLong_AsLongLong(PyTuple_GET_ITEM(shape, j)));
            for (Py_ssize_t j = 0; j < PyTuple_GET_SIZE(types); ++j) {
                PyObject *type = PyTuple_GET_ITEM(types, j);
                if (!THPDtype_Check(type)) PyErr_SetString(PyExc_TypeError, "types must be torch dtypes");
                else a.types.push_back(reinterpret_cast<THPDtype *>(type)->scalar_type);
            }
            if (!PyErr_Occurred() && no_middle && a.shape.size() != 3) PyErr_SetString(PyExc_ValueError, "no_middle wants three sizes");
            if (PyErr_Occurred()) { Py_DECREF(capsule); return nullptr; }
            call->arguments.push_back(std::move(a));
        }
        return capsule;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *refuse(const Call &call, const Argument &a, const std::string &why) {
    PyErr_SetString(PyExc_ValueError, (call.what + ": " + a.name + " " + why).c_str());
    return nullptr;
}

// run(handle, tensor, ...) -> the entry point's status
PyObject *run(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n < 1) { PyErr_SetString(PyExc_TypeError, "run(handle, tensors...)"); return nullptr; }
    const Call *call = static_cast<const Call *>(PyCapsule_GetPointer(args[0], kCapsule));
    if (!call) return nullptr;
    const size_t count = call->arguments.size();
    if ((size_t)(n - 1) != count || count < kFewestPointers || count > kMostPointers) { PyErr_SetString(PyExc_TypeError, "wrong number of tensors"); return nullptr; }
    try {
        Params params = call->params;
        void *at[kMostPointers] = {};
        int64_t ws_bytes = 0;
        c10::DeviceIndex device = -1;
        for (size_t i = 0; i < count; ++i) {
            const Argument &a = call->arguments[i];
            if (args[i + 1] == Py_None && a.optional) continue;
            if (!THPVariable_Check(args[i + 1])) return refuse(*call, a, "must be a tensor");
            const at::Tensor &t = THPVariable_Unpack(args[i + 1]);
            if (!t.is_cuda()) return refuse(*call, a, "must be a CUDA tensor");
            if (device < 0) device = c10::cuda::current_device();
            if (t.device().index() != device) return refuse(*call, a, "is not on the current device");
            const auto sizes = t.sizes(), strides = t.strides();
            bool same = sizes.size() == a.shape.size();
            for (size_t d = 0; same && d < sizes.size(); ++d) same = a.shape[d] < 0 || sizes[d] == a.shape[d];
            if (!same && a.no_middle && sizes.size() == 2) same = sizes[0] == a.shape[0] && sizes[1] == a.shape[2];
            bool type = false;
            for (c10::ScalarType s : a.types) type = type || t.scalar_type() == s;
            if (!same || !type) {
                std::string want = "must be a ";
                for (size_t d = 0; d < a.types.size(); ++d) want += (d ? " or " : "") + std::string(c10::toString(a.types[d]));
                want += " tensor of shape [";
                for (size_t d = 0; d < a.shape.size(); ++d) want += (d ? ", " : "") + (a.shape[d] < 0 ? std::string("any") : std::to_string(a.shape[d]));
                return refuse(*call, a, want + "]");
            }
            if (a.dense) {
                if (strides[3] != 1) return refuse(*call, a, "must have contiguous head_dim");
                int64_t three[3] = {strides[0], strides[1], strides[2]};
                std::memcpy(params.bytes + a.dense, three, sizeof(three));
            } else if (!t.is_contiguous()) {
                return refuse(*call, a, "must be contiguous");
            }
            at[i] = t.data_ptr();
            if (call->workspace && i == count - 1) ws_bytes = t.numel();
        }
        void *stream = c10::cuda::getCurrentCUDAStream(device).stream();
        typedef flowmm_status (*Six)(const void *, void *, void *, void *, void *, void *, void *, void *);
        typedef flowmm_status (*Seven)(const void *, void *, void *, void *, void *, void *, void *, void *, void *, size_t, void *);
        typedef flowmm_status (*Eight)(const void *, void *, void *, void *, void *, void *, void *, void *, void *, void *, size_t, void *);
        int status = -1;
        Py_BEGIN_ALLOW_THREADS
        if (count == 6 && !call->workspace)
            status = reinterpret_cast<Six>(call->function)(&params, at[0], at[1], at[2], at[3], at[4], at[5], stream);
        else if (count == 8 && call->workspace)
            status = reinterpret_cast<Seven>(call->function)(&params, at[0], at[1], at[2], at[3], at[4], at[5], at[6], at[7], (size_t)ws_bytes, stream);
        else if (count == 9 && call->workspace)
            status = reinterpret_cast<Eight>(call->function)(&params, at[0], at[1], at[2], at[3], at[4], at[5], at[6], at[7], at[8], (size_t)ws_bytes, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {{"make", make, METH_VARARGS, nullptr},
                         {"run", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(run)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
