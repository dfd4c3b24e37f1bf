// sizes(*tensors) -> bytes: what the checks of a call go by, each tensor's type, device, sizes and strides (a single byte for None).
//
// A key for the plans that the binding keeps.  Asked for one by one from Python, the four of eleven tensors took 5 us of a call whose kernel takes
// four; here they are copied out of the tensors in one go.  What torch throws on the way (a nested tensor has no sizes, a subclass may have its own
// in Python) becomes a Python exception: nothing may pass through the interpreter's C frames.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

namespace {

constexpr int kMostDims = 8, kMostTensors = 32;

PyObject* sizes(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    int64_t words[kMostTensors * (1 + 2 * kMostDims)];
    size_t at = 0;
    if (n > kMostTensors) {
        PyErr_SetString(PyExc_ValueError, "sizes: too many tensors");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (args[i] == Py_None) {
            words[at++] = -1;
            continue;
        }
        if (!THPVariable_Check(args[i])) {
            PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(args[i]);
        const int64_t dims = t.is_nested() ? kMostDims + 1 : t.dim();
        if (dims > kMostDims || t.layout() != at::kStrided) {
            PyErr_SetString(PyExc_TypeError, "a strided tensor of at most eight dimensions is wanted");
            return nullptr;
        }
        const c10::Device device = t.device();
        words[at++] = dims | (int64_t)t.scalar_type() << 8 | (int64_t)device.type() << 16 | (int64_t)(device.index() + 1) << 32;
        std::memcpy(words + at, t.sizes().data(), dims * sizeof(int64_t));
        std::memcpy(words + at + dims, t.strides().data(), dims * sizeof(int64_t));
        at += 2 * dims;
    }
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(words), (Py_ssize_t)(at * sizeof(int64_t)));
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"sizes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(sizes)), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_signature", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__signature() { return PyModule_Create(&module); }
