// Python module _host: reads lists of tensors into the arrays that the C entries
// take.  In Python this is five attribute calls a tensor, 18 us of a step of 65 short
// tensors whose kernel takes 2.3.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

namespace {

// Address of the entry for tensor i of an array (or of a field of an array of
// structs), or null for no array.
struct Field {
    char* base;
    Py_ssize_t stride;
    template <class T> T* at(Py_ssize_t i) const { return reinterpret_cast<T*>(base + i * stride); }
};

// read(tensors, device, addresses, stride, types, stride, sizes, stride, given)
//
// For each tensor of the list or tuple: its address as uint64, its type as int32 (0
// fp32, 1 bf16) and its number of entries as int64, into arrays given by the
// address of their first entry and their stride in bytes.  With `given`, the
// sizes are compared instead.  Returns the position of the first entry that is no
// contiguous fp32 or bf16 tensor on cuda:`device` (or has another size), or -1.
PyObject* read(PyObject*, PyObject* const* args, Py_ssize_t count) {
    if (count != 9) {
        PyErr_SetString(PyExc_TypeError, "read takes nine arguments");
        return nullptr;
    }
    PyObject* list = args[0];
    if (!PyList_Check(list) && !PyTuple_Check(list)) {
        PyErr_SetString(PyExc_TypeError, "a list or tuple of tensors is needed");
        return nullptr;
    }
    const long device = PyLong_AsLong(args[1]);
    Field f[3];
    for (int k = 0; k < 3; ++k) {
        f[k].base = static_cast<char*>(PyLong_AsVoidPtr(args[2 + 2 * k]));
        f[k].stride = PyLong_AsSsize_t(args[3 + 2 * k]);
    }
    const int given = PyObject_IsTrue(args[8]);
    if (given < 0 || PyErr_Occurred()) return nullptr;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
    try {
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject* o = PySequence_Fast_GET_ITEM(list, i);
            if (!THPVariable_Check(o)) return PyLong_FromSsize_t(i);
            const at::Tensor& t = THPVariable_Unpack(o);
            const at::ScalarType type = t.scalar_type();
            if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device || !t.is_contiguous() ||
                (type != at::kFloat && type != at::kBFloat16))
                return PyLong_FromSsize_t(i);
            if (given && *f[2].at<int64_t>(i) != t.numel()) return PyLong_FromSsize_t(i);
            *f[0].at<uint64_t>(i) = reinterpret_cast<uint64_t>(t.const_data_ptr());
            *f[1].at<int32_t>(i) = type == at::kBFloat16;
            if (!given) *f[2].at<int64_t>(i) = t.numel();
        }
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(-1);
}

PyMethodDef methods[] = {
    {"read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(read)), METH_FASTCALL,
     "read(tensors, device, addresses, stride, types, stride, sizes, stride, given) -> first misfit, or -1"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "Lists of tensors as the C entries take them.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
