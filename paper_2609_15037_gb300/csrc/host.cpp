// Python module _host: tensors as the C entries take them, where marshalling in Python
// costs more than the kernels.  read() takes lists (five attribute calls a tensor are
// 18 us of a step of 65 short tensors whose kernel takes 2.3); the fp4 calls take
// the matrices of one entry, allocate its output and call it by its address.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "moara.h"

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

// A matrix whose rows are contiguous.
struct Matrix {
    void* p;
    int dtype, rows, cols;
    int64_t ld;
};

// Null, or what is wrong with `o`.
const char* matrix_of(PyObject* o, long device, Matrix& m) {
    if (!THPVariable_Check(o)) return "a float32 or bfloat16 matrix is needed";
    const at::Tensor& t = THPVariable_Unpack(o);
    const at::ScalarType type = t.scalar_type();
    if (t.layout() != at::kStrided || t.dim() != 2 || !t.is_cuda() || t.get_device() != device ||
        (type != at::kFloat && type != at::kBFloat16))
        return "a float32 or bfloat16 matrix on the group's device is needed";
    if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) return "a matrix of at most 2^31 - 1 rows and columns is needed";
    if (t.size(1) > 1 && t.stride(1) != 1) return "the entries of a row must be contiguous";
    m = Matrix{const_cast<void*>(t.const_data_ptr()), type == at::kBFloat16, static_cast<int>(t.size(0)),
               static_cast<int>(t.size(1)), t.size(0) > 1 ? t.stride(0) : t.size(1) > 1 ? t.size(1) : 1};
    return nullptr;
}

at::Tensor allocate(int64_t rows, int64_t cols, at::ScalarType type, long device) {
    return at::empty({rows, cols}, at::TensorOptions().dtype(type).device(at::kCUDA, static_cast<at::DeviceIndex>(device)));
}

// The output of a call: `o`, or a new matrix for None.
const char* output_of(PyObject* o, int64_t rows, int64_t cols, int dtype, long device, PyObject*& held, Matrix& m) {
    if (o == Py_None) {
        at::Tensor t = allocate(rows, cols, dtype ? at::kBFloat16 : at::kFloat, device);
        held = THPVariable_Wrap(t);
        if (held == nullptr) return "";
    } else {
        Py_INCREF(o);
        held = o;
    }
    const char* wrong = matrix_of(held, device, m);
    if (wrong == nullptr && (m.rows != rows || m.cols != cols)) wrong = "out: a matrix of the product's shape is needed";
    return wrong;
}

template <class F> F entry(PyObject* o) { return reinterpret_cast<F>(PyLong_AsVoidPtr(o)); }

// The result of an entry: the tensor, or its error code.
PyObject* finish(PyObject* held, const char* wrong, int code) {
    if (wrong != nullptr || PyErr_Occurred()) {
        Py_XDECREF(held);
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, wrong);
        return nullptr;
    }
    if (code == MOARA_OK) return held;
    Py_XDECREF(held);
    return PyLong_FromLong(code);
}

bool arguments(Py_ssize_t have, Py_ssize_t want) {
    if (have != want) PyErr_Format(PyExc_TypeError, "%zd arguments are needed", want);
    return have == want;
}

// fp4_product(entry, ctx, m, n, k, a_q, a_sf, b_q, b_sf, out, bf16, device, stream)
PyObject* fp4_product(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 13)) return nullptr;
    const auto fn = entry<decltype(&moara_fp4_product)>(a[0]);
    const long m = PyLong_AsLong(a[2]), n = PyLong_AsLong(a[3]), k = PyLong_AsLong(a[4]), device = PyLong_AsLong(a[11]);
    PyObject* held = nullptr;
    Matrix d{};
    try {
        const char* wrong = output_of(a[9], m, n, PyObject_IsTrue(a[10]), device, held, d);
        const int code = wrong != nullptr || PyErr_Occurred() ? 0
            : fn(static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1])), m, n, k, PyLong_AsVoidPtr(a[5]), PyLong_AsVoidPtr(a[6]),
                 PyLong_AsVoidPtr(a[7]), PyLong_AsVoidPtr(a[8]), d.p, d.dtype, d.ld, PyLong_AsVoidPtr(a[12]));
        return finish(held, wrong, code);
    } catch (const std::exception& e) {
        Py_XDECREF(held);
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// fp4_linear(entry, ctx, x, n, k, b_q, b_sf, out, bf16, device, stream, workspace_entry)
PyObject* fp4_linear(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 12)) return nullptr;
    const auto fn = entry<decltype(&moara_fp4_linear)>(a[0]);
    const auto bytes = entry<decltype(&moara_fp4_linear_workspace_bytes)>(a[11]);
    const long n = PyLong_AsLong(a[3]), k = PyLong_AsLong(a[4]), device = PyLong_AsLong(a[9]);
    PyObject* held = nullptr;
    Matrix x{}, d{};
    try {
        const char* wrong = matrix_of(a[2], device, x);
        if (wrong == nullptr && x.cols != k) wrong = "x and the operand have different numbers of columns";
        if (wrong == nullptr) wrong = output_of(a[7], x.rows, n, PyObject_IsTrue(a[8]), device, held, d);
        int code = 0;
        if (wrong == nullptr && !PyErr_Occurred()) {
            size_t size = 0;
            at::Tensor ws;
            // a shape that has no workspace is refused by the entry itself
            if (bytes(x.rows, n, k, &size) == MOARA_OK && size > 0) ws = allocate(1, size, at::kByte, device);
            code = fn(static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1])), x.rows, n, k, x.p, x.dtype, x.ld,
                      PyLong_AsVoidPtr(a[5]), PyLong_AsVoidPtr(a[6]), d.p, d.dtype, d.ld,
                      size > 0 ? ws.data_ptr() : nullptr, size, PyLong_AsVoidPtr(a[10]));
        }
        return finish(held, wrong, code);
    } catch (const std::exception& e) {
        Py_XDECREF(held);
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// fp4_dequantize(entry, ctx, q, sf, rows, cols, out, bf16, device, stream)
PyObject* fp4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 10)) return nullptr;
    const auto fn = entry<decltype(&moara_fp4_dequantize)>(a[0]);
    const long rows = PyLong_AsLong(a[4]), cols = PyLong_AsLong(a[5]), device = PyLong_AsLong(a[8]);
    PyObject* held = nullptr;
    Matrix d{};
    try {
        const char* wrong = output_of(a[6], rows, cols, PyObject_IsTrue(a[7]), device, held, d);
        const int code = wrong != nullptr || PyErr_Occurred() ? 0
            : fn(static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1])), PyLong_AsVoidPtr(a[2]), PyLong_AsVoidPtr(a[3]), rows,
                 cols, d.p, d.dtype, d.ld, PyLong_AsVoidPtr(a[9]));
        return finish(held, wrong, code);
    } catch (const std::exception& e) {
        Py_XDECREF(held);
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// matrix(x, device) -> (address, type, rows, columns, row pitch)
PyObject* matrix(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 2)) return nullptr;
    Matrix m{};
    try {
        const char* wrong = matrix_of(a[0], PyLong_AsLong(a[1]), m);
        if (wrong != nullptr || PyErr_Occurred()) return finish(nullptr, wrong, 0);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return Py_BuildValue("(KiiiL)", reinterpret_cast<unsigned long long>(m.p), m.dtype, m.rows, m.cols,
                         static_cast<long long>(m.ld));
}

// bytes(count, device) -> (uint8 tensor, its address)
PyObject* bytes(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 2)) return nullptr;
    const long long size = PyLong_AsLongLong(a[0]);
    const long device = PyLong_AsLong(a[1]);
    if (PyErr_Occurred()) return nullptr;
    try {
        at::Tensor t = at::empty({size}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, static_cast<at::DeviceIndex>(device)));
        const unsigned long long at = reinterpret_cast<unsigned long long>(t.data_ptr());
        return Py_BuildValue("(NK)", THPVariable_Wrap(t), at);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define MOARA_METHOD(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, doc}

PyMethodDef methods[] = {
    MOARA_METHOD(read, "read(tensors, device, addresses, stride, types, stride, sizes, stride, given) -> first misfit, or -1"),
    MOARA_METHOD(fp4_product, "moara_fp4_product into a matrix or a new one -> the matrix, or an error code"),
    MOARA_METHOD(fp4_linear, "moara_fp4_linear into a matrix or a new one -> the matrix, or an error code"),
    MOARA_METHOD(fp4_dequantize, "moara_fp4_dequantize into a matrix or a new one -> the matrix, or an error code"),
    MOARA_METHOD(matrix, "matrix(x, device) -> (address, type, rows, columns, row pitch)"),
    MOARA_METHOD(bytes, "bytes(count, device) -> (uint8 tensor, its address)"),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "Tensors as the C entries take them.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
