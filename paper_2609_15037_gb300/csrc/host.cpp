// Python module _host: tensors as the C entries take them, where marshalling in Python
// costs more than the kernels (five attribute calls a tensor are 18 us of a step of 65
// short tensors whose kernel takes 2.3).  Each call checks its tensors, allocates its
// output where none is given, and calls the entry, whose address it is given.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/StorageImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <optional>
#include <vector>

#include "moara.h"

namespace {

// A contiguous fp32 or bf16 tensor on cuda:`device`: its type (0 fp32, 1 bf16), or -1.
int flat_type(const at::Tensor& t, long device) {
    const at::ScalarType type = t.scalar_type();
    if (t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device || !t.is_contiguous()) return -1;
    return type == at::kFloat ? 0 : type == at::kBFloat16 ? 1 : -1;
}

// Tensors of a list or tuple, one at a time.  False with a Python error set for
// anything else.
struct Tensors {
    PyObject* list;
    Py_ssize_t n = 0;
    explicit Tensors(PyObject* o) : list(o) {
        if (!PyList_Check(o) && !PyTuple_Check(o)) PyErr_SetString(PyExc_TypeError, "a list or tuple of tensors is needed");
        else n = PySequence_Fast_GET_SIZE(o);
    }
    // tensor i, its address and type; or null, with an error set that names `what`
    const at::Tensor* get(Py_ssize_t i, const char* what, long device, int64_t entries, void*& at, int& type) const {
        PyObject* o = PySequence_Fast_GET_ITEM(list, i);
        if (THPVariable_Check(o)) {
            const at::Tensor& t = THPVariable_Unpack(o);
            type = flat_type(t, device);
            if (type >= 0 && (entries < 0 || t.numel() == entries)) {
                at = const_cast<void*>(t.const_data_ptr());
                return &t;
            }
        }
        if (entries < 0)
            PyErr_Format(PyExc_ValueError, "%s %zd: a contiguous float32 or bfloat16 tensor on cuda:%ld is needed", what, i, device);
        else
            PyErr_Format(PyExc_ValueError, "%s %zd: a contiguous float32 or bfloat16 tensor of %lld entries on cuda:%ld is needed",
                         what, i, static_cast<long long>(entries), device);
        return nullptr;
    }
};

bool arguments(Py_ssize_t have, Py_ssize_t want) {
    if (have != want) PyErr_Format(PyExc_TypeError, "%zd arguments are needed", want);
    return have == want;
}

template <class F> F entry(PyObject* o) { return reinterpret_cast<F>(PyLong_AsVoidPtr(o)); }

// A float32 scalar on the device, or null for None; an error is set for anything else.
float* scalar_of(PyObject* o, const char* what, long device) {
    if (o == Py_None) return nullptr;
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (flat_type(t, device) == 0 && t.numel() == 1) return const_cast<float*>(t.const_data_ptr<float>());
    }
    PyErr_Format(PyExc_ValueError, "%s: a one-element float32 tensor on cuda:%ld is needed", what, device);
    return nullptr;
}

PyObject* caught(const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// Whether `o` is still what a descriptor was made from: None for no address, or a
// contiguous tensor of this type and size at it.  A tensor keeps its identity while its
// storage is replaced (an assignment to .data, module.to).
bool in_place(PyObject* o, const void* at, at::ScalarType type, int64_t entries) {
    if (o == Py_None) return at == nullptr;         // asking torch about None takes 60 ns
    if (!THPVariable_Check(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.const_data_ptr() == at && t.scalar_type() == type && t.numel() == entries && t.is_contiguous();
}

// Where the storages of a tensor's moments had their memory: adamw.py holds the
// storages, whose memory can be freed or taken anew in place (resize_).
struct Places {
    const c10::StorageImpl* storage[4];
    const void* data[4];
    bool hold() const {
        for (int i = 0; i < 4; ++i)
            if (storage[i] != nullptr && storage[i]->data() != data[i]) return false;
        return true;
    }
};

// own(moments, places): tensors of their own on the memory of up to four tensors (or None), whose
// storages nobody else can replace; writes where they have their memory to the address `places`.
PyObject* own(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 2)) return nullptr;
    PyObject* held = nullptr;
    try {
        auto* places = static_cast<Places*>(PyLong_AsVoidPtr(a[1]));
        if (PyErr_Occurred()) return nullptr;
        if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) > 4) return PyErr_Format(PyExc_TypeError, "a tuple of four is needed");
        const Py_ssize_t n = PyTuple_GET_SIZE(a[0]);
        held = PyTuple_New(n);
        *places = Places{};
        for (Py_ssize_t i = 0; held != nullptr && i < n; ++i) {
            PyObject* o = PyTuple_GET_ITEM(a[0], i);
            if (THPVariable_Check(o)) {
                at::Tensor t = THPVariable_Unpack(o).detach();
                places->storage[i] = t.storage().unsafeGetStorageImpl();
                places->data[i] = places->storage[i]->data();
                o = THPVariable_Wrap(std::move(t));
            } else {
                Py_INCREF(o);
            }
            PyTuple_SET_ITEM(held, i, o);
        }
        if (PyErr_Occurred()) Py_CLEAR(held);
        return held;
    } catch (const std::exception& e) {
        Py_XDECREF(held);
        return caught(e);
    }
}

// adamw_step(entry, ctx, count, descriptors, gradients, hparams, t, lr, grad_scale, device, stream,
// places, params, copies) -> error code, or None if a parameter, a copy (or None) or a moment is not
// where its descriptor says.  The gradients' addresses and types go into the descriptors.
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 14)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_adamw_step)>(a[0]);
        const Py_ssize_t n = PyLong_AsSsize_t(a[2]);
        auto* d = static_cast<moara_adamw_tensor*>(PyLong_AsVoidPtr(a[3]));
        const Tensors grads(a[4]);
        const long device = PyLong_AsLong(a[9]);
        float* scale = scalar_of(a[8], "grad_scale", device);
        if (PyErr_Occurred()) return nullptr;
        if (grads.n != n) return PyErr_Format(PyExc_ValueError, "%zd gradients for %zd tensors", grads.n, n);
        const auto* places = static_cast<const Places*>(PyLong_AsVoidPtr(a[11]));
        if (!PyList_Check(a[12]) || PyList_GET_SIZE(a[12]) != n || !PyList_Check(a[13]) || PyList_GET_SIZE(a[13]) != n)
            return PyErr_Format(PyExc_TypeError, "lists of %zd parameters and copies are needed", n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            if (!in_place(PyList_GET_ITEM(a[12], i), d[i].param, d[i].param_dtype == MOARA_DTYPE_BF16 ? at::kBFloat16 : at::kFloat,
                          d[i].n) ||
                !in_place(PyList_GET_ITEM(a[13], i), d[i].param_bf16, at::kBFloat16, d[i].n) || !places[i].hold())
                Py_RETURN_NONE;
            void* at;
            if (grads.get(i, "gradient", device, d[i].n, at, d[i].grad_dtype) == nullptr) return nullptr;
            d[i].grad = at;
        }
        const int64_t t = PyLong_AsLongLong(a[6]);
        const double lr = PyFloat_AsDouble(a[7]);
        auto* hp = static_cast<moara_adamw_hparams*>(PyLong_AsVoidPtr(a[5]));
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        void* stream = PyLong_AsVoidPtr(a[10]);
        if (PyErr_Occurred()) return nullptr;
        return PyLong_FromLong(fn(ctx, static_cast<int>(n), d, hp, t, static_cast<float>(lr), scale, stream));
    } catch (const std::exception& e) {
        return caught(e);
    }
}

// adamw_moments(entry, ctx, count, descriptors, exp_avg, exp_avg_sq, device, stream, places)
// -> error code, or None as adamw_step
PyObject* adamw_moments(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 9)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_adamw_moments)>(a[0]);
        const Py_ssize_t n = PyLong_AsSsize_t(a[2]);
        auto* d = static_cast<moara_adamw_tensor*>(PyLong_AsVoidPtr(a[3]));
        const Tensors outs[2] = {Tensors(a[4]), Tensors(a[5])};
        const long device = PyLong_AsLong(a[6]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        void* stream = PyLong_AsVoidPtr(a[7]);
        if (PyErr_Occurred()) return nullptr;
        const auto* places = static_cast<const Places*>(PyLong_AsVoidPtr(a[8]));
        if (PyErr_Occurred()) return nullptr;
        for (Py_ssize_t i = 0; i < n; ++i)
            if (!places[i].hold()) Py_RETURN_NONE;
        std::vector<float*> to[2];
        for (int k = 0; k < 2; ++k) {
            if (outs[k].n != n) return PyErr_Format(PyExc_ValueError, "%zd outputs for %zd tensors", outs[k].n, n);
            to[k].resize(n);
            for (Py_ssize_t i = 0; i < n; ++i) {
                void* at;
                int type;
                if (outs[k].get(i, "output", device, d[i].n, at, type) == nullptr) return nullptr;
                if (type != 0) return PyErr_Format(PyExc_ValueError, "output %zd: the moments are float32", i);
                to[k][i] = static_cast<float*>(at);
            }
        }
        return PyLong_FromLong(fn(ctx, static_cast<int>(n), d, to[0].data(), to[1].data(), stream));
    } catch (const std::exception& e) {
        return caught(e);
    }
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

// grad_norm(entry, ctx, gradients, max_norm, extra_sq, out, workspace, bytes, device, stream)
// -> the three floats (a new tensor for out = None), or an error code
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 10)) return nullptr;
    PyObject* held = nullptr;
    try {
        const auto fn = entry<decltype(&moara_grad_norm)>(a[0]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const Tensors grads(a[2]);
        const double max_norm = PyFloat_AsDouble(a[3]);
        const long device = PyLong_AsLong(a[8]);
        float* extra = scalar_of(a[4], "extra_sq", device);
        void* ws = PyLong_AsVoidPtr(a[6]);
        const size_t size = PyLong_AsSize_t(a[7]);
        void* stream = PyLong_AsVoidPtr(a[9]);
        if (PyErr_Occurred()) return nullptr;
        const Py_ssize_t n = grads.n;
        std::vector<const void*> p(n);
        std::vector<int64_t> sizes(n);
        std::vector<int> types(n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            void* at;
            const at::Tensor* t = grads.get(i, "gradient", device, -1, at, types[i]);
            if (t == nullptr) return nullptr;
            p[i] = at;
            sizes[i] = t->numel();
        }
        at::Tensor out;
        if (a[5] == Py_None) {
            out = at::empty({3}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, static_cast<at::DeviceIndex>(device)));
            held = THPVariable_Wrap(out);
        } else {
            if (!THPVariable_Check(a[5]) || flat_type(THPVariable_Unpack(a[5]), device) != 0 || THPVariable_Unpack(a[5]).numel() != 3)
                return PyErr_Format(PyExc_ValueError, "out: a contiguous float32 tensor of three on cuda:%ld is needed", device);
            held = a[5];
            Py_INCREF(held);
            out = THPVariable_Unpack(held);
        }
        return finish(held, nullptr, fn(ctx, static_cast<int>(n), p.data(), sizes.data(), types.data(), static_cast<float>(max_norm),
                                        extra, out.data_ptr<float>(), ws, size, stream));
    } catch (const std::exception& e) {
        Py_XDECREF(held);
        return caught(e);
    }
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
        return caught(e);
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
        return caught(e);
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
        return caught(e);
    }
}

// A buffer for an operand, the codes and from the next 256 bytes on the scales.
struct Operand {
    at::Tensor both;
    char* q;
    char* sf;
    Operand(int64_t rows, int64_t cols, long device) {
        size_t nq = rows * ((cols + 31) / 32) * 16, ns = ((rows + 127) / 128) * ((cols + 127) / 128) * 512;
        const size_t start = (nq + 255) / 256 * 256;
        both = at::empty({static_cast<int64_t>(start + ns)},
                         at::TensorOptions().dtype(at::kByte).device(at::kCUDA, static_cast<at::DeviceIndex>(device)));
        q = static_cast<char*>(both.data_ptr());
        sf = q + start;
    }
    // (buffer, address of the codes, address of the scales)
    PyObject* tuple() const {
        return Py_BuildValue("(NKK)", THPVariable_Wrap(both), reinterpret_cast<unsigned long long>(q),
                             reinterpret_cast<unsigned long long>(sf));
    }
};

// fp4_quantize(entry, ctx, x, rows, cols, device, stream): quantises into new buffers, by
// rows and by columns as asked -> ((buffer, q, sf) or None, the same, rows, columns), or
// an error code.  Zero rows or columns are refused by the entry itself.
PyObject* fp4_quantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 7)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_fp4_quantize)>(a[0]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const int rows = PyObject_IsTrue(a[3]), cols = PyObject_IsTrue(a[4]);
        const long device = PyLong_AsLong(a[5]);
        void* stream = PyLong_AsVoidPtr(a[6]);
        Matrix x{};
        const char* wrong = matrix_of(a[2], device, x);
        if (wrong != nullptr || PyErr_Occurred()) return finish(nullptr, wrong, 0);
        std::optional<Operand> r, c;
        if (rows) r.emplace(x.rows, x.cols, device);
        if (cols) c.emplace(x.cols, x.rows, device);
        const int code = fn(ctx, x.p, x.dtype, x.rows, x.cols, x.ld, rows ? r->q : nullptr, rows ? r->sf : nullptr,
                            cols ? c->q : nullptr, cols ? c->sf : nullptr, stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        PyObject* none = Py_None;
        return Py_BuildValue("(NNii)", rows ? r->tuple() : Py_NewRef(none), cols ? c->tuple() : Py_NewRef(none), x.rows, x.cols);
    } catch (const std::exception& e) {
        return caught(e);
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
        return caught(e);
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
        return caught(e);
    }
}

#define MOARA_METHOD(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, doc}

PyMethodDef methods[] = {
    MOARA_METHOD(own, "own(moments, places) -> tensors of their own on the same memory"),
    MOARA_METHOD(adamw_step, "moara_adamw_step with a list of gradients -> error code"),
    MOARA_METHOD(adamw_moments, "moara_adamw_moments into two lists of tensors -> error code"),
    MOARA_METHOD(grad_norm, "moara_grad_norm of a list of gradients -> tensor of three, or an error code"),
    MOARA_METHOD(fp4_quantize, "moara_fp4_quantize into new operands -> their buffers, or an error code"),
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
