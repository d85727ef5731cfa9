// Python module _host: tensors as the C entries take them, where marshalling in Python
// costs more than the kernels (five attribute calls a tensor are 18 us of a step of 65
// short tensors whose kernel takes 2.3).  Each call checks its tensors, allocates its
// output where none is given, and calls the entry, whose address it is given.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
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

// ------------------------------------------------------- operators of a decoder's layers
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, long device, bool zero = false) {
    const auto o = at::TensorOptions().dtype(type).device(at::kCUDA, static_cast<at::DeviceIndex>(device));
    return zero ? at::zeros(shape, o) : at::empty(shape, o);
}

// The entries of a contiguous tensor of this type and size (null for None where it may be),
// or an error that names `what`.
const void* entries_of(PyObject* o, const char* what, at::ScalarType type, int64_t n, long device, bool optional = false) {
    if (optional && o == Py_None) return nullptr;
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.layout() == at::kStrided && t.is_cuda() && t.get_device() == device && t.is_contiguous() && t.scalar_type() == type &&
            t.numel() == n)
            return t.const_data_ptr();
    }
    PyErr_Format(PyExc_ValueError, "%s: a contiguous %s tensor of %lld entries on cuda:%ld is needed", what,
                 type == at::kLong ? "int64" : type == at::kFloat ? "float32" : "bfloat16", static_cast<long long>(n), device);
    return nullptr;
}

// Errors of a matrix argument by its name.
bool matrix_arg(PyObject* o, const char* what, long device, Matrix& m) {
    const char* wrong = matrix_of(o, device, m);
    if (wrong != nullptr && !PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: %s", what, wrong);
    return !PyErr_Occurred();
}

bool like_arg(PyObject* o, const char* what, long device, const Matrix& like, Matrix& m) {
    if (!matrix_arg(o, what, device, m)) return false;
    if (m.rows != like.rows || m.cols != like.cols || (like.dtype >= 0 && m.dtype != like.dtype))
        PyErr_Format(PyExc_ValueError, "%s: a %s matrix of %d x %d is needed", what,
                     like.dtype < 0 ? "float32 or bfloat16" : like.dtype ? "bfloat16" : "float32", like.rows, like.cols);
    return !PyErr_Occurred();
}

// `o`, or a new matrix for None; of like's type, or of the given one's own for -1.
PyObject* output_arg(PyObject* o, const char* what, long device, const Matrix& like, int dtype, Matrix& m) {
    if (o == Py_None) {
        const at::Tensor t = fresh({like.rows, like.cols}, dtype ? at::kBFloat16 : at::kFloat, device);
        m = Matrix{t.data_ptr(), dtype, like.rows, like.cols, like.cols > 0 ? like.cols : 1};
        return THPVariable_Wrap(t);
    }
    if (!like_arg(o, what, device, like, m)) return nullptr;
    return Py_NewRef(o);
}

// References that are given up unless they are handed on.
struct Held {
    PyObject* at[5] = {};
    ~Held() {
        for (PyObject* o : at) Py_XDECREF(o);
    }
    PyObject* take(int i) {
        PyObject* o = at[i];
        at[i] = nullptr;
        return o;
    }
};

struct NormArgs {
    Matrix x{}, r{}, h{};
    const float* gain = nullptr;
    float* rstd = nullptr;
    float eps = 0;
    long device = 0;
    bool res = false;
};

// x, gain, residual (or None), eps and h (or None) of a norm's call; held.at[0]: h, held.at[1]: rstd
bool norm_args(PyObject* x, PyObject* gain, PyObject* res, PyObject* eps, PyObject* h, NormArgs& n, Held& held) {
    n.eps = static_cast<float>(PyFloat_AsDouble(eps));
    if (PyErr_Occurred() || !matrix_arg(x, "x", n.device, n.x)) return false;
    n.res = res != Py_None;
    if (n.res && !like_arg(res, "residual", n.device, n.x, n.r)) return false;
    n.gain = static_cast<const float*>(entries_of(gain, "gain", at::kFloat, n.x.cols, n.device));
    if (PyErr_Occurred()) return false;
    if (n.res) {
        held.at[0] = output_arg(h, "h", n.device, n.x, n.x.dtype, n.h);
    } else if (h != Py_None) {
        PyErr_SetString(PyExc_ValueError, "h: without a residual h is x");
    } else {
        held.at[0] = Py_NewRef(x);
    }
    if (PyErr_Occurred()) return false;
    const at::Tensor rstd = fresh({n.x.rows}, at::kFloat, n.device);
    n.rstd = rstd.data_ptr<float>();
    held.at[1] = THPVariable_Wrap(rstd);
    return held.at[1] != nullptr;
}

// rms_norm(entry, ctx, x, gain, residual, eps, bf16, h, y, device, stream) -> (h, y, rstd) or an error code
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 11)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_rms_norm)>(a[0]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const int bf16 = PyObject_IsTrue(a[6]);
        NormArgs n;
        Held held;
        n.device = PyLong_AsLong(a[9]);
        void* stream = PyLong_AsVoidPtr(a[10]);
        if (PyErr_Occurred() || !norm_args(a[2], a[3], a[4], a[5], a[7], n, held)) return nullptr;
        Matrix y{}, any = n.x;
        any.dtype = -1;
        held.at[2] = output_arg(a[8], "out", n.device, any, bf16, y);
        if (held.at[2] == nullptr) return nullptr;
        const int code = fn(ctx, n.x.rows, n.x.cols, n.x.p, n.x.ld, n.r.p, n.r.ld, n.x.dtype, n.gain, n.eps, n.h.p, n.h.ld, y.p,
                            y.dtype, y.ld, n.rstd, stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        PyObject *h = held.take(0), *rstd = held.take(1);
        return Py_BuildValue("(NNN)", h, held.take(2), rstd);
    } catch (const std::exception& e) {
        return caught(e);
    }
}

// rms_norm_quantize(entry, ctx, x, gain, residual, eps, rows, cols, h, device, stream)
// -> (h, (buffer, q, sf) or None, the same, rstd, rows, columns), or an error code
PyObject* rms_norm_quantize(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 11)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_rms_norm_quantize)>(a[0]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const int rows = PyObject_IsTrue(a[6]), cols = PyObject_IsTrue(a[7]);
        NormArgs n;
        Held held;
        n.device = PyLong_AsLong(a[9]);
        void* stream = PyLong_AsVoidPtr(a[10]);
        if (PyErr_Occurred() || !norm_args(a[2], a[3], a[4], a[5], a[8], n, held)) return nullptr;
        std::optional<Operand> r, c;
        if (rows) r.emplace(n.x.rows, n.x.cols, n.device);
        if (cols) c.emplace(n.x.cols, n.x.rows, n.device);
        const int code = fn(ctx, n.x.rows, n.x.cols, n.x.p, n.x.ld, n.r.p, n.r.ld, n.x.dtype, n.gain, n.eps, n.h.p, n.h.ld,
                            rows ? r->q : nullptr, rows ? r->sf : nullptr, cols ? c->q : nullptr, cols ? c->sf : nullptr, n.rstd,
                            stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        PyObject *h = held.take(0), *rstd = held.take(1);
        return Py_BuildValue("(NNNNii)", h, rows ? r->tuple() : Py_NewRef(Py_None), cols ? c->tuple() : Py_NewRef(Py_None), rstd,
                             n.x.rows, n.x.cols);
    } catch (const std::exception& e) {
        return caught(e);
    }
}

// rms_norm_backward(entry, ctx, dy, h, gain, rstd, dh, dx, device, stream, workspace_entry) -> (dx, dgain) or an error code
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 11)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_rms_norm_backward)>(a[0]);
        const auto bytes = entry<decltype(&moara_rms_norm_backward_workspace_bytes)>(a[10]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const long device = PyLong_AsLong(a[8]);
        void* stream = PyLong_AsVoidPtr(a[9]);
        Matrix dy{}, h{}, dh{}, dx{};
        Held held;
        if (PyErr_Occurred() || !matrix_arg(a[3], "h", device, h)) return nullptr;
        Matrix any = h;
        any.dtype = -1;
        if (!like_arg(a[2], "dy", device, any, dy)) return nullptr;
        if (a[6] != Py_None && !like_arg(a[6], "dh", device, h, dh)) return nullptr;
        const auto* gain = static_cast<const float*>(entries_of(a[4], "gain", at::kFloat, h.cols, device));
        if (PyErr_Occurred()) return nullptr;
        const auto* rstd = static_cast<const float*>(entries_of(a[5], "rstd", at::kFloat, h.rows, device));
        if (PyErr_Occurred()) return nullptr;
        held.at[0] = output_arg(a[7], "out", device, h, h.dtype, dx);
        if (held.at[0] == nullptr) return nullptr;
        const at::Tensor dgain = fresh({h.cols}, at::kFloat, device);
        held.at[1] = THPVariable_Wrap(dgain);
        size_t size = 0;
        at::Tensor ws;
        // a shape that has no workspace is refused by the entry itself
        if (bytes(h.rows, h.cols, &size) == MOARA_OK && size > 0) ws = fresh({static_cast<int64_t>(size)}, at::kByte, device);
        const int code = fn(ctx, h.rows, h.cols, dy.p, dy.dtype, dy.ld, h.p, h.dtype, h.ld, gain, rstd, dh.p, dh.ld, dx.p, dx.ld,
                            dgain.data_ptr<float>(), size > 0 ? ws.data_ptr() : nullptr, size, stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        PyObject* first = held.take(0);
        return Py_BuildValue("(NN)", first, held.take(1));
    } catch (const std::exception& e) {
        return caught(e);
    }
}

// policy_loss(entry, ctx, logits, targets, old, adv, weights, ref, low, high, kl, grad, out, device, stream,
// workspace_entry) -> (sums, logp, gradient or None) or an error code
PyObject* policy_loss(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 16)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_policy_loss)>(a[0]);
        const auto bytes = entry<decltype(&moara_policy_loss_workspace_bytes)>(a[15]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const long device = PyLong_AsLong(a[13]);
        void* stream = PyLong_AsVoidPtr(a[14]);
        const double low = PyFloat_AsDouble(a[8]), high = PyFloat_AsDouble(a[9]), kl = PyFloat_AsDouble(a[10]);
        const int grad = PyObject_IsTrue(a[11]);
        Matrix z{}, dz{};
        Held held;
        if (PyErr_Occurred() || !matrix_arg(a[2], "logits", device, z)) return nullptr;
        const auto* target = static_cast<const int64_t*>(entries_of(a[3], "targets", at::kLong, z.rows, device));
        if (PyErr_Occurred()) return nullptr;
        const char* const names[4] = {"old", "adv", "weights", "ref"};
        const float* v[4];
        for (int i = 0; i < 4; ++i) {
            v[i] = static_cast<const float*>(entries_of(a[4 + i], names[i], at::kFloat, z.rows, device, i >= 2));
            if (PyErr_Occurred()) return nullptr;
        }
        if (grad) {
            held.at[2] = output_arg(a[12], "out", device, z, z.dtype, dz);
        } else if (a[12] != Py_None) {
            PyErr_SetString(PyExc_ValueError, "out: no gradient is asked for");
        } else {
            held.at[2] = Py_NewRef(Py_None);
        }
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor sums = fresh({3}, at::kFloat, device), logp = fresh({z.rows}, at::kFloat, device);
        held.at[0] = THPVariable_Wrap(sums);
        held.at[1] = THPVariable_Wrap(logp);
        size_t size = 0;
        at::Tensor ws;
        if (bytes(z.rows, &size) == MOARA_OK) ws = fresh({static_cast<int64_t>(size)}, at::kByte, device);
        const int code = fn(ctx, z.rows, z.cols, z.p, z.dtype, z.ld, target, v[0], v[3], v[1], v[2], static_cast<float>(low),
                            static_cast<float>(high), static_cast<float>(kl), sums.data_ptr<float>(), logp.data_ptr<float>(), dz.p,
                            dz.ld, size > 0 ? ws.data_ptr() : nullptr, size, stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        PyObject *s = held.take(0), *l = held.take(1);
        return Py_BuildValue("(NNN)", s, l, held.take(2));
    } catch (const std::exception& e) {
        return caught(e);
    }
}

// A bf16 tensor of tokens x heads x entries whose entries are contiguous.
struct Heads {
    void* p;
    int tokens, heads, dim;
    int64_t row, head;
};

bool heads_arg(PyObject* o, const char* what, long device, Heads& h) {
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.layout() == at::kStrided && t.dim() == 3 && t.is_cuda() && t.get_device() == device && t.scalar_type() == at::kBFloat16 &&
            t.size(0) <= INT32_MAX && t.size(1) <= INT32_MAX && t.size(2) <= INT32_MAX && (t.size(2) == 1 || t.stride(2) == 1)) {
            h = Heads{const_cast<void*>(t.const_data_ptr()), static_cast<int>(t.size(0)), static_cast<int>(t.size(1)),
                      static_cast<int>(t.size(2)), t.stride(0), t.stride(1)};
            return true;
        }
    }
    PyErr_Format(PyExc_ValueError, "%s: a bfloat16 tensor of tokens x heads x contiguous entries on cuda:%ld is needed", what, device);
    return false;
}

bool attention_args(PyObject* const* a, long device, Heads& q, Heads& k, Heads& v) {
    if (!heads_arg(a[0], "q", device, q) || !heads_arg(a[1], "k", device, k) || !heads_arg(a[2], "v", device, v)) return false;
    if (k.tokens != q.tokens || v.tokens != q.tokens || k.dim != q.dim || v.dim != q.dim || k.heads != v.heads) {
        PyErr_SetString(PyExc_ValueError, "q, k and v need the same tokens and entries, k and v the same heads");
        return false;
    }
    return true;
}

// attention(entry, ctx, sequences, q, k, v, scale, train, device, stream) -> (out, lse, rest or None) or an error code
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 10)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_attention)>(a[0]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const auto* seqs = static_cast<const moara_sequences*>(PyLong_AsVoidPtr(a[2]));
        const double scale = PyFloat_AsDouble(a[6]);
        const int train = PyObject_IsTrue(a[7]);
        const long device = PyLong_AsLong(a[8]);
        void* stream = PyLong_AsVoidPtr(a[9]);
        Heads q, k, v;
        if (PyErr_Occurred() || !attention_args(a + 3, device, q, k, v)) return nullptr;
        // rows that belong to no sequence are not written
        const bool zero = q.tokens > seqs->tokens;
        const at::Tensor out = fresh({q.tokens, q.heads, q.dim}, at::kBFloat16, device, zero);
        const at::Tensor lse = fresh({q.heads, q.tokens}, at::kFloat, device, zero);
        at::Tensor rest;
        if (train) rest = fresh({q.tokens, q.heads, q.dim}, at::kBFloat16, device, zero);
        const int code = fn(ctx, seqs, q.tokens, q.heads, k.heads, q.dim, static_cast<float>(scale), q.p, q.row, q.head, k.p, k.row,
                            k.head, v.p, v.row, v.head, out.data_ptr(), train ? rest.data_ptr() : nullptr, lse.data_ptr<float>(), stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        return Py_BuildValue("(NNN)", THPVariable_Wrap(out), THPVariable_Wrap(lse), train ? THPVariable_Wrap(rest) : Py_NewRef(Py_None));
    } catch (const std::exception& e) {
        return caught(e);
    }
}

// attention_backward(entry, ctx, sequences, dout, q, k, v, out, lse, rest, scale, device, stream)
// -> (dq, dk, dv) or an error code
PyObject* attention_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
    if (!arguments(count, 13)) return nullptr;
    try {
        const auto fn = entry<decltype(&moara_attention_backward)>(a[0]);
        auto* ctx = static_cast<moara_ctx*>(PyLong_AsVoidPtr(a[1]));
        const auto* seqs = static_cast<const moara_sequences*>(PyLong_AsVoidPtr(a[2]));
        const double scale = PyFloat_AsDouble(a[10]);
        const long device = PyLong_AsLong(a[11]);
        void* stream = PyLong_AsVoidPtr(a[12]);
        Heads q, k, v, d;
        if (PyErr_Occurred() || !heads_arg(a[3], "dout", device, d) || !attention_args(a + 4, device, q, k, v)) return nullptr;
        if (d.tokens != q.tokens || d.heads != q.heads || d.dim != q.dim)
            return PyErr_Format(PyExc_ValueError, "dout needs q's shape");
        const int64_t rows = static_cast<int64_t>(q.tokens) * q.heads, entries = rows * q.dim;
        const void* out = entries_of(a[7], "out", at::kBFloat16, entries, device);
        if (PyErr_Occurred()) return nullptr;
        const void* lse = entries_of(a[8], "lse", at::kFloat, rows, device);
        if (PyErr_Occurred()) return nullptr;
        const void* rest = entries_of(a[9], "rest", at::kBFloat16, entries, device, true);
        if (PyErr_Occurred()) return nullptr;
        const bool zero = q.tokens > seqs->tokens;
        const at::Tensor dq = fresh({q.tokens, q.heads, q.dim}, at::kBFloat16, device, zero);
        const at::Tensor dk = fresh({q.tokens, k.heads, q.dim}, at::kBFloat16, device, zero);
        const at::Tensor dv = fresh({q.tokens, k.heads, q.dim}, at::kBFloat16, device, zero);
        const at::Tensor delta = fresh({rows + 1}, at::kFloat, device);
        const int code = fn(ctx, seqs, q.tokens, q.heads, k.heads, q.dim, static_cast<float>(scale), d.p, d.row, d.head, q.p, q.row,
                            q.head, k.p, k.row, k.head, v.p, v.row, v.head, out, rest, static_cast<const float*>(lse),
                            delta.data_ptr<float>(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), stream);
        if (code != MOARA_OK) return PyLong_FromLong(code);
        return Py_BuildValue("(NNN)", THPVariable_Wrap(dq), THPVariable_Wrap(dk), THPVariable_Wrap(dv));
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
    MOARA_METHOD(rms_norm, "moara_rms_norm -> (h, y, rstd), or an error code"),
    MOARA_METHOD(rms_norm_quantize, "moara_rms_norm_quantize into new operands -> their buffers, or an error code"),
    MOARA_METHOD(rms_norm_backward, "moara_rms_norm_backward -> (dx, dgain), or an error code"),
    MOARA_METHOD(policy_loss, "moara_policy_loss -> (sums, logp, gradient), or an error code"),
    MOARA_METHOD(attention, "moara_attention -> (out, lse, rest), or an error code"),
    MOARA_METHOD(attention_backward, "moara_attention_backward -> (dq, dk, dv), or an error code"),
    MOARA_METHOD(matrix, "matrix(x, device) -> (address, type, rows, columns, row pitch)"),
    MOARA_METHOD(bytes, "bytes(count, device) -> (uint8 tensor, its address)"),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "Tensors as the C entries take them.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
