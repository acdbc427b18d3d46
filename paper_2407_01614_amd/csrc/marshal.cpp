// The Python binding's tensor checks and pointers, natively: one call takes
// all tensors of an entry point.  In Python each tensor's type, device, dtype,
// layout, size and address cost about a microsecond, so that a receive of 64
// sources spent longer on its 128 small tensors than the GPU on the pass.
//
// A check that fails, or a tensor this file does not know to treat (a
// subclass, a wrapper without storage), is answered with None: the binding
// then runs its own checks, which raise the error or accept the tensor.
//
// The layer operators, whose smallest calls are a few microseconds on the GPU,
// are called from here as well, their arguments read and checked on the way.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include "zpp.h"

#include <vector>

namespace {

// dtypes an argument may have, as bits of a mask (kOptional: None may stand
// in the tensor's place)
enum : unsigned { kF32 = 1, kBF16 = 2, kI16 = 4, kU16 = 8, kI8 = 16, kU8 = 32, kOptional = 64 };

unsigned dtype_bit(at::ScalarType t) {
    switch (t) {
    case at::kFloat: return kF32;
    case at::kBFloat16: return kBF16;
    case at::kShort: return kI16;
    case at::kUInt16: return kU16;
    case at::kChar: return kI8;
    case at::kByte: return kU8;
    default: return 0;
    }
}

// The address of a contiguous tensor of device `device` with one of the
// dtypes of `mask` and at least `need` elements.
bool address(PyObject *o, long device, unsigned mask, long long need, void **out) {
    if (!THPVariable_CheckExact(o))
        return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.device().index() != device || !(dtype_bit(t.scalar_type()) & mask) ||
        !t.is_contiguous() || t.numel() < need)
        return false;
    *out = t.data_ptr();
    return true;
}

// addresses(device, tensor, mask, need, tensor, mask, need, ...): a tuple of
// addresses (None for an optional tensor that is not given), or None.
PyObject *addresses(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n < 1 || (n - 1) % 3) {
        PyErr_SetString(PyExc_TypeError, "addresses(device, (tensor, mask, need)...)");
        return nullptr;
    }
    const long device = PyLong_AsLong(args[0]);
    const Py_ssize_t count = (n - 1) / 3;
    PyObject *result = PyTuple_New(count);
    if (!result)
        return nullptr;
    try {
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject *const *a = args + 1 + 3 * i;
            PyObject *value = Py_None;
            const unsigned mask = (unsigned)PyLong_AsUnsignedLong(a[1]);
            if (a[0] != Py_None || !(mask & kOptional)) {
                void *p = nullptr;
                const long long need = PyLong_AsLongLong(a[2]);
                if (PyErr_Occurred() || !address(a[0], device, mask, need, &p)) {
                    Py_DECREF(result);
                    PyErr_Clear();
                    Py_RETURN_NONE;
                }
                value = PyLong_FromVoidPtr(p);
                if (!value) {
                    Py_DECREF(result);
                    return nullptr;
                }
            } else {
                Py_INCREF(value);
            }
            PyTuple_SET_ITEM(result, i, value);
        }
    } catch (const std::exception &) {
        Py_DECREF(result);
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return result;
}

// address_array(device, tensors, mask, need): the addresses of a list or tuple
// of tensors as the bytes of a C array of pointers, or None.
PyObject *address_array(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "address_array(device, tensors, mask, need)");
        return nullptr;
    }
    if (!PyList_CheckExact(args[1]) && !PyTuple_CheckExact(args[1]))
        Py_RETURN_NONE;
    const long device = PyLong_AsLong(args[0]);
    const unsigned mask = (unsigned)PyLong_AsUnsignedLong(args[2]);
    const long long need = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(args[1]);
    PyObject *const *items = PySequence_Fast_ITEMS(args[1]);
    try {
        std::vector<void *> p((size_t)count);
        for (Py_ssize_t i = 0; i < count; ++i)
            if (!address(items[i], device, mask, need, &p[(size_t)i]))
                Py_RETURN_NONE;
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(p.data()),
                                         count * (Py_ssize_t)sizeof(void *));
    } catch (const std::exception &) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// Element type of a matrix (zpp_type), or -1.
int matrix_type(at::ScalarType t) {
    switch (t) {
    case at::kBFloat16:
    case at::kShort:
    case at::kUInt16: return ZPP_BF16;
    case at::kFloat: return ZPP_F32;
    case at::kChar: return ZPP_I8;
    default: return -1;
    }
}

// The arguments of one layer operator's call, read one after the other: the
// entry point's address, the device, the stream and the two events (integers or
// None), then the tensors.  `good` ends false where one is not what the call
// takes: the binding's own checks then say why.
class Call {
  public:
    Call(PyObject *const *args, Py_ssize_t n) : args_(args), end_(args + n) {
        fn = pointer();
        device_ = take() ? PyLong_AsLong(args_[-1]) : -1;
        stream = reinterpret_cast<hipStream_t>(pointer());
        wait = reinterpret_cast<hipEvent_t>(pointer());
        done = reinterpret_cast<hipEvent_t>(pointer());
    }

    // The shape of the tensor, or of the checkpoint's codes, that comes next.
    bool shape(size_t *rows, size_t *cols) const {
        if (!good || args_ >= end_)
            return false;
        PyObject *o = *args_;
        if (PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2)
            o = PyTuple_GET_ITEM(o, 0);
        if (!THPVariable_CheckExact(o) || THPVariable_Unpack(o).dim() != 2)
            return false;
        *rows = (size_t)THPVariable_Unpack(o).size(0);
        *cols = (size_t)THPVariable_Unpack(o).size(1);
        return true;
    }

    // A [rows, cols] matrix with one of the types of the mask (1 << zpp_type);
    // nullptr where None may stand and does.
    const zpp_matrix *matrix(zpp_matrix *m, unsigned types, bool needed, size_t rows, size_t cols) {
        if (!take())
            return nullptr;
        PyObject *o = args_[-1];
        if (o == Py_None && !needed)
            return nullptr;
        void *exps = nullptr;
        const bool pair = PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2;
        if (pair) {
            good = address(PyTuple_GET_ITEM(o, 1), device_, kU8,
                           (long long)(rows * ((cols + 63) / 64)), &exps);
            o = PyTuple_GET_ITEM(o, 0);
        }
        if (!good || !THPVariable_CheckExact(o))
            return fail();
        const at::Tensor &t = THPVariable_Unpack(o);
        const int type = matrix_type(t.scalar_type());
        if (!t.is_cuda() || t.device().index() != device_ || t.dim() != 2 ||
            (size_t)t.size(0) != rows || (size_t)t.size(1) != cols ||
            (cols > 1 && t.stride(1) != 1) || type < 0 || !((types >> type) & 1u) ||
            pair != (type == ZPP_I8))
            return fail();
        *m = {t.data_ptr(), reinterpret_cast<uint8_t *>(exps), (size_t)t.stride(0), type};
        return m;
    }

    // `count` contiguous values with one of the dtypes of the mask.
    template <class T = void>
    T *vector(unsigned mask, bool needed, size_t count) {
        if (!take() || (args_[-1] == Py_None && !needed))
            return nullptr;
        void *p = nullptr;
        good = address(args_[-1], device_, mask, (long long)count, &p);
        return reinterpret_cast<T *>(p);
    }

    // Layer norm's weight and, unless None, bias: the same type both.
    int params(const void **gamma, const void **beta, size_t cols) {
        *gamma = vector(kF32 | kBF16 | kI16 | kU16, true, cols);
        const int type = good ? matrix_type(THPVariable_Unpack(args_[-1]).scalar_type()) : 0;
        *beta = vector(kF32 | kBF16 | kI16 | kU16, false, cols);
        if (good && *beta && matrix_type(THPVariable_Unpack(args_[-1]).scalar_type()) != type)
            fail();
        return type;
    }

    // Bytes to work in, at least `need` of them; None where none are needed.
    void *workspace(size_t need, size_t *size) {
        *size = 0;
        if (!take() || (args_[-1] == Py_None && need == 0))
            return nullptr;
        void *p = nullptr;
        good = address(args_[-1], device_, kU8, (long long)need, &p);
        if (good)
            *size = (size_t)THPVariable_Unpack(args_[-1]).numel();
        return p;
    }

    // An address as an integer.
    void *handle() { return pointer(); }
    double number() { return take() ? PyFloat_AsDouble(args_[-1]) : 0.0; }
    bool truth() { return take() && PyObject_IsTrue(args_[-1]) == 1; }

    void *fn;
    hipStream_t stream;
    hipEvent_t wait, done;
    bool good = true;

  private:
    bool take() {
        if (good && args_ < end_) {
            ++args_;
            return true;
        }
        good = false;
        return false;
    }
    void *pointer() {
        if (!take() || args_[-1] == Py_None)
            return nullptr;
        return PyLong_AsVoidPtr(args_[-1]);
    }
    const zpp_matrix *fail() {
        good = false;
        return nullptr;
    }

    PyObject *const *args_, *const *end_;
    long device_;
};

// Runs f on the call's arguments: the status that it returns, or None where an
// argument is not what the call takes.
template <class F>
PyObject *run_call(PyObject *const *args, Py_ssize_t n, F &&f) {
    try {
        Call c(args, n);
        const int status = f(c);
        if (c.good && !PyErr_Occurred())
            return PyLong_FromLong(status);
    } catch (const std::exception &) {
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

constexpr unsigned kPlain = 1u << ZPP_BF16 | 1u << ZPP_F32, kSaved = 1u << ZPP_I8;

PyObject *checkpoint(PyObject *const *args, Py_ssize_t n, bool save) {
    return run_call(args, n, [save](Call &c) {
        zpp_matrix from, to;
        size_t rows = 0, cols = 0;
        c.good = c.shape(&rows, &cols);
        const zpp_matrix *pf = c.matrix(&from, save ? kPlain : kSaved, true, rows, cols);
        const zpp_matrix *pt = c.matrix(&to, save ? kSaved : kPlain, true, rows, cols);
        return c.good ? (int)reinterpret_cast<decltype(&zpp_checkpoint_save)>(c.fn)(
                            pf, pt, rows, cols, c.stream, c.wait, c.done)
                      : 0;
    });
}
// checkpoint_save(fn, device, stream, wait, done, x, saved)
PyObject *checkpoint_save(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return checkpoint(args, n, true);
}
// checkpoint_load(fn, device, stream, wait, done, saved, out)
PyObject *checkpoint_load(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return checkpoint(args, n, false);
}

// layer_norm_forward(fn, device, stream, wait, done, x, residual, y, total, saved,
//                    gamma, beta, mean, rstd, eps)
PyObject *layer_norm_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return run_call(args, n, [](Call &c) {
        zpp_matrix m[5];
        size_t rows = 0, cols = 0;
        c.good = c.shape(&rows, &cols);
        const zpp_matrix *x = c.matrix(&m[0], kPlain, true, rows, cols);
        const zpp_matrix *residual = c.matrix(&m[1], kPlain, false, rows, cols);
        const zpp_matrix *y = c.matrix(&m[2], kPlain, true, rows, cols);
        const zpp_matrix *total = c.matrix(&m[3], kPlain, false, rows, cols);
        const zpp_matrix *saved = c.matrix(&m[4], kSaved, false, rows, cols);
        const void *gamma, *beta;
        const int type = c.params(&gamma, &beta, cols);
        float *mean = c.vector<float>(kF32, false, rows);
        float *rstd = c.vector<float>(kF32, false, rows);
        const float eps = (float)c.number();
        if (!c.good || PyErr_Occurred())
            return 0;
        return (int)reinterpret_cast<decltype(&zpp_layer_norm_forward)>(c.fn)(
            x, residual, gamma, beta, type, rows, cols, eps, y, total, saved, mean, rstd, c.stream,
            c.wait, c.done);
    });
}

// layer_norm_backward(fn, device, stream, wait, done, dy, x, dresidual, dx, y, gamma,
//                     beta, mean, rstd, dgamma, dbeta, accumulate, sizes, workspace)
// sizes: the address of zpp_layer_norm_backward_workspace
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return run_call(args, n, [](Call &c) {
        zpp_matrix m[5];
        size_t rows = 0, cols = 0, size = 0;
        c.good = c.shape(&rows, &cols);
        const zpp_matrix *dy = c.matrix(&m[0], kPlain, true, rows, cols);
        const zpp_matrix *x = c.matrix(&m[1], kPlain | kSaved, true, rows, cols);
        const zpp_matrix *dresidual = c.matrix(&m[2], kPlain, false, rows, cols);
        const zpp_matrix *dx = c.matrix(&m[3], kPlain, true, rows, cols);
        const zpp_matrix *y = c.matrix(&m[4], kPlain, false, rows, cols);
        const void *gamma, *beta;
        const int type = c.params(&gamma, &beta, cols);
        const float *mean = c.vector<float>(kF32, true, rows);
        const float *rstd = c.vector<float>(kF32, true, rows);
        float *dgamma = c.vector<float>(kF32, false, cols);
        float *dbeta = c.vector<float>(kF32, false, cols);
        const bool add = c.truth();
        const auto sizes = reinterpret_cast<decltype(&zpp_layer_norm_backward_workspace)>(c.handle());
        void *ws = c.good ? c.workspace(sizes(rows, cols), &size) : nullptr;
        if (!c.good || PyErr_Occurred())
            return 0;
        return (int)reinterpret_cast<decltype(&zpp_layer_norm_backward)>(c.fn)(
            dy, x, gamma, beta, type, mean, rstd, dresidual, rows, cols, dx, y, dgamma, dbeta, add,
            ws, size, c.stream, c.wait, c.done);
    });
}

// gelu_forward(fn, device, stream, wait, done, u, a, saved)
PyObject *gelu_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return run_call(args, n, [](Call &c) {
        zpp_matrix m[3];
        size_t rows = 0, cols = 0;
        c.good = c.shape(&rows, &cols);
        const zpp_matrix *u = c.matrix(&m[0], kPlain, true, rows, cols);
        const zpp_matrix *a = c.matrix(&m[1], kPlain, true, rows, cols);
        const zpp_matrix *saved = c.matrix(&m[2], kSaved, false, rows, cols);
        return c.good ? (int)reinterpret_cast<decltype(&zpp_gelu_forward)>(c.fn)(
                            u, rows, cols, a, saved, c.stream, c.wait, c.done)
                      : 0;
    });
}

// gelu_backward(fn, device, stream, wait, done, da, u, du, a)
PyObject *gelu_backward(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return run_call(args, n, [](Call &c) {
        zpp_matrix m[4];
        size_t rows = 0, cols = 0;
        c.good = c.shape(&rows, &cols);
        const zpp_matrix *da = c.matrix(&m[0], kPlain, true, rows, cols);
        const zpp_matrix *u = c.matrix(&m[1], kPlain | kSaved, true, rows, cols);
        const zpp_matrix *du = c.matrix(&m[2], kPlain, true, rows, cols);
        const zpp_matrix *a = c.matrix(&m[3], kPlain, false, rows, cols);
        return c.good ? (int)reinterpret_cast<decltype(&zpp_gelu_backward)>(c.fn)(
                            da, u, rows, cols, du, a, c.stream, c.wait, c.done)
                      : 0;
    });
}

// weight_grad(fn, device, stream, wait, done, dy, x, dw, accumulate, sizes, workspace)
// sizes: the address of zpp_weight_grad_workspace
PyObject *weight_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return run_call(args, n, [](Call &c) {
        zpp_matrix m[3];
        size_t rows = 0, cols = 0, rows_x = 0, k = 0, size = 0;
        c.good = c.shape(&rows, &cols);
        const zpp_matrix *dy = c.matrix(&m[0], 1u << ZPP_BF16, true, rows, cols);
        c.good = c.good && c.shape(&rows_x, &k);
        const zpp_matrix *x = c.matrix(&m[1], 1u << ZPP_BF16 | kSaved, true, rows, k);
        const zpp_matrix *dw = c.matrix(&m[2], 1u << ZPP_F32, true, cols, k);
        const bool add = c.truth();
        const auto sizes = reinterpret_cast<decltype(&zpp_weight_grad_workspace)>(c.handle());
        void *ws = c.good ? c.workspace(sizes(rows, cols, k), &size) : nullptr;
        if (!c.good || PyErr_Occurred())
            return 0;
        return (int)reinterpret_cast<decltype(&zpp_weight_grad)>(c.fn)(
            dy, x, rows, cols, k, dw, add, ws, size, c.stream, c.wait, c.done);
    });
}

PyMethodDef methods[] = {
#define ZPP_CALL(name)                                              \
    {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL,       \
     #name "(entry point, device, stream, events, arguments...) -> status or None"}
    ZPP_CALL(checkpoint_save),
    ZPP_CALL(checkpoint_load),
    ZPP_CALL(layer_norm_forward),
    ZPP_CALL(layer_norm_backward),
    ZPP_CALL(gelu_forward),
    ZPP_CALL(gelu_backward),
    ZPP_CALL(weight_grad),
    {"addresses", (PyCFunction)(void (*)(void))addresses, METH_FASTCALL,
     "addresses(device, tensor, mask, need, ...) -> tuple or None"},
    {"address_array", (PyCFunction)(void (*)(void))address_array, METH_FASTCALL,
     "address_array(device, tensors, mask, need) -> bytes or None"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject *m = PyModule_Create(&module);
    if (m && (PyModule_AddIntConstant(m, "F32", kF32) || PyModule_AddIntConstant(m, "BF16", kBF16) ||
              PyModule_AddIntConstant(m, "I16", kI16) || PyModule_AddIntConstant(m, "U16", kU16) ||
              PyModule_AddIntConstant(m, "I8", kI8) || PyModule_AddIntConstant(m, "U8", kU8) ||
              PyModule_AddIntConstant(m, "OPTIONAL", kOptional))) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
