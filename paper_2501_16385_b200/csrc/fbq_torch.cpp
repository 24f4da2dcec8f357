// Native marshalling of torch tensors into the C ABI of libfbq.so (module _fbq_torch): the part of the Python binding
// that a decode loop runs once per linear.  A linear at one token takes the GPU about five microseconds; marshalling
// its fourteen arguments in Python and through ctypes took the host more than ten (4096 -> 4096, INT4, rank 32, call
// after call: 15.2 us per call before, 4.2 us to issue and 5.7 us in all now).
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <initializer_list>
#include <sstream>

#include "../../include/fbq.h"

namespace {

// A tensor argument's address (NULL for None); false with an exception set when it is neither.
bool address(PyObject *o, void **out)
{
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a tensor");
        return false;
    }
    *out = THPVariable_Unpack(o).data_ptr();
    return true;
}

bool stream_of(PyObject *o, void **out)
{
    if (o == Py_None) {
        *out = static_cast<void *>(c10::cuda::getCurrentCUDAStream().stream());
        return true;
    }
    PyObject *h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) return false;
    *out = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

// While it lives new tensors are memory of `stream`, on which the call will write them, also where another stream is current: a block of that
// one's may still be written by work that it has queued, and one that is dropped goes back to those whose work is in order with the call.
class OutputsOf {
    c10::cuda::OptionalCUDAStreamGuard guard;

public:
    explicit OutputsOf(void *stream)
    {
        const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream();
        if (static_cast<void *>(current.stream()) != stream)
            guard.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), current.device_index()));
    }
};

// linear(x, qweight, scales, zeros, A, B, N, group, bits, y, stream) -> y, or the error code of the call
PyObject *py_linear(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (n != 11) {
        PyErr_SetString(PyExc_TypeError, "linear takes 11 arguments");
        return nullptr;
    }
    try {
        if (!THPVariable_Check(v[0])) {
            PyErr_SetString(PyExc_TypeError, "expected a tensor");
            return nullptr;
        }
        const at::Tensor &x = THPVariable_Unpack(v[0]);
        if (!x.is_cuda() || !x.is_contiguous() || x.dim() != 2) {
            PyErr_SetString(PyExc_AssertionError, "x must be a contiguous CUDA matrix");
            return nullptr;
        }
        const bool f16 = x.scalar_type() == at::kHalf;
        if (!f16 && x.scalar_type() != at::kBFloat16) {
            PyErr_SetString(PyExc_TypeError, "x must be float16 or bfloat16");
            return nullptr;
        }
        const int64_t M = x.size(0), K = x.size(1);
        const long N = PyLong_AsLong(v[6]), group = PyLong_AsLong(v[7]), bits = PyLong_AsLong(v[8]);
        if (PyErr_Occurred()) return nullptr;
        int64_t rank = 0;
        if (v[4] != Py_None) {
            if (!THPVariable_Check(v[4])) {
                PyErr_SetString(PyExc_TypeError, "expected a tensor");
                return nullptr;
            }
            rank = THPVariable_Unpack(v[4]).size(0);
        }
        void *p[6], *stream;
        for (int i = 1; i < 6; ++i)
            if (!address(v[i], &p[i])) return nullptr;
        if (!stream_of(v[10], &stream)) return nullptr;
        PyObject *y;
        if (v[9] == Py_None) {
            const OutputsOf there(stream);
            y = THPVariable_Wrap(at::empty({M, (int64_t)N}, x.options()));
            if (!y) return nullptr;
        } else {
            y = v[9];
            Py_INCREF(y);
        }
        void *yp;
        if (!address(y, &yp)) {
            Py_DECREF(y);
            return nullptr;
        }
        void *xp = x.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = (f16 ? fbq_linear : fbq_linear_bf16)(xp, static_cast<const uint32_t *>(p[1]), p[2], p[3], p[4], p[5], yp, (int)M, (int)N, (int)K,
                                                  (int)group, (int)bits, (int)rank, stream);
        Py_END_ALLOW_THREADS
        if (rc == FBQ_OK) return y;
        Py_DECREF(y);
        return PyLong_FromLong(rc);
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());   // (memory that is used up is torch.OutOfMemoryError)
        return nullptr;
    }
}

// linear_batch(address of the descriptors, count, M, group, bits, rank, bf16, host_io, stream) -> error code
PyObject *py_linear_batch(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "linear_batch takes 9 arguments");
        return nullptr;
    }
    const fbq_problem *problems = static_cast<const fbq_problem *>(PyLong_AsVoidPtr(v[0]));
    int a[7];
    for (int i = 0; i < 7; ++i) a[i] = (int)PyLong_AsLong(v[i + 1]);
    if (PyErr_Occurred()) return nullptr;
    void *stream;
    if (!stream_of(v[8], &stream)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (a[6] ? fbq_linear_batch_hostio : fbq_linear_batch)(problems, a[0], a[1], a[2], a[3], a[4], a[5], stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// ---- the feed-forward block's calls: every tensor is checked, for what gets past here is an address ----
struct BadOperand {};            // a Python exception is set

const char *type_name(at::ScalarType t) { return at::toString(t); }

// A contiguous tensor of the current device with the given type and shape; returns its address.
void *operand(PyObject *o, const char *what, at::ScalarType type, at::IntArrayRef shape)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
        throw BadOperand();
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous() || t.get_device() != c10::cuda::current_device()) {
        std::ostringstream msg;
        msg << what << " must be a contiguous " << type_name(type) << " tensor of shape " << shape << " on the current CUDA device, got " << type_name(t.scalar_type())
            << " of shape " << t.sizes() << " on " << t.device() << (t.is_contiguous() ? "" : ", not contiguous");
        PyErr_SetString(PyExc_ValueError, msg.str().c_str());
        throw BadOperand();
    }
    return t.data_ptr();
}
const at::Tensor &tensor_of(PyObject *o, const char *what, int dims)
{
    if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != dims) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor of %d dimensions", what, dims);
        throw BadOperand();
    }
    return THPVariable_Unpack(o);
}
at::ScalarType act_type(const at::Tensor &t, const char *what)
{
    const at::ScalarType s = t.scalar_type();
    if (s != at::kHalf && s != at::kBFloat16) {
        PyErr_Format(PyExc_TypeError, "%s must be float16 or bfloat16", what);
        throw BadOperand();
    }
    return s;
}
[[noreturn]] void bad_value(const char *text)
{
    PyErr_SetString(PyExc_ValueError, text);
    throw BadOperand();
}
int int_arg(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw BadOperand();
    if (v > 0x7FFFFFFF || v < -0x7FFFFFFFl) bad_value("a size does not fit 32 bits");
    return (int)v;
}
bool bool_arg(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw BadOperand();                               // (what has no truth value: a tensor of several elements, say)
    return v != 0;
}
int size_arg(int64_t n)
{
    if (n > 0x7FFFFFFF) bad_value("a size does not fit 31 bits");
    return (int)n;
}
int64_t groups_of(int64_t columns) { return (columns + 127) / 128; }

// A new tensor of the current device and stream (OutputsOf), without the dispatcher's detours: 0.5 us less, and dispatch modes do not see it.
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type) { return at::Tensor(at::detail::empty_cuda(shape, type, at::Device(at::kCUDA), std::nullopt)); }

struct Layer {
    void *q, *s, *z, *A = nullptr, *B = nullptr;
    int rank = 0;
};
// v: qweight, scales, zeros, A, B
Layer layer_of(PyObject *const *v, int64_t N, int64_t K, int group, int bits, at::ScalarType act)
{
    Layer l;
    if (group < 1 || K % group != 0) bad_value("K is not a multiple of group");
    const at::Tensor &q = THPVariable_Check(v[0]) ? THPVariable_Unpack(v[0]) : tensor_of(v[0], "qweight", 1);
    if (q.numel() != (int64_t)fbq_packed_words(size_arg(N), size_arg(K), bits)) bad_value("qweight does not hold the packed words of this layer");
    l.q = operand(v[0], "qweight", at::kInt, q.sizes());
    l.s = operand(v[1], "scales", at::kHalf, {N, K / group});
    l.z = operand(v[2], "zeros", at::kHalf, {N, K / group});
    if ((v[3] == Py_None) != (v[4] == Py_None)) bad_value("A and B belong together");
    if (v[3] != Py_None) {
        const int64_t r = tensor_of(v[3], "A", 2).size(0);
        l.A = operand(v[3], "A", act, {r, K});
        l.B = operand(v[4], "B", act, {N, r});
        l.rank = size_arg(r);
    }
    return l;
}

template <typename F> PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f)
{
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (const BadOperand &) {
        return nullptr;
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());   // (memory that is used up is torch.OutOfMemoryError)
        return nullptr;
    }
}
template <typename F> int without_gil(F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}
void *stream_arg(PyObject *o)
{
    void *s;
    if (!stream_of(o, &s)) throw BadOperand();
    return s;
}
// New references of `t` (None where it is undefined), as a tuple; or the one alone.
PyObject *results(std::initializer_list<at::Tensor> ts)
{
    PyObject *tuple = PyTuple_New((Py_ssize_t)ts.size());
    if (!tuple) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) {
        PyObject *o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, i++, o);
    }
    return tuple;
}

// gated(x, qweight, scales, zeros, A, B, N, group, bits, gate, save, h, stream) -> h or (h, codes, scales), or the error code of the call
PyObject *py_gated(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    return guarded(n, 13, [&]() -> PyObject * {
        const at::Tensor &x = tensor_of(v[0], "x", 2);
        const at::ScalarType act = act_type(x, "x");
        const int64_t M = x.size(0), K = x.size(1);
        const int N = int_arg(v[6]), group = int_arg(v[7]), bits = int_arg(v[8]), gate = int_arg(v[9]);
        const bool save = bool_arg(v[10]);
        if (N < 2) bad_value("N must be positive");
        void *px = operand(v[0], "x", act, {M, K});
        const Layer l = layer_of(v + 1, N, K, group, bits, act);
        void *stream = stream_arg(v[12]);
        const OutputsOf there(stream);
        at::Tensor h, codes, scales;
        if (v[11] == Py_None) {
            h = fresh({M, N / 2}, act);
        } else {
            operand(v[11], "h", act, {M, N / 2});
            h = THPVariable_Unpack(v[11]);
        }
        if (save) {
            codes = fresh({M, N}, at::kChar);
            scales = fresh({M, groups_of(N)}, at::kFloat);
        }
        const int m = size_arg(M), k = size_arg(K);
        const int rc = without_gil([&] {
            return fbq_gated(px, (const uint32_t *)l.q, l.s, l.z, l.A, l.B, h.data_ptr(), save ? (int8_t *)codes.data_ptr() : nullptr,
                             save ? (float *)scales.data_ptr() : nullptr, m, N, k, group, bits, l.rank, gate, act == at::kBFloat16, stream);
        });
        if (rc != FBQ_OK) return PyLong_FromLong(rc);
        return save ? results({h, codes, scales}) : THPVariable_Wrap(h);
    });
}

// act8_pack(x, stream) -> (codes, scales), or the error code
PyObject *py_act8_pack(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    return guarded(n, 2, [&]() -> PyObject * {
        const at::Tensor &x = tensor_of(v[0], "x", 2);
        const at::ScalarType act = act_type(x, "x");
        const int64_t M = x.size(0), K = x.size(1);
        void *px = operand(v[0], "x", act, {M, K}), *stream = stream_arg(v[1]);
        const OutputsOf there(stream);
        const at::Tensor codes = fresh({M, K}, at::kChar), scales = fresh({M, groups_of(K)}, at::kFloat);
        const int m = size_arg(M), k = size_arg(K);
        const int rc = without_gil([&] { return fbq_act8_pack(px, (int8_t *)codes.data_ptr(), (float *)scales.data_ptr(), m, k, act == at::kBFloat16, stream); });
        return rc == FBQ_OK ? results({codes, scales}) : PyLong_FromLong(rc);
    });
}

// act8_unpack(codes, scales, bf16, stream) -> x, or the error code
PyObject *py_act8_unpack(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    return guarded(n, 4, [&]() -> PyObject * {
        const at::Tensor &codes = tensor_of(v[0], "codes", 2);
        const int64_t M = codes.size(0), K = codes.size(1);
        void *pc = operand(v[0], "codes", at::kChar, {M, K}), *ps = operand(v[1], "scales", at::kFloat, {M, groups_of(K)});
        const bool bf16 = bool_arg(v[2]);
        void *stream = stream_arg(v[3]);
        const OutputsOf there(stream);
        const at::Tensor x = fresh({M, K}, bf16 ? at::kBFloat16 : at::kHalf);
        const int m = size_arg(M), k = size_arg(K);
        const int rc = without_gil([&] { return fbq_act8_unpack((const int8_t *)pc, (const float *)ps, x.data_ptr(), m, k, bf16, stream); });
        return rc == FBQ_OK ? THPVariable_Wrap(x) : PyLong_FromLong(rc);
    });
}

// backward(gated, dy or dh, kept codes, kept scales, x or codes, x's scales or None, qweight, scales, zeros, A, B, group, bits, gate, want dx, want factors, stream)
// -> (dx, dA, dB), or the error code
PyObject *py_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    return guarded(n, 17, [&]() -> PyObject * {
        const bool gated = bool_arg(v[0]), want_dx = bool_arg(v[14]), want_factors = bool_arg(v[15]);
        const char *what = gated ? "dh" : "dy";
        const at::Tensor &dy = tensor_of(v[1], what, 2);
        const at::ScalarType act = act_type(dy, what);
        const int group = int_arg(v[11]), bits = int_arg(v[12]), gate = int_arg(v[13]);
        const int64_t M = dy.size(0), N = gated ? 2 * dy.size(1) : dy.size(1), K = tensor_of(v[7], "scales", 2).size(1) * group;
        void *pdy = operand(v[1], what, act, dy.sizes());
        const Layer l = layer_of(v + 6, N, K, group, bits, act);
        void *kept = nullptr, *kept_scales = nullptr, *x = nullptr, *x8 = nullptr, *x8_scales = nullptr;
        if (gated) {
            kept = operand(v[2], "kept codes", at::kChar, {M, N});
            kept_scales = operand(v[3], "kept scales", at::kFloat, {M, groups_of(N)});
        }
        if (v[5] != Py_None) {
            x8 = operand(v[4], "x codes", at::kChar, {M, K});
            x8_scales = operand(v[5], "x scales", at::kFloat, {M, groups_of(K)});
        } else if (v[4] != Py_None) {
            x = operand(v[4], "x", act, {M, K});
        }
        void *stream = stream_arg(v[16]);
        const OutputsOf there(stream);
        at::Tensor dx, dA, dB;
        if (want_dx) dx = fresh({M, K}, act);
        if (want_factors && l.rank > 0) {
            dA = fresh({l.rank, K}, act);
            dB = fresh({N, l.rank}, act);
        }
        auto at_of = [](const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        const int m = size_arg(M), nn = size_arg(N), k = size_arg(K);
        const int rc = without_gil([&] {
            if (gated)
                return fbq_gated_backward(pdy, (const int8_t *)kept, (const float *)kept_scales, x, (const int8_t *)x8, (const float *)x8_scales, (const uint32_t *)l.q, l.s, l.z,
                                          l.A, l.B, at_of(dx), at_of(dA), at_of(dB), m, nn, k, group, bits, l.rank, gate, act == at::kBFloat16, stream);
            return fbq_linear_backward(pdy, x, (const int8_t *)x8, (const float *)x8_scales, (const uint32_t *)l.q, l.s, l.z, l.A, l.B, at_of(dx), at_of(dA), at_of(dB), m, nn,
                                       k, group, bits, l.rank, act == at::kBFloat16, stream);
        });
        return rc == FBQ_OK ? results({dx, dA, dB}) : PyLong_FromLong(rc);
    });
}

PyMethodDef methods[] = {{"gated", (PyCFunction)(void (*)(void))py_gated, METH_FASTCALL, nullptr},
                         {"act8_pack", (PyCFunction)(void (*)(void))py_act8_pack, METH_FASTCALL, nullptr},
                         {"act8_unpack", (PyCFunction)(void (*)(void))py_act8_unpack, METH_FASTCALL, nullptr},
                         {"backward", (PyCFunction)(void (*)(void))py_backward, METH_FASTCALL, nullptr},
                         {"linear", (PyCFunction)(void (*)(void))py_linear, METH_FASTCALL, nullptr},
                         {"linear_batch", (PyCFunction)(void (*)(void))py_linear_batch, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fbq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fbq_torch() { return PyModule_Create(&module); }
