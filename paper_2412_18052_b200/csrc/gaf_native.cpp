// Argument marshalling of the calls that a training loop makes every step, as a CPython extension over the C ABI of
// include/gaf.h.  With ctypes a filter call on 3 or 4 gradients spent 10 to 13 us in the interpreter (tensor
// attributes one by one, pointer arrays, the current stream, 14 converted arguments), which is longer than the
// GPU needs for a million parameters; here the tensors are read directly.
//
// Every function takes its arguments by position (binding.py has the signatures with defaults), checks what the
// binding has always checked, allocates outputs that were not given and raises the error class that
// binding.py registers.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <new>
#include <optional>
#include <vector>

#include "../../include/gaf.h"

namespace {

PyObject *g_error = nullptr;            // GafError(code, where)

struct Failed {};                       // a Python exception is set

[[noreturn]] void fail(PyObject *type, const char *text) {
    PyErr_SetString(type, text);
    throw Failed();
}
[[noreturn]] void fail_code(int code, const char *where) {
    PyObject *e = g_error ? PyObject_CallFunction(g_error, "is", code, where) : nullptr;
    if (e) { PyErr_SetObject(g_error, e); Py_DECREF(e); }
    else if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, where);
    throw Failed();
}
void check(int code, const char *where) {
    if (code != GAF_OK) fail_code(code, where);
}

const at::Tensor &tensor(PyObject *o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a torch tensor");
    return THPVariable_Unpack(o);
}
int dtype_code(const at::Tensor &t) {
    if (t.scalar_type() == at::kFloat) return GAF_F32;
    if (t.scalar_type() == at::kBFloat16) return GAF_BF16;
    PyErr_Format(PyExc_TypeError, "gradients must be float32 or bfloat16, got %s", c10::toString(t.scalar_type()));
    throw Failed();
}
void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

double number(PyObject *o) {
    if (PyFloat_Check(o)) return PyFloat_AS_DOUBLE(o);
    PyObject *f = PyNumber_Float(o);    // what float() takes: numpy and torch scalars, texts
    if (!f) throw Failed();
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return v;
}
int64_t integer(PyObject *o) {
    if (PyLong_Check(o)) {
        const int64_t v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) throw Failed();
        return v;
    }
    PyObject *i = PyNumber_Long(o);     // (numpy integers and the like)
    if (!i) throw Failed();
    const int64_t v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw Failed();
    return v;
}

// The items of anything that has a length and, where `indexed`, can be indexed (a generator has neither: its items would be
// used up by one call).  They stay alive as long as this object does.
struct Sequence {
    PyObject *fast;
    Py_ssize_t n;
    explicit Sequence(PyObject *o, bool indexed = false) : fast(nullptr), n(0) {
        if (!PyList_Check(o) && !PyTuple_Check(o)) {
            const Py_ssize_t len = PyObject_Size(o);
            if (len < 0) throw Failed();
            if (indexed && len > 0) {
                PyObject *zero = PyLong_FromLong(0), *item = zero ? PyObject_GetItem(o, zero) : nullptr;
                Py_XDECREF(zero);
                if (!item) throw Failed();
                Py_DECREF(item);
            }
        }
        fast = PySequence_Fast(o, "expected a sequence");
        if (!fast) throw Failed();
        n = PySequence_Fast_GET_SIZE(fast);
    }
    ~Sequence() { Py_DECREF(fast); }
    Sequence(const Sequence &) = delete;
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

// The gradients of a call: pointers, length, type, device.  It holds the tensors until the call has been made: a sequence may make
// them as they are asked for, and memory that is freed before the outputs are allocated becomes the outputs.
struct Gradients {
    const Sequence seq;
    std::vector<const void *> ptr;
    int64_t D = 0;
    int dtype = 0;
    at::Device device = at::kCPU;
    Gradients(PyObject *o, bool must_match) : seq(o, true) {
        if (seq.n == 0) fail(PyExc_IndexError, "no gradients");
        ptr.reserve(seq.n);
        const at::Tensor &first = tensor(seq[0]);
        D = first.numel();
        dtype = dtype_code(first);
        device = first.device();
        for (Py_ssize_t i = 0; i < seq.n; ++i) {
            const at::Tensor &t = tensor(seq[i]);
            if (must_match && (t.numel() != D || t.scalar_type() != first.scalar_type() || !t.is_contiguous()))
                fail(PyExc_AssertionError, "gradients must be contiguous tensors of one length and type");
            ptr.push_back(t.data_ptr());
        }
    }
    int K() const { return static_cast<int>(ptr.size()); }
};

// A step order for K gradients, or null for the identity.  What is missing from one that is too short, and a number that no int32
// holds, become -1, which the library refuses; what a longer one has beyond K is not looked at.
struct Order {
    std::vector<int32_t> v;
    const int32_t *ptr = nullptr;
    Order(PyObject *o, int K) {
        if (o == Py_None) return;
        const Sequence seq(o);
        v.assign(K, -1);
        for (Py_ssize_t i = 0; i < seq.n && i < K; ++i) {
            const int64_t x = integer(seq[i]);
            if (x >= 0 && x <= INT32_MAX) v[i] = static_cast<int32_t>(x);
        }
        ptr = v.data();
    }
};

// An output: the given tensor, or a new one.
struct Output {
    PyObject *object;
    void *ptr;
    Output(PyObject *given, at::IntArrayRef shape, at::ScalarType type, at::Device device) {
        if (given != Py_None) {
            ptr = tensor(given).data_ptr();
            object = Py_NewRef(given);
        } else {
            const at::Tensor t = at::empty(shape, at::TensorOptions().dtype(type).device(device));
            ptr = t.data_ptr();
            object = THPVariable_Wrap(t);
            if (!object) throw Failed();
        }
    }
    ~Output() { Py_XDECREF(object); }
    Output(const Output &) = delete;
    PyObject *take() { PyObject *o = object; object = nullptr; return o; }
};
template <typename T> T *as(const Output &o) { return static_cast<T *>(o.ptr); }

struct Workspace {
    void *ptr;
    size_t bytes;
    explicit Workspace(PyObject *o) {
        const at::Tensor &t = tensor(o);
        ptr = t.data_ptr();
        bytes = static_cast<size_t>(t.numel());
    }
};

template <typename F>
int without_gil(F &&f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}
// Runs a body that throws Failed (a Python exception is set) or a torch error.
template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F &&f) {
    if (n != want) { PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n); return nullptr; }
    try {
        return f();
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
template <typename... O>
PyObject *tuple_of(O &...o) {
    PyObject *t = PyTuple_New(sizeof...(o));
    if (!t) throw Failed();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(t, i++, o.take()), ...);
    return t;
}

PyObject *py_filter_accumulate(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const Gradients g(a[0], true);
        const double tau = number(a[1]);
        const Workspace ws(a[2]);
        const Order order(a[3], g.K());
        Output macro(a[4], {g.D}, at::kFloat, g.device), mask(a[5], {g.K()}, at::kByte, g.device),
            dist(a[6], {g.K()}, at::kFloat, g.device), count(a[7], {1}, at::kInt, g.device);
        const int schedule = static_cast<int>(integer(a[8]));
        void *const st = stream();
        check(without_gil([&] {
            return gaf_filter_accumulate(g.ptr.data(), g.K(), g.D, g.dtype, tau, order.ptr, as<float>(macro), as<uint8_t>(mask),
                                         as<float>(dist), as<int32_t>(count), ws.ptr, ws.bytes, schedule, st);
        }), "gaf_filter_accumulate");
        return tuple_of(macro, mask, dist, count);
    });
}

PyObject *py_filter_accumulate_any_seed(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        const Gradients g(a[0], false);
        const double tau = number(a[1]);
        const Workspace ws(a[2]);
        Output macro(a[3], {g.D}, at::kFloat, g.device), mask(Py_None, {g.K()}, at::kByte, g.device),
            dist(Py_None, {g.K()}, at::kFloat, g.device), count(Py_None, {1}, at::kInt, g.device),
            seed(Py_None, {1}, at::kInt, g.device);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_filter_accumulate_any_seed(g.ptr.data(), g.K(), g.D, g.dtype, tau, as<float>(macro), as<uint8_t>(mask),
                                                  as<float>(dist), as<int32_t>(count), as<int32_t>(seed), ws.ptr, ws.bytes, st);
        }), "gaf_filter_accumulate_any_seed");
        return tuple_of(macro, mask, dist, count, seed);
    });
}

PyObject *py_filter_accumulate_bucketed(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const Gradients g(a[0], false);
        const double tau = number(a[1]);
        std::vector<int64_t> offsets;
        {
            const Sequence seq(a[2]);
            offsets.reserve(seq.n);
            for (Py_ssize_t i = 0; i < seq.n; ++i) offsets.push_back(integer(seq[i]));
        }
        const int64_t S = static_cast<int64_t>(offsets.size()) - 1;
        if (S < 0) fail(PyExc_ValueError, "no bucket offsets");
        const Workspace ws(a[3]);
        const Order order(a[4], g.K());
        Output macro(a[5], {g.D}, at::kFloat, g.device), mask(Py_None, {S, g.K()}, at::kByte, g.device),
            dist(Py_None, {S, g.K()}, at::kFloat, g.device), count(Py_None, {S}, at::kInt, g.device);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_filter_accumulate_bucketed(g.ptr.data(), g.K(), g.D, g.dtype, tau, order.ptr, static_cast<int>(S),
                                                  offsets.data(), as<float>(macro), as<uint8_t>(mask), as<float>(dist),
                                                  as<int32_t>(count), ws.ptr, ws.bytes, st);
        }), "gaf_filter_accumulate_bucketed");
        return tuple_of(macro, mask, dist, count);
    });
}

PyObject *py_pairwise_cosdist(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        const Gradients g(a[0], false);
        const Workspace ws(a[1]);
        Output dist(a[2], {g.K(), g.K()}, at::kFloat, g.device), gram(a[3], {g.K(), g.K()}, at::kDouble, g.device);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_pairwise_cosdist(g.ptr.data(), g.K(), g.D, g.dtype, as<float>(dist), as<double>(gram), ws.ptr, ws.bytes, st);
        }), "gaf_pairwise_cosdist");
        return tuple_of(dist, gram);
    });
}

PyObject *py_cosdist(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 5, [&] {
        const at::Tensor &x = tensor(a[0]), &y = tensor(a[1]);
        if (x.numel() != y.numel() || x.scalar_type() != y.scalar_type())
            fail(PyExc_AssertionError, "the two tensors must have one length and type");
        const int dtype = dtype_code(x);
        const Workspace ws(a[2]);
        Output dist(a[3], {1}, at::kFloat, x.device()), stats(a[4], {3}, at::kDouble, x.device());
        void *const st = stream();
        check(without_gil([&] {
            return gaf_cosdist(x.data_ptr(), y.data_ptr(), x.numel(), dtype, as<float>(dist), as<double>(stats), ws.ptr, ws.bytes, st);
        }), "gaf_cosdist");
        return tuple_of(dist, stats);
    });
}

PyObject *py_stream_begin(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 3, [&] {
        const at::Tensor &seed = tensor(a[0]);
        const int dtype = dtype_code(seed);
        float *const acc = static_cast<float *>(tensor(a[1]).data_ptr());
        const Workspace ws(a[2]);
        void *const st = stream();
        check(without_gil([&] { return gaf_stream_begin(seed.data_ptr(), seed.numel(), dtype, acc, ws.ptr, ws.bytes, st); }),
              "gaf_stream_begin");
        return Py_NewRef(Py_None);
    });
}

PyObject *py_stream_push(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 5, [&] {
        const at::Tensor &g = tensor(a[0]);
        const int dtype = dtype_code(g), t = static_cast<int>(integer(a[1]));
        const double tau = number(a[2]);
        float *const acc = static_cast<float *>(tensor(a[3]).data_ptr());
        const Workspace ws(a[4]);
        void *const st = stream();
        check(without_gil([&] { return gaf_stream_push(g.data_ptr(), t, g.numel(), dtype, tau, acc, ws.ptr, ws.bytes, st); }),
              "gaf_stream_push");
        return Py_NewRef(Py_None);
    });
}

PyObject *py_stream_end(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 3, [&] {
        const int64_t K = integer(a[0]);
        const at::Tensor &acc = tensor(a[1]);
        const Workspace ws(a[2]);
        Output mask(Py_None, {K}, at::kByte, acc.device()), dist(Py_None, {K}, at::kFloat, acc.device()),
            count(Py_None, {1}, at::kInt, acc.device());
        void *const st = stream();
        check(without_gil([&] {
            return gaf_stream_end(static_cast<int>(K), acc.numel(), static_cast<float *>(acc.data_ptr()), as<uint8_t>(mask), as<float>(dist),
                                  as<int32_t>(count), ws.ptr, ws.bytes, st);
        }), "gaf_stream_end");
        return tuple_of(mask, dist, count);
    });
}

// ---- layers of a language model -----------------------------------------------------------------------------------

[[noreturn]] void fail_value(const char *what, const char *text) {
    PyErr_Format(PyExc_ValueError, "%s %s", what, text);
    throw Failed();
}
bool truth(PyObject *o) {
    const int t = PyObject_IsTrue(o);
    if (t < 0) throw Failed();          // (what an object's own conversion raised)
    return t == 1;
}
// A tensor on the current device, whose stream the call will use.
const at::Tensor &cuda_tensor(PyObject *o, const char *what) {
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.device().index() != c10::cuda::current_device()) fail_value(what, "must be on the current CUDA device");
    return t;
}
int float_code(const at::Tensor &t, const char *what) {
    if (t.scalar_type() == at::kFloat) return GAF_F32;
    if (t.scalar_type() == at::kBFloat16) return GAF_BF16;
    PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16, got %s", what, c10::toString(t.scalar_type()));
    throw Failed();
}
at::ScalarType float_type(int code) { return code == GAF_F32 ? at::kFloat : at::kBFloat16; }

// Rows of elements next to one another: any leading dimensions that are laid out as one (a missing matrix: null).
struct Matrix {
    void *ptr = nullptr;
    int64_t rows = 0, cols = 0, stride = 0;
    int dtype = 0;
    const at::Tensor *t = nullptr;
    Matrix() = default;
    Matrix(PyObject *o, const char *what, at::ScalarType want = at::ScalarType::Undefined) {
        if (o == Py_None) return;
        t = &cuda_tensor(o, what);
        if (want == at::ScalarType::Undefined) dtype = float_code(*t, what);
        else if (t->scalar_type() != want) {
            PyErr_Format(PyExc_TypeError, "%s must be %s, got %s", what, c10::toString(want), c10::toString(t->scalar_type()));
            throw Failed();
        }
        if (t->dim() < 1) fail_value(what, "must have rows");
        const int64_t n = t->dim();
        cols = t->size(n - 1);
        rows = 1;
        stride = cols;
        bool any = false;                // whether a dimension longer than 1 has set the stride
        for (int64_t i = n - 2; i >= 0; --i) {
            if (t->size(i) != 1) {
                if (!any) { stride = t->stride(i); any = true; }
                else if (t->numel() > 0 && t->stride(i) != stride * rows) fail_value(what, "must have rows at equal distances");
            }
            rows *= t->size(i);
        }
        if (cols > 1 && t->stride(n - 1) != 1) fail_value(what, "must have rows of neighbouring elements");
        ptr = t->data_ptr();
    }
    bool has(int64_t r, int64_t c) const { return rows == r && cols == c; }
};
void same_shape(const Matrix &m, int64_t rows, int64_t cols, int dtype, const char *what) {
    if (m.t && (!m.has(rows, cols) || m.dtype != dtype)) fail_value(what, "has another shape or type than the call's matrices");
}
// A vector, or a block of memory that is used as one.
const at::Tensor &dense(PyObject *o, const char *what, int64_t numel) {
    const at::Tensor &t = cuda_tensor(o, what);
    if (!t.is_contiguous() || t.numel() != numel) fail_value(what, "must be contiguous and of the right size");
    return t;
}
// An output that is given (dense, of this size and type) or made; `like`: the shape that a new one takes.
struct LayerOutput {
    PyObject *object = nullptr;
    void *ptr = nullptr;
    LayerOutput() = default;
    LayerOutput(PyObject *given, at::IntArrayRef shape, at::ScalarType type, at::Device device, const char *what) {
        if (given != Py_None) {
            int64_t n = 1;
            for (int64_t s : shape) n *= s;
            const at::Tensor &t = dense(given, what, n);
            if (t.scalar_type() != type || t.dim() < 1 || t.size(t.dim() - 1) != shape.back()) fail_value(what, "has another shape or type than the result");
            ptr = t.data_ptr();
            object = Py_NewRef(given);
        } else {
            const at::Tensor t = at::empty(shape, at::TensorOptions().dtype(type).device(device));
            ptr = t.data_ptr();
            object = THPVariable_Wrap(t);
            if (!object) throw Failed();
        }
    }
    ~LayerOutput() { Py_XDECREF(object); }
    LayerOutput(const LayerOutput &) = delete;
    PyObject *take() {
        PyObject *o = object ? object : Py_NewRef(Py_None);
        object = nullptr;
        return o;
    }
};
// Codes and scales of a matrix of `rows` x `cols`: a pair of uint8 tensors, or None.  It holds the tensors until the call has been made: a
// sequence may make them as they are asked for, and another thread may put others into a list.
struct Checkpoint {
    std::optional<Sequence> seq;
    at::Tensor held[2];
    Matrix codes;
    uint8_t *scales = nullptr;
    Checkpoint(PyObject *o, const char *what, int64_t rows = -1, int64_t cols = -1) {
        if (o == Py_None) return;
        seq.emplace(o, true);
        if (seq->n != 2) fail_value(what, "is a pair of codes and scales");
        for (int i = 0; i < 2; ++i) held[i] = tensor((*seq)[i]);
        codes = Matrix((*seq)[0], what, at::kByte);
        if (rows < 0) { rows = codes.rows; cols = codes.cols; }
        if (!codes.has(rows, cols)) fail_value(what, "has another shape than the call's matrices");
        const at::Tensor &s = dense((*seq)[1], what, rows * ((cols + 127) / 128));
        if (s.scalar_type() != at::kByte) fail_value(what, "has scales that are not uint8");
        scales = static_cast<uint8_t *>(s.data_ptr());
    }
    uint8_t *ptr() const { return static_cast<uint8_t *>(codes.ptr); }
};
struct Tokens {
    const void *ptr;
    int64_t n;
    int type;
    const at::Tensor &t;
    explicit Tokens(PyObject *o) : t(cuda_tensor(o, "tokens")) {
        if (t.scalar_type() == at::kLong) type = GAF_I64;
        else if (t.scalar_type() == at::kInt) type = GAF_I32;
        else fail(PyExc_TypeError, "tokens must be int64 or int32");
        if (!t.is_contiguous()) fail_value("tokens", "must be contiguous");
        ptr = t.data_ptr();
        n = t.numel();
    }
};
struct LayerWorkspace {
    void *ptr;
    size_t bytes;
    explicit LayerWorkspace(PyObject *o) {
        const at::Tensor &t = cuda_tensor(o, "workspace");
        if (!t.is_contiguous()) fail_value("workspace", "must be contiguous");
        ptr = t.data_ptr();
        bytes = t.nbytes();
    }
};
// The gradient of a weight (any dense view of a flat gradient) and what is added to it.
struct WeightGradient {
    void *ptr;
    const void *base = nullptr;
    int dtype;
    PyObject *object;
    WeightGradient(PyObject *grad, PyObject *base_o, int64_t numel, const char *what) : object(grad) {
        const at::Tensor &t = dense(grad, what, numel);
        dtype = float_code(t, what);
        ptr = t.data_ptr();
        if (base_o != Py_None) {
            const at::Tensor &b = dense(base_o, "base", numel);
            if (b.scalar_type() != t.scalar_type()) fail_value("base", "has another type than the gradient");
            base = b.data_ptr();
        }
    }
};
std::vector<int64_t> shape_with(const at::Tensor &like, bool drop_last, int64_t last) {
    std::vector<int64_t> s(like.sizes().begin(), like.sizes().end());
    if (drop_last) s.pop_back();
    if (last >= 0) s.push_back(last);
    return s;
}

PyObject *py_embedding(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        const Matrix table(a[0], "table");
        if (!table.t || table.t->dim() != 2) fail_value("table", "must be a matrix");
        const Tokens tokens(a[1]);
        const double scale = number(a[2]);
        const std::vector<int64_t> shape = shape_with(tokens.t, false, table.cols);
        LayerOutput out(a[3], shape, table.t->scalar_type(), table.t->device(), "out");
        void *const st = stream();
        check(without_gil([&] {
            return gaf_embedding(table.ptr, table.stride, table.rows, table.cols, table.dtype, tokens.ptr, tokens.type, tokens.n, scale, out.ptr, st);
        }), "gaf_embedding");
        return out.take();
    });
}

PyObject *py_embedding_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const Matrix dy(a[0], "dy");
        if (!dy.t) fail_value("dy", "is missing");
        const Tokens tokens(a[1]);
        if (tokens.n != dy.rows) fail_value("tokens", "must be one per row of dy");
        const at::Tensor &grad = cuda_tensor(a[2], "grad");
        if (grad.dim() != 2 || grad.size(1) != dy.cols) fail_value("grad", "must be a matrix as wide as dy");
        const WeightGradient g(a[2], a[5], grad.numel(), "grad");
        const LayerWorkspace ws(a[3]);
        const double scale = number(a[4]);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_embedding_grad(dy.ptr, dy.stride, dy.rows, dy.cols, dy.dtype, tokens.ptr, tokens.type, scale, g.base, g.ptr, g.dtype, grad.size(0),
                                      ws.ptr, ws.bytes, st);
        }), "gaf_embedding_grad");
        return Py_NewRef(a[2]);
    });
}

PyObject *py_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        // x, weight, residual, eps, want_y, y, h, rstd, y_checkpoint, coded_y, h_checkpoint
        const Matrix x(a[0], "x");
        if (!x.t) fail_value("x", "is missing");
        const at::Tensor &weight = dense(a[1], "weight", x.cols);
        if (weight.scalar_type() != x.t->scalar_type()) fail_value("weight", "has another type than x");
        const Matrix residual(a[2], "residual");
        same_shape(residual, x.rows, x.cols, x.dtype, "residual");
        const double eps = number(a[3]);
        const bool want_y = truth(a[4]), coded_y = truth(a[9]);
        const std::vector<int64_t> shape = shape_with(*x.t, false, -1), rows = shape_with(*x.t, true, -1);
        const at::ScalarType type = x.t->scalar_type();
        const at::Device device = x.t->device();
        LayerOutput y, h, rstd;
        auto make = [&](LayerOutput &o, PyObject *given, const char *what) { new (&o) LayerOutput(given, shape, type, device, what); };
        if (want_y || a[5] != Py_None) make(y, a[5], "y");
        if (residual.t) make(h, a[6], "h");
        else if (a[6] != Py_None) fail_value("h", "is only written with a residual");
        if (a[7] != Py_None) {
            const at::Tensor &t = dense(a[7], "rstd", x.rows);
            if (t.scalar_type() != at::kFloat) fail_value("rstd", "must be float32");
            rstd.ptr = t.data_ptr();
            rstd.object = Py_NewRef(a[7]);
        } else {
            const at::Tensor t = at::empty(rows, at::TensorOptions().dtype(at::kFloat).device(device));
            rstd.ptr = t.data_ptr();
            rstd.object = THPVariable_Wrap(t);
            if (!rstd.object) throw Failed();
        }
        const Checkpoint yc(a[8], "y_checkpoint", x.rows, x.cols), hc(a[10], "h_checkpoint", x.rows, x.cols);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_rms_norm(x.ptr, x.stride, residual.ptr, residual.stride, weight.data_ptr(), x.rows, x.cols, x.dtype, eps, h.ptr, y.ptr, yc.ptr(),
                                yc.codes.stride, yc.scales, coded_y, hc.ptr(), hc.codes.stride, hc.scales, static_cast<float *>(rstd.ptr), st);
        }), "gaf_rms_norm");
        return tuple_of(y, h, rstd);
    });
}

PyObject *py_rms_norm_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        // dy, h (a matrix or a checkpoint), weight, rstd, dweight, workspace, residual_grad, dx, base
        const Matrix dy(a[0], "dy");
        if (!dy.t) fail_value("dy", "is missing");
        const bool coded = PyTuple_Check(a[1]) || PyList_Check(a[1]);
        const Matrix h(coded ? Py_None : a[1], "h");
        if (!coded && !h.t) fail_value("h", "is missing");
        const Checkpoint hc(coded ? a[1] : Py_None, "h", dy.rows, dy.cols);
        same_shape(h, dy.rows, dy.cols, dy.dtype, "h");
        const at::Tensor &weight = dense(a[2], "weight", dy.cols);
        if (weight.scalar_type() != dy.t->scalar_type()) fail_value("weight", "has another type than dy");
        const at::Tensor &rstd = dense(a[3], "rstd", dy.rows);
        if (rstd.scalar_type() != at::kFloat) fail_value("rstd", "must be float32");
        const WeightGradient g(a[4], a[8], dy.cols, "dweight");
        const LayerWorkspace ws(a[5]);
        const Matrix residual_grad(a[6], "residual_grad");
        same_shape(residual_grad, dy.rows, dy.cols, dy.dtype, "residual_grad");
        const std::vector<int64_t> shape = shape_with(*dy.t, false, -1);
        LayerOutput dx(a[7], shape, dy.t->scalar_type(), dy.t->device(), "dx");
        void *const st = stream();
        check(without_gil([&] {
            return gaf_rms_norm_grad(dy.ptr, dy.stride, h.ptr, h.stride, hc.ptr(), hc.codes.stride, hc.scales, weight.data_ptr(),
                                     static_cast<const float *>(rstd.data_ptr()), residual_grad.ptr, residual_grad.stride, dy.rows, dy.cols, dy.dtype, dx.ptr,
                                     g.base, g.ptr, g.dtype, ws.ptr, ws.bytes, st);
        }), "gaf_rms_norm_grad");
        PyObject *const r = PyTuple_New(2);
        if (!r) throw Failed();
        PyTuple_SET_ITEM(r, 0, dx.take());
        PyTuple_SET_ITEM(r, 1, Py_NewRef(a[4]));
        return r;
    });
}

PyObject *py_checkpoint_pack(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 2, [&] {
        const Matrix x(a[0], "x");
        if (!x.t) fail_value("x", "is missing");
        const Checkpoint c(a[1], "checkpoint", x.rows, x.cols);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_checkpoint_pack(x.ptr, x.stride, x.rows, x.cols, x.dtype, c.ptr(), c.codes.stride, c.scales, st);
        }), "gaf_checkpoint_pack");
        return Py_NewRef(a[1]);
    });
}

PyObject *py_checkpoint_unpack(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 2, [&] {
        const Checkpoint c(a[0], "checkpoint");
        const Matrix out(a[1], "out");
        if (!out.t || !out.has(c.codes.rows, c.codes.cols)) fail_value("out", "has another shape than the checkpoint");
        void *const st = stream();
        check(without_gil([&] {
            return gaf_checkpoint_unpack(c.ptr(), c.codes.stride, c.scales, out.rows, out.cols, out.dtype, out.ptr, out.stride, st);
        }), "gaf_checkpoint_unpack");
        return Py_NewRef(a[1]);
    });
}

PyObject *py_linear_weight_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 5, [&] {
        // dy, checkpoint, dweight, workspace, base
        const Matrix dy(a[0], "dy");
        if (!dy.t) fail_value("dy", "is missing");
        const Checkpoint c(a[1], "checkpoint");
        if (!c.codes.t) fail_value("checkpoint", "is missing");
        if (c.codes.rows != dy.rows) fail_value("checkpoint", "must have as many rows as dy");
        const at::Tensor &dweight = cuda_tensor(a[2], "dweight");
        if (dweight.dim() != 2 || dweight.size(0) != dy.cols || dweight.size(1) != c.codes.cols)
            fail_value("dweight", "must be a matrix of dy's columns by the checkpoint's");
        const WeightGradient g(a[2], a[4], dweight.numel(), "dweight");
        const LayerWorkspace ws(a[3]);
        void *const st = stream();
        check(without_gil([&] {
            return gaf_linear_weight_grad(dy.ptr, dy.stride, dy.dtype, c.ptr(), c.codes.stride, c.scales, dy.rows, dy.cols, c.codes.cols, g.base, g.ptr, g.dtype,
                                          ws.ptr, ws.bytes, st);
        }), "gaf_linear_weight_grad");
        return Py_NewRef(a[2]);
    });
}

PyObject *py_register_error(PyObject *, PyObject *cls) {
    Py_XSETREF(g_error, Py_NewRef(cls));
    return Py_NewRef(Py_None);
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FAST(filter_accumulate), FAST(filter_accumulate_any_seed), FAST(filter_accumulate_bucketed), FAST(pairwise_cosdist),
    FAST(cosdist), FAST(stream_begin), FAST(stream_push), FAST(stream_end),
    FAST(embedding), FAST(embedding_grad), FAST(rms_norm), FAST(rms_norm_grad), FAST(checkpoint_pack), FAST(checkpoint_unpack),
    FAST(linear_weight_grad),
    {"register_error", py_register_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gaf_native", "Argument marshalling over the C ABI of gaf.h.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gaf_native(void) { return PyModule_Create(&module); }
