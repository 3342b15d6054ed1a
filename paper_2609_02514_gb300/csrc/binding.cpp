// The calls of the 4-bit KV cache for Python, as one native step each: the
// arguments' checks, the outputs' allocation and the C entry point.  A call on one
// token is bound by the host, and in Python these steps took 12 us (kv4_read) to
// 19 us (kv4_attention) of a Grace core.  The C entry points come as addresses, so
// the module serves the product library and the checked one.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>

#include "../../include/acespec.h"

namespace {

using at::Tensor;
using Shape = std::initializer_list<int64_t>;

struct Refusal {
    std::string why;
};

std::string text(const Shape &s) {
    std::string t = "[";
    for (int64_t x : s) t += (t.size() > 1 ? ", " : "") + std::to_string(x);
    return t + "]";
}

const Tensor &cuda(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw Refusal{std::string(name) + " must be a CUDA tensor"};
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) throw Refusal{std::string(name) + " must be a CUDA tensor"};
    return t;
}

// a dense tensor of a type and shape on the cache's device
void *dense(PyObject *o, const char *name, Shape shape, at::ScalarType type, const Tensor &cache) {
    const Tensor &t = cuda(o, name);
    if (t.scalar_type() != type || t.sizes() != at::IntArrayRef(shape) || t.device() != cache.device() || !t.is_contiguous())
        throw Refusal{std::string(name) + " must be a contiguous " + c10::toString(type) + " " + text(shape) + " on " +
                      cache.device().str()};
    return t.data_ptr();
}

struct Cache {
    const Tensor &t;
    int planes, B, H, S, D;
};
Cache cache_of(PyObject *o) {
    const Tensor &t = cuda(o, "cache");
    if (t.scalar_type() != at::kByte || t.dim() != 5 || !t.is_contiguous())
        throw Refusal{"cache must be a contiguous uint8 [planes, B, H, S, row]"};
    for (int i = 0; i < 5; ++i)
        if (t.size(i) > INT32_MAX) throw Refusal{"cache has a dimension above 2^31"};
    return {t, (int)t.size(0), (int)t.size(1), (int)t.size(2), (int)t.size(3), 2 * ((int)t.size(4) - 16)};
}

// [B, n, heads, D] numbers whose last dimension is dense
const Tensor &rows(PyObject *o, const char *name, const Cache &c, int64_t (&strides)[3]) {
    const Tensor &t = cuda(o, name);
    if (t.dim() != 4 || (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16))
        throw Refusal{std::string(name) + " must be float32 or bfloat16 [B, n, heads, D]"};
    if ((t.stride(3) != 1 && t.size(3) != 1) || t.device() != c.t.device())
        throw Refusal{std::string(name) + " must have a dense last dimension and lie on " + c.t.device().str()};
    if (t.size(0) != c.B || t.size(3) != c.D || t.size(1) > INT32_MAX || t.size(2) > INT32_MAX)
        throw Refusal{std::string(name) + " must be [" + std::to_string(c.B) + ", n, heads, " + std::to_string(c.D) + "]"};
    for (int i = 0; i < 3; ++i) strides[i] = t.stride(i);
    return t;
}
aces_dtype code(at::ScalarType t) { return t == at::kFloat ? ACES_F32 : ACES_BF16; }

long long whole(PyObject *o) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Refusal{""};
    return x;
}
int integer(PyObject *o, const char *name) {
    const long long x = whole(o);
    if (x > INT32_MAX || x < INT32_MIN) throw Refusal{std::string(name) + " is out of range"};
    return (int)x;
}
void *address(PyObject *o) { return reinterpret_cast<void *>((uintptr_t)whole(o)); }

// One output: the caller's object, or a tensor made here, which only becomes an object
// on the way back to Python, so that what fails in between gives it back.
struct Output {
    PyObject *given = nullptr;
    Tensor made;
    void *p = nullptr;
    void take(PyObject *o, const char *name, Shape shape, at::ScalarType type, const Tensor &cache) {
        if (o != Py_None) given = o, p = dense(o, name, shape, type, cache);
    }
    void make(Shape shape, at::ScalarType type, const Tensor &cache) {
        if (given) return;
        made = at::empty(shape, cache.options().dtype(type));
        p = made.data_ptr();
    }
    PyObject *object() const {
        if (!given) return THPVariable_Wrap(made);
        Py_INCREF(given);
        return given;
    }
};

// Runs f, and turns what it throws into a Python error.
template <typename F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F f) {
    if (have != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (const Refusal &r) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, r.why.c_str());
    } catch (...) {  // torch's own kinds stay what they are (out of memory, for one)
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

using Append = decltype(&aces_kv4_append);
using Read = decltype(&aces_kv4_read);
using Attention = decltype(&aces_kv4_attention);
using Bytes = decltype(&aces_kv4_workspace_bytes);

// append(entry, cache, layer, k, v, start, count, out, stream) -> (status code, row_status)
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 9, [&]() -> PyObject * {
        const Cache c = cache_of(a[1]);
        int64_t ks[3], vs[3];
        const Tensor &k = rows(a[3], "k", c, ks), &v = rows(a[4], "v", c, vs);
        if (k.size(2) != c.H || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
            throw Refusal{"k and v must be alike, [" + std::to_string(c.B) + ", n, " + std::to_string(c.H) + ", " + std::to_string(c.D) + "]"};
        const int n = (int)k.size(1), layer = integer(a[2], "layer");
        const auto entry = reinterpret_cast<Append>(address(a[0]));
        const auto stream = (aces_stream_t)address(a[8]);
        const void *start = dense(a[5], "start", {c.B}, at::kInt, c.t);
        const void *count = a[6] == Py_None ? nullptr : dense(a[6], "count", {c.B}, at::kInt, c.t);
        Output st;
        st.take(a[7], "out", {c.B, n}, at::kInt, c.t);
        st.make({c.B, n}, at::kInt, c.t);
        const aces_status s = entry(c.t.data_ptr(), c.planes, layer, c.B, c.H, c.S, c.D, k.data_ptr(), v.data_ptr(), code(k.scalar_type()), ks,
                                    vs, (const int32_t *)start, (const int32_t *)count, n, (int32_t *)st.p, stream);
        return Py_BuildValue("(iN)", (int)s, st.object());
    });
}

// read(entry, cache, layer, start, n, float32, k, v, stream) -> (status code, k, v)
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 9, [&]() -> PyObject * {
        const Cache c = cache_of(a[1]);
        const int n = integer(a[4], "n"), layer = integer(a[2], "layer");
        const auto entry = reinterpret_cast<Read>(address(a[0]));
        const auto stream = (aces_stream_t)address(a[8]);
        const at::ScalarType type = a[5] == Py_True ? at::kFloat : at::kBFloat16;
        const void *start = dense(a[3], "start", {c.B}, at::kInt, c.t);
        if (n < 1) return Py_BuildValue("(iOO)", (int)ACES_ERR_INVALID_ARG, Py_None, Py_None);
        Output out[2];
        for (int x = 0; x < 2; ++x) out[x].take(a[6 + x], x ? "v" : "k", {c.B, n, c.H, c.D}, type, c.t);
        for (int x = 0; x < 2; ++x) out[x].make({c.B, n, c.H, c.D}, type, c.t);
        const aces_status s = entry(c.t.data_ptr(), c.planes, layer, c.B, c.H, c.S, c.D, (const int32_t *)start, n, out[0].p, out[1].p, code(type),
                                    stream);
        return Py_BuildValue("(iNN)", (int)s, out[0].object(), out[1].object());
    });
}

// attention(entry, workspace_bytes, q, cache, layer, prefix_len, mask, depth, count, scale, window, sinks, out, lse, status,
//           workspace, stream) -> (status code, out, lse, status)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 17, [&]() -> PyObject * {
        const Cache c = cache_of(a[3]);
        int64_t qs[3];
        const Tensor &q = rows(a[2], "q", c, qs);
        const int n = (int)q.size(1), Hq = (int)q.size(2), words = (n + 31) / 32;
        const void *prefix = dense(a[5], "prefix_len", {c.B}, at::kInt, c.t);
        const void *mask = nullptr, *depth = nullptr;
        int64_t ms = 0, ds = 0;
        if ((a[6] == Py_None) != (a[7] == Py_None)) throw Refusal{"mask and depth go together"};
        if (a[6] != Py_None) {
            if (cuda(a[6], "mask").dim() == 3)
                mask = dense(a[6], "mask", {c.B, n, words}, at::kInt, c.t), ms = (int64_t)n * words;
            else
                mask = dense(a[6], "mask", {n, words}, at::kInt, c.t);
            if (cuda(a[7], "depth").dim() == 2)
                depth = dense(a[7], "depth", {c.B, n}, at::kInt, c.t), ds = n;
            else
                depth = dense(a[7], "depth", {n}, at::kInt, c.t);
        }
        const void *count = a[8] == Py_None ? nullptr : dense(a[8], "count", {c.B}, at::kInt, c.t);
        double scale = 1.0 / std::sqrt((double)(c.D > 0 ? c.D : 1));
        if (a[9] != Py_None) {
            scale = PyFloat_AsDouble(a[9]);
            if (scale == -1.0 && PyErr_Occurred()) throw Refusal{""};
        }
        const Shape full{c.B, n, Hq, c.D}, row{c.B, n, Hq}, one{c.B};
        Output out, lse, status;
        out.take(a[12], "out", full, q.scalar_type(), c.t);
        lse.take(a[13], "lse", row, at::kFloat, c.t);
        status.take(a[14], "status", one, at::kInt, c.t);
        const int layer = integer(a[4], "layer"), window = integer(a[10], "window"), sinks = integer(a[11], "sinks");
        const auto entry = reinterpret_cast<Attention>(address(a[0]));
        const auto stream = (aces_stream_t)address(a[16]);
        // The workspace is the call's own: given back on return, it is only used again
        // behind the call's work on this stream.
        Tensor scratch;
        if (a[15] == Py_None) {
            const size_t need = reinterpret_cast<Bytes>(address(a[1]))(c.B, n, Hq, c.H, c.D);
            scratch = at::empty({(int64_t)std::max<size_t>(need, 16)}, c.t.options());
        } else {
            scratch = cuda(a[15], "workspace");
            if (!scratch.is_contiguous() || scratch.device() != c.t.device())
                throw Refusal{"workspace must be contiguous and on " + c.t.device().str()};
        }
        void *ws = scratch.data_ptr();
        const size_t bytes = scratch.nbytes();
        out.make(full, q.scalar_type(), c.t);
        lse.make(row, at::kFloat, c.t);
        status.make(one, at::kInt, c.t);
        const aces_status s = entry(
            q.data_ptr(), code(q.scalar_type()), qs, c.t.data_ptr(), c.planes, layer, c.B, n, Hq, c.H, c.S, c.D, (const int32_t *)prefix,
            (const int32_t *)count, (const uint32_t *)mask, ms, (const int32_t *)depth, ds, (float)scale, window, sinks, out.p, (float *)lse.p,
            (int32_t *)status.p, ws, bytes, stream);
        return Py_BuildValue("(iNNN)", (int)s, out.object(), lse.object(), status.object());
    });
}

PyMethodDef methods[] = {{"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL, nullptr},
                         {"read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(read)), METH_FASTCALL, nullptr},
                         {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attention)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
