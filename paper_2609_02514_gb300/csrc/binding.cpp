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

// A caller's tensor that the call has written: as an object once more.  Its version goes
// up, so that autograd does not take what it saved of it before for its numbers.
PyObject *written(PyObject *o) {
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    Py_INCREF(o);
    return o;
}

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
        return given ? written(given) : THPVariable_Wrap(made);
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

using SharedAttention = decltype(&aces_kv4_shared_attention);
using SharedBytes = decltype(&aces_kv4_shared_workspace_bytes);

// attention(entry, workspace_bytes, q, cache, layer, prefix_len, mask, depth, count, scale, window, sinks, out, lse, status,
//           workspace, stream) -> (status code, out, lse, status); with two more, shared and shared_len, behind prefixes
PyObject *attend(PyObject *const *a, Py_ssize_t n_args, bool behind) {
    return guarded(n_args, behind ? 19 : 17, [&]() -> PyObject * {
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
        const auto stream = (aces_stream_t)address(a[16]);
        Cache p = c;
        const void *shared_len = nullptr;
        if (behind) {
            const Tensor &t = cuda(a[17], "shared");
            if (t.device() != c.t.device()) throw Refusal{"shared must lie on " + c.t.device().str()};
            if (t.scalar_type() != at::kByte || t.dim() != 5 || !t.is_contiguous() || t.size(2) != c.H || t.size(4) != c.t.size(4) || t.size(1) < 1 ||
                c.B % t.size(1) != 0 || t.size(0) > INT32_MAX || t.size(3) > INT32_MAX)
                throw Refusal{"shared must be a contiguous uint8 [planes, groups, " + std::to_string(c.H) + ", S0, " + std::to_string(c.t.size(4)) +
                              "], and the batch a multiple of groups"};
            p.planes = (int)t.size(0), p.B = (int)t.size(1), p.S = (int)t.size(3);
            shared_len = dense(a[18], "shared_len", {p.B}, at::kInt, c.t);
        }
        // The workspace is the call's own: given back on return, it is only used again
        // behind the call's work on this stream.
        Tensor scratch;
        if (a[15] == Py_None) {
            const size_t need = behind ? reinterpret_cast<SharedBytes>(address(a[1]))(c.B, p.B, n, Hq, c.H, c.D)
                                       : reinterpret_cast<Bytes>(address(a[1]))(c.B, n, Hq, c.H, c.D);
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
        const aces_status s =
            behind ? reinterpret_cast<SharedAttention>(address(a[0]))(
                         q.data_ptr(), code(q.scalar_type()), qs, cuda(a[17], "shared").data_ptr(), p.planes, p.B, p.S, (const int32_t *)shared_len,
                         c.t.data_ptr(), c.planes, layer, c.B, n, Hq, c.H, c.S, c.D, (const int32_t *)prefix, (const int32_t *)count,
                         (const uint32_t *)mask, ms, (const int32_t *)depth, ds, (float)scale, window, sinks, out.p, (float *)lse.p,
                         (int32_t *)status.p, ws, bytes, stream)
                   : reinterpret_cast<Attention>(address(a[0]))(
                         q.data_ptr(), code(q.scalar_type()), qs, c.t.data_ptr(), c.planes, layer, c.B, n, Hq, c.H, c.S, c.D, (const int32_t *)prefix,
                         (const int32_t *)count, (const uint32_t *)mask, ms, (const int32_t *)depth, ds, (float)scale, window, sinks, out.p,
                         (float *)lse.p, (int32_t *)status.p, ws, bytes, stream);
        return Py_BuildValue("(iNNN)", (int)s, out.object(), lse.object(), status.object());
    });
}

PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n_args) { return attend(a, n_args, false); }
PyObject *shared_attention(PyObject *, PyObject *const *a, Py_ssize_t n_args) { return attend(a, n_args, true); }

using Rotate = decltype(&aces_rotate_qk);
using AppendRotated = decltype(&aces_kv4_append_rotated);

double real(PyObject *o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Refusal{""};
    return x;
}
// heads [B, n, heads, D] of a type on a device, the last dimension dense
struct Heads {
    void *p = nullptr;
    PyObject *given = nullptr;
    Tensor made;
    int64_t stride[3];
    void take(PyObject *o, const char *name, const Tensor &q, int64_t n_heads) {
        const Tensor &t = cuda(o, name);
        if (t.scalar_type() != q.scalar_type() || t.dim() != 4 || t.device() != q.device() || t.size(0) != q.size(0) || t.size(1) != q.size(1) ||
            (n_heads >= 0 && t.size(2) != n_heads) || t.size(2) > INT32_MAX || t.size(3) != q.size(3))
            throw Refusal{std::string(name) + " must be a " + c10::toString(q.scalar_type()) + " [" + std::to_string(q.size(0)) + ", " +
                          std::to_string(q.size(1)) + ", " + (n_heads < 0 ? "heads" : std::to_string(n_heads)) + ", " + std::to_string(q.size(3)) +
                          "] on " + q.device().str()};
        if (t.stride(3) != 1 && t.size(3) != 1) throw Refusal{std::string(name) + " must have a dense last dimension"};
        given = o, p = t.data_ptr();
        for (int i = 0; i < 3; ++i) stride[i] = t.stride(i);
    }
    // an output: the caller's (`in` itself, or something that does not overlap it) or a new one
    void put(PyObject *o, const char *name, const Tensor &q, const Heads &in, int64_t n_heads) {
        if (o != Py_None) {
            take(o, name, q, n_heads);
            if (p == in.p && !std::equal(stride, stride + 3, in.stride)) throw Refusal{std::string(name) + " overlaps its input in another layout"};
            return;
        }
        made = at::empty({q.size(0), q.size(1), n_heads, q.size(3)}, q.options());
        p = made.data_ptr();
        for (int i = 0; i < 3; ++i) stride[i] = made.stride(i);
    }
    PyObject *object() const {
        return given ? written(given) : THPVariable_Wrap(made);
    }
};
const Tensor &queries(PyObject *o) {
    const Tensor &q = cuda(o, "q");
    if (q.dim() != 4 || (q.scalar_type() != at::kFloat && q.scalar_type() != at::kBFloat16))
        throw Refusal{"q must be float32 or bfloat16 [B, n, heads, D]"};
    for (int i = 0; i < 4; ++i)
        if (q.size(i) > INT32_MAX) throw Refusal{"q has a dimension above 2^31"};
    return q;
}
// a[0..10]: inv_freq, start, base, depth, positions, axes, q_weight, k_weight, eps, interleaved, scale
aces_turn turn_of(PyObject *const *a, const Tensor &q, int64_t Hq, int64_t H) {
    const int64_t B = q.size(0), n = q.size(1), D = q.size(3);
    aces_turn t = {};
    const Tensor &f = cuda(a[0], "inv_freq");
    if (f.dim() != 1 || f.size(0) > D / 2) throw Refusal{"inv_freq must be float32 [R / 2] with R at most " + std::to_string(D)};
    t.inv_freq = (const float *)dense(a[0], "inv_freq", {f.size(0)}, at::kFloat, q);
    t.rot_dim = 2 * (int)f.size(0);
    if (a[1] != Py_None) t.start = (const int32_t *)dense(a[1], "start", {B}, at::kInt, q);
    if (a[2] != Py_None) t.base = (const int32_t *)dense(a[2], "base", {B}, at::kInt, q);
    if (a[3] != Py_None) {
        if (cuda(a[3], "depth").dim() == 2)
            t.depth = (const int32_t *)dense(a[3], "depth", {B, n}, at::kInt, q), t.depth_stride = n;
        else
            t.depth = (const int32_t *)dense(a[3], "depth", {n}, at::kInt, q);
    }
    t.n_axes = 1;
    if (a[4] != Py_None) {
        const Tensor &p = cuda(a[4], "positions");
        if (p.dim() == 3) {
            if (p.size(0) < 1 || p.size(0) > ACES_MAX_AXES) throw Refusal{"positions must have 1 to " + std::to_string(ACES_MAX_AXES) + " axes"};
            t.n_axes = (int)p.size(0);
            t.positions = (const int32_t *)dense(a[4], "positions", {t.n_axes, B, n}, at::kInt, q);
        } else {
            t.positions = (const int32_t *)dense(a[4], "positions", {B, n}, at::kInt, q);
        }
        if (a[2] != Py_None || a[3] != Py_None) throw Refusal{"positions stand for base and depth, not beside them"};
    }
    if (a[5] != Py_None) t.axes = (const int32_t *)dense(a[5], "axes", {f.size(0)}, at::kInt, q);
    if (t.n_axes > 1 && !t.axes) throw Refusal{"positions of several axes need axes"};
    for (int i = 0; i < 2; ++i) {
        if (a[6 + i] == Py_None) continue;
        const char *name = i ? "k_weight" : "q_weight";
        const Tensor &w = cuda(a[6 + i], name);
        if (w.scalar_type() != at::kFloat && w.scalar_type() != at::kBFloat16) throw Refusal{std::string(name) + " must be float32 or bfloat16"};
        const bool each = w.dim() == 2;
        const void *p = each ? dense(a[6 + i], name, {i ? H : Hq, D}, w.scalar_type(), q) : dense(a[6 + i], name, {D}, w.scalar_type(), q);
        (i ? t.k_weight : t.q_weight) = p;
        (i ? t.k_weight_dt : t.q_weight_dt) = code(w.scalar_type());
        (i ? t.k_weight_stride : t.q_weight_stride) = each ? D : 0;
        if (a[8] == Py_None) throw Refusal{std::string(name) + " goes with eps"};
    }
    if (a[8] != Py_None) t.norm = 1, t.eps = real(a[8]);
    const int turned = PyObject_IsTrue(a[9]);
    if (turned < 0) throw Refusal{""};
    t.interleaved = turned;
    t.scale = real(a[10]);
    return t;
}

// rotate(entry, q, k, the eleven of turn_of, q_out, k_out, stream) -> (status code, q, k)
PyObject *rotate(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 17, [&]() -> PyObject * {
        const Tensor &q = queries(a[1]);
        Heads in[2], out[2];
        in[0].take(a[1], "q", q, -1);
        in[1].take(a[2], "k", q, -1);
        const int64_t Hq = q.size(2), H = cuda(a[2], "k").size(2);
        const aces_turn t = turn_of(a + 3, q, Hq, H);
        if (!t.positions && !t.start) throw Refusal{"start or positions must be given"};
        const auto entry = reinterpret_cast<Rotate>(address(a[0]));
        const auto stream = (aces_stream_t)address(a[16]);
        out[0].put(a[14], "q of out", q, in[0], Hq);
        out[1].put(a[15], "k of out", q, in[1], H);
        const aces_status s = entry(in[0].p, in[1].p, code(q.scalar_type()), in[0].stride, in[1].stride, (int)q.size(0), (int)q.size(1), (int)Hq,
                                    (int)H, (int)q.size(3), &t, out[0].p, out[1].p, out[0].stride, out[1].stride, stream);
        return Py_BuildValue("(iNN)", (int)s, out[0].object(), out[1].object());
    });
}

// append_rotated(entry, cache, layer, q, k, v, start, count, the eleven of turn_of, q_out, status, stream) -> (status code, q, status)
PyObject *append_rotated(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
    return guarded(n_args, 22, [&]() -> PyObject * {
        const Cache c = cache_of(a[1]);
        const Tensor &q = queries(a[3]);
        if (q.device() != c.t.device() || q.size(0) != c.B || q.size(3) != c.D)
            throw Refusal{"q must be [" + std::to_string(c.B) + ", n, heads, " + std::to_string(c.D) + "] on " + c.t.device().str()};
        Heads in[3], out;
        in[0].take(a[3], "q", q, -1);
        in[1].take(a[4], "k", q, c.H);
        in[2].take(a[5], "v", q, c.H);
        const int64_t Hq = q.size(2);
        const int n = (int)q.size(1), layer = integer(a[2], "layer");
        const void *start = dense(a[6], "start", {c.B}, at::kInt, c.t);
        const void *count = a[7] == Py_None ? nullptr : dense(a[7], "count", {c.B}, at::kInt, c.t);
        const aces_turn t = turn_of(a + 8, q, Hq, c.H);
        const auto entry = reinterpret_cast<AppendRotated>(address(a[0]));
        const auto stream = (aces_stream_t)address(a[21]);
        Output st;
        st.take(a[20], "status of out", {c.B, n}, at::kInt, c.t);
        out.put(a[19], "q of out", q, in[0], Hq);
        st.make({c.B, n}, at::kInt, c.t);
        const aces_status s = entry(c.t.data_ptr(), c.planes, layer, c.B, c.H, c.S, c.D, in[0].p, in[1].p, in[2].p, code(q.scalar_type()),
                                    in[0].stride, in[1].stride, in[2].stride, (int)Hq, (const int32_t *)start, (const int32_t *)count, n, &t, out.p,
                                    out.stride, (int32_t *)st.p, stream);
        return Py_BuildValue("(iNN)", (int)s, out.object(), st.object());
    });
}

PyMethodDef methods[] = {{"shared_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(shared_attention)), METH_FASTCALL, nullptr},
                         {"rotate", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotate)), METH_FASTCALL, nullptr},
                         {"append_rotated", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append_rotated)), METH_FASTCALL, nullptr},
                         {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append)), METH_FASTCALL, nullptr},
                         {"read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(read)), METH_FASTCALL, nullptr},
                         {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attention)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
