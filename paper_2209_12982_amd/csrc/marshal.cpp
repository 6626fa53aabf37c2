// Argument marshalling of the decoder operators for Python: checks that each
// tensor is what the C function needs (the C ABI sees plain addresses and
// cannot tell), and calls it.  The calls take a few microseconds on the GPU;
// the same checks written in Python take longer than that, so they are here.
// Nothing is computed and nothing is kept.  A tensor that does not fit raises
// ValueError; the C function's status is returned.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>

#include <initializer_list>
#include <sstream>
#include <string>

#include "winof4.h"

namespace {

struct Misfit {
    std::string what;
};

[[noreturn]] void misfit(const at::Tensor& t, const char* what, at::ScalarType type, std::initializer_list<int64_t> shape,
                         const char* why) {
    std::ostringstream s;
    s << what << ": expected " << why << c10::toString(type) << " [";
    const char* sep = "";
    for (const int64_t n : shape) s << sep << n, sep = ", ";
    s << "] on the GPU, got " << c10::toString(t.scalar_type()) << " " << t.sizes() << " on " << t.device();
    throw Misfit{s.str()};
}

bool fits(const at::Tensor& t, at::ScalarType type, std::initializer_list<int64_t> shape) {
    if (t.scalar_type() != type || t.dim() != (int64_t)shape.size()) return false;
    int64_t i = 0;
    for (const int64_t n : shape)
        if (t.size(i++) != n) return false;
    return true;
}

// The GPU that the call is launched on.  Every tensor has to be there: the stream is one of its streams, and gives no
// order against work on another.
struct Gpu {
    int64_t index;

    const at::Tensor& tensor(PyObject* o, const char* what) const {
        if (!THPVariable_Check(o)) throw Misfit{std::string(what) + ": expected a torch tensor on the GPU, got " + Py_TYPE(o)->tp_name};
        const at::Tensor& t = THPVariable_Unpack(o);
        const c10::Device d = t.device();
        if (!d.is_cuda() || d.index() != index) {
            std::ostringstream s;
            s << what << ": expected a tensor on the current GPU (" << index << "), got one on " << d;
            throw Misfit{s.str()};
        }
        return t;
    }

    // Address of a dense tensor of a type and shape.
    void* dense(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, const char* what) const {
        const at::Tensor& t = tensor(o, what);
        if (!fits(t, type, shape) || !t.is_contiguous()) misfit(t, what, type, shape, "dense ");
        return t.data_ptr();
    }
    void* dense_or_none(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, const char* what) const {
        return o == Py_None ? nullptr : dense(o, type, shape, what);
    }

    // Address and row stride of a tensor whose rows (all dimensions but the first) are dense; the rows may lie apart.
    void* rows(PyObject* o, at::ScalarType type, std::initializer_list<int64_t> shape, const char* what, int64_t* stride) const {
        const at::Tensor& t = tensor(o, what);
        if (!fits(t, type, shape)) misfit(t, what, type, shape, "");
        int64_t want = 1;
        for (int64_t i = t.dim() - 1; i > 0; --i) {
            if (t.size(i) > 1 && t.stride(i) != want) misfit(t, what, type, shape, "rows that are dense: ");
            want *= t.size(i);
        }
        *stride = t.size(0) > 1 ? t.stride(0) : want;
        return t.data_ptr();
    }

    // A workspace: any dense tensor, or None.
    void* scratch(PyObject* o, size_t* bytes) const {
        *bytes = 0;
        if (o == Py_None) return nullptr;
        const at::Tensor& t = tensor(o, "workspace");
        if (!t.is_contiguous()) throw Misfit{"workspace: expected a dense tensor"};
        *bytes = t.nbytes();
        return t.data_ptr();
    }

    kv4_cache cache(PyObject* o) const;
};

wino_float_type float_type(const at::Tensor& t, const char* what) {
    if (t.scalar_type() == at::kBFloat16) return WINO_BF16;
    if (t.scalar_type() == at::kHalf) return WINO_FP16;
    throw Misfit{std::string(what) + ": expected a bf16 or fp16 tensor"};
}

void dims(const at::Tensor& t, int64_t n, const char* what) {
    if (t.dim() != n) throw Misfit{std::string(what) + ": expected " + std::to_string(n) + " dimensions, got " + std::to_string(t.dim())};
}

int32_t fit32(int64_t n, const char* what) {
    if (n > 0x7fffffff) throw Misfit{std::string(what) + ": too many"};
    return (int32_t)n;
}

// (k_codes, k_scales, v_codes, v_scales)
kv4_cache Gpu::cache(PyObject* o) const {
    if ((!PyTuple_Check(o) && !PyList_Check(o)) || PySequence_Size(o) != 4)
        throw Misfit{"cache: expected (k_codes, k_scales, v_codes, v_scales)"};
    PyObject** c = PySequence_Fast_ITEMS(o);
    const at::Tensor& t = tensor(c[0], "k_codes");
    dims(t, 4, "k_codes");
    const int64_t pages = t.size(0), heads = t.size(1), page = t.size(2), half = t.size(3);
    kv4_cache k;
    k.k_codes = (uint8_t*)dense(c[0], at::kByte, {pages, heads, page, half}, "k_codes");
    k.k_scales = (uint8_t*)dense(c[1], at::kByte, {pages, heads, page, half / 16}, "k_scales");
    k.v_codes = (uint8_t*)dense(c[2], at::kByte, {pages, heads, page, half}, "v_codes");
    k.v_scales = (uint8_t*)dense(c[3], at::kByte, {pages, heads, page, half / 16}, "v_scales");
    k.pages = pages;
    k.kv_heads = fit32(heads, "heads of the cache");
    k.page_size = fit32(page, "tokens of a page");
    k.head_dim = fit32(2 * half, "dimensions of a head");
    return k;
}

long integer(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Misfit{""};
    return v;
}
int32_t small(PyObject* o, const char* what) {
    const long v = integer(o);
    if (v < -0x7fffffffl || v > 0x7fffffffl) throw Misfit{std::string(what) + ": out of range"};
    return (int32_t)v;
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Misfit{""};
    return (float)v;
}
hipStream_t stream_of(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Misfit{""};
    return (hipStream_t)p;
}

// Runs a call: its status, or the Python error for what it threw.
template <class F> PyObject* call(Py_ssize_t given, Py_ssize_t want, F f) {
    if (given != want) return PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, given);
    try {
        return PyLong_FromLong(f());
    } catch (const Misfit& m) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, m.what.c_str());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// x, codes, scales, y, bias, workspace, stream, device
PyObject* matvec(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 8, [&]() -> long {
        const Gpu gpu{integer(a[7])};
        const at::Tensor &x = gpu.tensor(a[0], "x"), &codes = gpu.tensor(a[1], "codes");
        dims(x, 2, "x");
        dims(codes, 2, "codes");
        const wino_float_type kind = float_type(x, "x");
        const at::ScalarType t = x.scalar_type();
        const int64_t m = x.size(0), k = x.size(1), n = codes.size(0);
        int64_t xs, ys;
        size_t bytes;
        const void* xp = gpu.rows(a[0], t, {m, k}, "x", &xs);
        const uint8_t* cp = (const uint8_t*)gpu.dense(a[1], at::kByte, {n, k / 2}, "codes");
        const uint8_t* sp = (const uint8_t*)gpu.dense(a[2], at::kByte, {n, k / 32}, "scales");
        void* yp = gpu.rows(a[3], t, {m, n}, "y", &ys);
        const void* bp = gpu.dense_or_none(a[4], t, {n}, "bias");
        void* ws = gpu.scratch(a[5], &bytes);
        const hipStream_t stream = stream_of(a[6]);
        return w4_matvec(xp, xs, cp, sp, bp, yp, ys, fit32(m, "rows of x"), fit32(n, "rows of the weights"),
                         fit32(k, "columns"), kind, ws, bytes, stream);
    });
}

// q, k, v, cos_sin, positions, slots, cache, q_out, k_out, v_out, rotary, values, stream, device
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 14, [&]() -> long {
        const Gpu gpu{integer(a[13])};
        const at::Tensor &k = gpu.tensor(a[1], "k"), &table = gpu.tensor(a[3], "cos_sin");
        dims(k, 3, "k");
        dims(table, 2, "cos_sin");
        const wino_float_type kind = float_type(k, "k");
        const at::ScalarType t = k.scalar_type();
        const kv4_cache c = gpu.cache(a[6]);
        const int64_t n = k.size(0), hkv = k.size(1), d = k.size(2);
        if (hkv != c.kv_heads || d != c.head_dim) throw Misfit{"k: other heads than the cache's"};
        int64_t qs = 0, ks, vs, hq = 0;
        const void* qp = nullptr;
        if ((a[0] == Py_None) != (a[7] == Py_None)) throw Misfit{"q and q_out go together"};
        if (a[0] != Py_None) {
            const at::Tensor& q = gpu.tensor(a[0], "q");
            dims(q, 3, "q");
            hq = q.size(1);
            qp = gpu.rows(a[0], t, {n, hq, d}, "q", &qs);
        }
        const void* kp = gpu.rows(a[1], t, {n, hkv, d}, "k", &ks);
        const void* vp = gpu.rows(a[2], t, {n, hkv, d}, "v", &vs);
        const int64_t length = table.size(0), rot = table.size(1);
        const float* cp = (const float*)gpu.dense(a[3], at::kFloat, {length, rot}, "cos_sin");
        const int32_t* pos = (const int32_t*)gpu.dense(a[4], at::kInt, {n}, "positions");
        const int64_t* slots = (const int64_t*)gpu.dense(a[5], at::kLong, {n}, "slots");
        void* qo = gpu.dense_or_none(a[7], t, {n, hq, d}, "q_out");
        void* ko = gpu.dense_or_none(a[8], t, {n, hkv, d}, "k_out");
        void* vo = gpu.dense_or_none(a[9], t, {n, hkv, d}, "v_out");
        return kv4_append(qp, qs, kp, ks, vp, vs, fit32(n, "tokens"), fit32(hq, "heads"), cp,
                          (int32_t)std::min<int64_t>(length, 0x7fffffff), fit32(rot, "columns of cos_sin"), pos, slots, &c, qo,
                          ko, vo, (wino_rotary)small(a[10], "rotary"), (kv4_values)small(a[11], "values"), kind,
                          stream_of(a[12]));
    });
}

// q, cache, block_table, lens, out, scale, workspace, stream, device
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 9, [&]() -> long {
        const Gpu gpu{integer(a[8])};
        const at::Tensor &q = gpu.tensor(a[0], "q"), &table = gpu.tensor(a[2], "block_table");
        dims(q, 3, "q");
        dims(table, 2, "block_table");
        const wino_float_type kind = float_type(q, "q");
        const at::ScalarType t = q.scalar_type();
        const kv4_cache c = gpu.cache(a[1]);
        const int64_t n = q.size(0), hq = q.size(1), d = q.size(2), batch = table.size(0), pages = table.size(1);
        if (d != c.head_dim || (batch ? n % batch : n)) throw Misfit{"q: rows or heads that do not go with the table or the cache"};
        int64_t qs;
        size_t bytes;
        const void* qp = gpu.rows(a[0], t, {n, hq, d}, "q", &qs);
        const int32_t* tp = (const int32_t*)gpu.dense(a[2], at::kInt, {batch, pages}, "block_table");
        const int32_t* lp = (const int32_t*)gpu.dense(a[3], at::kInt, {batch}, "lens");
        void* op = gpu.dense(a[4], t, {n, hq, d}, "out");
        const float scale = real(a[5]);
        void* ws = gpu.scratch(a[6], &bytes);
        return kv4_attention(qp, qs, &c, tp, fit32(pages, "pages"), lp, op, fit32(batch, "sequences"),
                             batch ? fit32(n / batch, "queries") : 0, fit32(hq, "heads"), scale, kind, ws, bytes,
                             stream_of(a[7]));
    });
}

// q, k, v, cu_q, cu_k, max_q, out, scale, causal, stream, device
PyObject* prompt(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 11, [&]() -> long {
        const Gpu gpu{integer(a[10])};
        const at::Tensor &q = gpu.tensor(a[0], "q"), &k = gpu.tensor(a[1], "k"), &cu = gpu.tensor(a[3], "cu_q");
        dims(q, 3, "q");
        dims(k, 3, "k");
        dims(cu, 1, "cu_q");
        const wino_float_type kind = float_type(q, "q");
        const at::ScalarType t = q.scalar_type();
        const int64_t nq = q.size(0), hq = q.size(1), d = q.size(2), nk = k.size(0), hkv = k.size(1), ends = cu.size(0);
        int64_t qs, ks, vs;
        const void* qp = gpu.rows(a[0], t, {nq, hq, d}, "q", &qs);
        const void* kp = gpu.rows(a[1], t, {nk, hkv, d}, "k", &ks);
        const void* vp = gpu.rows(a[2], t, {nk, hkv, d}, "v", &vs);
        const int32_t* cq = (const int32_t*)gpu.dense(a[3], at::kInt, {ends}, "cu_q");
        const int32_t* ck = (const int32_t*)gpu.dense(a[4], at::kInt, {ends}, "cu_k");
        const int32_t max_q = small(a[5], "max_q");
        void* op = gpu.dense(a[6], t, {nq, hq, d}, "out");
        const float scale = real(a[7]);
        const int causal = PyObject_IsTrue(a[8]);
        if (causal < 0) throw Misfit{""};
        return prompt_attention(qp, qs, kp, ks, vp, vs, cq, ck, fit32(ends > 0 ? ends - 1 : 0, "sequences"), fit32(nq, "queries"),
                                fit32(nk, "keys"), max_q, fit32(hq, "heads"), fit32(hkv, "heads"), fit32(d, "dimensions"), scale,
                                causal, op, kind, stream_of(a[9]));
    });
}

// x, codes, scales, stream, device
PyObject* quantize8(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 5, [&]() -> long {
        const Gpu gpu{integer(a[4])};
        const at::Tensor& x = gpu.tensor(a[0], "x");
        dims(x, 2, "x");
        const wino_float_type kind = float_type(x, "x");
        const int64_t m = x.size(0), k = x.size(1);
        int64_t xs;
        const void* xp = gpu.rows(a[0], x.scalar_type(), {m, k}, "x", &xs);
        int8_t* cp = (int8_t*)gpu.dense(a[1], at::kChar, {m, k}, "codes");
        float* sp = (float*)gpu.dense(a[2], at::kFloat, {m}, "scales");
        return w8_quantize(xp, xs, cp, sp, fit32(m, "rows of x"), fit32(k, "columns"), kind, stream_of(a[3]));
    });
}

// x, x_scales, w, w_scales, y, bias, workspace, stream, device
PyObject* matmul8(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 9, [&]() -> long {
        const Gpu gpu{integer(a[8])};
        const at::Tensor &x = gpu.tensor(a[0], "x"), &w = gpu.tensor(a[2], "w"), &y = gpu.tensor(a[4], "y");
        dims(x, 2, "x");
        dims(w, 2, "w");
        const wino_float_type kind = float_type(y, "y");
        const int64_t m = x.size(0), k = x.size(1), n = w.size(0);
        int64_t xs, ys;
        size_t bytes;
        const int8_t* xp = (const int8_t*)gpu.rows(a[0], at::kChar, {m, k}, "x", &xs);
        const float* sp = (const float*)gpu.dense(a[1], at::kFloat, {m}, "x_scales");
        const int8_t* wp = (const int8_t*)gpu.dense(a[2], at::kChar, {n, k}, "w");
        const float* tp = (const float*)gpu.dense(a[3], at::kFloat, {n}, "w_scales");
        void* yp = gpu.rows(a[4], y.scalar_type(), {m, n}, "y", &ys);
        const void* bp = gpu.dense_or_none(a[5], y.scalar_type(), {n}, "bias");
        void* ws = gpu.scratch(a[6], &bytes);
        return w8_matmul(xp, xs, sp, wp, tp, bp, yp, ys, fit32(m, "rows of x"), fit32(n, "rows of the weights"), fit32(k, "columns"),
                         kind, ws, bytes, stream_of(a[7]));
    });
}

// logits, chosen, weights, order, ends, bias, score, groups, top_groups, group_best, normalise, scale, live, workspace,
// stream, device
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 16, [&]() -> long {
        const Gpu gpu{integer(a[15])};
        const at::Tensor &logits = gpu.tensor(a[0], "logits"), &chosen = gpu.tensor(a[1], "chosen");
        dims(logits, 2, "logits");
        dims(chosen, 2, "chosen");
        const wino_float_type kind = logits.scalar_type() == at::kFloat ? WINO_FP32 : float_type(logits, "logits");
        const int64_t tokens = logits.size(0), experts = logits.size(1), top = chosen.size(1);
        int64_t stride;
        size_t bytes;
        const void* lp = gpu.rows(a[0], logits.scalar_type(), {tokens, experts}, "logits", &stride);
        int32_t* cp = (int32_t*)gpu.dense(a[1], at::kInt, {tokens, top}, "chosen");
        float* wp = (float*)gpu.dense(a[2], at::kFloat, {tokens, top}, "weights");
        if ((a[3] == Py_None) != (a[4] == Py_None)) throw Misfit{"order and ends go together"};
        int32_t* op = (int32_t*)gpu.dense_or_none(a[3], at::kInt, {tokens * top}, "order");
        int32_t* ep = (int32_t*)gpu.dense_or_none(a[4], at::kInt, {experts + 1}, "ends");
        const float* bp = (const float*)gpu.dense_or_none(a[5], at::kFloat, {experts}, "bias");
        const int normalise = PyObject_IsTrue(a[10]);
        if (normalise < 0) throw Misfit{""};
        const float scale = real(a[11]);
        const int32_t* vp = (const int32_t*)gpu.dense_or_none(a[12], at::kInt, {1}, "live");
        void* ws = gpu.scratch(a[13], &bytes);
        return route_experts(lp, stride, bp, fit32(tokens, "tokens"), fit32(experts, "experts"), fit32(top, "experts of a token"),
                             (wino_score)small(a[6], "score"), small(a[7], "groups"), small(a[8], "top_groups"),
                             small(a[9], "group_best"), normalise, scale, vp, cp, wp, op, ep, kind, ws, bytes, stream_of(a[14]));
    });
}

// x, x_scales, w, w_scales, order, ends, y, chosen, weights, workspace, stream, device
PyObject* experts8(PyObject*, PyObject* const* a, Py_ssize_t given) {
    return call(given, 12, [&]() -> long {
        const Gpu gpu{integer(a[11])};
        const at::Tensor &x = gpu.tensor(a[0], "x"), &w = gpu.tensor(a[2], "w"), &order = gpu.tensor(a[4], "order"),
                         &y = gpu.tensor(a[6], "y");
        dims(x, 2, "x");
        dims(w, 3, "w");
        dims(order, 1, "order");
        const wino_float_type kind = float_type(y, "y");
        const int64_t x_rows = x.size(0), k = x.size(1), experts = w.size(0), n = w.size(1), routes = order.size(0);
        if ((a[7] == Py_None) != (a[8] == Py_None)) throw Misfit{"chosen and weights go together"};
        int64_t top = 1, xs, ys;
        const int32_t* cp = nullptr;
        const float* gp = nullptr;
        if (a[8] != Py_None) {
            const at::Tensor& weights = gpu.tensor(a[8], "weights");
            dims(weights, 2, "weights");
            top = weights.size(1);
            if (weights.numel() != routes) throw Misfit{"weights: as many as routes in the order are expected"};
            gp = (const float*)gpu.dense(a[8], at::kFloat, {weights.size(0), top}, "weights");
            cp = (const int32_t*)gpu.dense(a[7], at::kInt, {weights.size(0), top}, "chosen");
        }
        if (x_rows ? routes % x_rows : routes) throw Misfit{"x: a row for each token or for each route is expected"};
        size_t bytes;
        const int8_t* xp = (const int8_t*)gpu.rows(a[0], at::kChar, {x_rows, k}, "x", &xs);
        const float* sp = (const float*)gpu.dense(a[1], at::kFloat, {x_rows}, "x_scales");
        const int8_t* wp = (const int8_t*)gpu.dense(a[2], at::kChar, {experts, n, k}, "w");
        const float* tp = (const float*)gpu.dense(a[3], at::kFloat, {experts, n}, "w_scales");
        const int32_t* op = (const int32_t*)gpu.dense(a[4], at::kInt, {routes}, "order");
        const int32_t* ep = (const int32_t*)gpu.dense(a[5], at::kInt, {experts + 1}, "ends");
        void* yp = gpu.rows(a[6], y.scalar_type(), {top ? routes / top : 0, n}, "y", &ys);
        void* ws = gpu.scratch(a[9], &bytes);
        return w8_experts_matmul(xp, xs, sp, fit32(x_rows, "rows of x"), wp, tp, op, ep, fit32(routes, "routes"),
                                 fit32(experts, "experts"), cp, gp, fit32(top, "experts of a token"), yp, ys,
                                 fit32(n, "rows of the weights"), fit32(k, "columns"), kind, ws, bytes, stream_of(a[10]));
    });
}

PyMethodDef methods[] = {
    {"w4_matvec", (PyCFunction)(void (*)())matvec, METH_FASTCALL, nullptr},
    {"kv4_append", (PyCFunction)(void (*)())append, METH_FASTCALL, nullptr},
    {"kv4_attention", (PyCFunction)(void (*)())attention, METH_FASTCALL, nullptr},
    {"prompt_attention", (PyCFunction)(void (*)())prompt, METH_FASTCALL, nullptr},
    {"w8_quantize", (PyCFunction)(void (*)())quantize8, METH_FASTCALL, nullptr},
    {"w8_matmul", (PyCFunction)(void (*)())matmul8, METH_FASTCALL, nullptr},
    {"route_experts", (PyCFunction)(void (*)())route, METH_FASTCALL, nullptr},
    {"w8_experts_matmul", (PyCFunction)(void (*)())experts8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the decoder operators.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
