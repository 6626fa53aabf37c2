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

PyMethodDef methods[] = {
    {"w4_matvec", (PyCFunction)(void (*)())matvec, METH_FASTCALL, nullptr},
    {"kv4_append", (PyCFunction)(void (*)())append, METH_FASTCALL, nullptr},
    {"kv4_attention", (PyCFunction)(void (*)())attention, METH_FASTCALL, nullptr},
    {"prompt_attention", (PyCFunction)(void (*)())prompt, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the decoder operators.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
