// Python module _paged_binding: the marshalling of the paged-cache calls (addresses, sizes and strides of tensors into
// the C ABI of include/emb_paged.h), for calls that are made once per layer on steps of a few microseconds: through ctypes
// an emb_qk_norm_rope of one token took 8.5 us of the host, the launch itself 2.
//
// Each function takes its tensors (None where the ABI takes NULL, a plain address where no size is read from it) and the plain
// values behind them, and returns the status, or a sentence if a tensor is not what the call would take it for: the ABI sees
// addresses and a few sizes only, so a shorter or strided tensor would be read and written beyond its elements. Looking them
// over takes 0.5 to 1.3 us of the host (a call of emb_paged_slots with its ten tensors 3.8 -> 5.1, of emb_qk_norm_rope
// 5.7 -> 6.5). bind() is given the addresses of the library's entry points first.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdio>

#include "../../include/emb_paged.h"

namespace {

decltype(&emb_paged_slots) f_slots;
decltype(&emb_qk_norm_rope) f_qk;
decltype(&emb_paged_attention) f_attention;
decltype(&emb_paged8_store) f_store8;
decltype(&emb_paged8_read) f_read8;
decltype(&emb_paged8_attention) f_attention8;
PyObject *s_data_ptr, *s_shape, *s_stride, *s_nbytes, *s_itemsize, *s_is_contiguous, *s_is_cuda;

// An attribute, or a method without arguments, of a tensor: found in its type once, for the type that came first (torch.Tensor), and
// then without a lookup by name. Objects of other types are asked by name.
struct Ask {
    PyObject** name;
    bool method;
    PyObject* found = nullptr;  // descriptor of the type `of`
    PyTypeObject* of = nullptr;
    Ask(PyObject** n, bool m) : name(n), method(m) {}
    PyObject* operator()(PyObject* o) {
        if (!of) {
            PyObject* d = PyObject_GetAttr(reinterpret_cast<PyObject*>(Py_TYPE(o)), *name);
            if (!d) PyErr_Clear();
            const bool fits = d && PyObject_TypeCheck(d, method ? &PyMethodDescr_Type : &PyGetSetDescr_Type) &&
                              PyType_IsSubtype(Py_TYPE(o), reinterpret_cast<PyDescrObject*>(d)->d_type);
            if (fits) {
                found = d;
                of = reinterpret_cast<PyTypeObject*>(Py_NewRef(reinterpret_cast<PyObject*>(Py_TYPE(o))));
            } else {
                Py_XDECREF(d);
            }
        }
        if (Py_TYPE(o) != of) return method ? PyObject_CallMethodNoArgs(o, *name) : PyObject_GetAttr(o, *name);
        if (method) return PyObject_Vectorcall(found, &o, 1, nullptr);
        const PyGetSetDef* d = reinterpret_cast<PyGetSetDescrObject*>(found)->d_getset;
        return d->get(o, d->closure);
    }
};
Ask ask_data_ptr(&s_data_ptr, true), ask_stride(&s_stride, true), ask_is_contiguous(&s_is_contiguous, true);
Ask ask_shape(&s_shape, false), ask_nbytes(&s_nbytes, false), ask_itemsize(&s_itemsize, false), ask_is_cuda(&s_is_cuda, false);

// Reads arguments one after another; `ok` turns false, with a Python exception set, at the first that cannot be read.
struct Reader {
    bool ok = true;

    int64_t integer(PyObject* o) {
        if (!ok) return 0;
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) ok = false;
        return v;
    }
    double real(PyObject* o) {
        if (!ok) return 0.0;
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) ok = false;
        return v;
    }
    void* address(PyObject* o) {  // of a tensor; of an integer, itself; NULL for None
        if (!ok || o == Py_None) return nullptr;
        PyObject* v = PyLong_Check(o) ? Py_NewRef(o) : ask_data_ptr(o);
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
        Py_XDECREF(v);
        if (PyErr_Occurred()) ok = false;
        return p;
    }
    // The sizes of a tensor of `n` dimensions.
    void sizes(PyObject* o, int n, int64_t* out) {
        if (!ok) return;
        PyObject* v = ask_shape(o);
        if (!v || !PyTuple_Check(v) || PyTuple_GET_SIZE(v) != n) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "a tensor of %d dimensions is expected", n);
            ok = false;
        } else {
            for (int i = 0; i < n; ++i) out[i] = integer(PyTuple_GET_ITEM(v, i));
        }
        Py_XDECREF(v);
    }
    // Elements between the rows of a tensor of two dimensions; those of a row lie side by side.
    int64_t row_stride(PyObject* o, const char* name, int64_t columns) {
        if (!ok) return 0;
        PyObject* v = ask_stride(o);
        int64_t s[2] = {};
        if (!v || !PyTuple_Check(v) || PyTuple_GET_SIZE(v) != 2) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a tensor of 2 dimensions is expected");
            ok = false;
        } else {
            for (int i = 0; i < 2; ++i) s[i] = integer(PyTuple_GET_ITEM(v, i));
        }
        Py_XDECREF(v);
        if (ok && s[1] != 1 && columns > 1) refuse("%s: the elements of a row do not lie side by side", name);
        return s[0];
    }

    char why[160] = "";  // the first refusal
    template <typename... A>
    void refuse(const char* format, A... a) {
        if (!why[0]) std::snprintf(why, sizeof(why), format, a...);
    }
    int64_t attribute(PyObject* o, Ask& ask) {
        if (!ok) return 0;
        PyObject* v = ask(o);
        const int64_t n = v ? integer(v) : 0;
        if (!v) ok = false;
        Py_XDECREF(v);
        return n;
    }
    void contiguous(PyObject* o, const char* name) {
        if (!ok) return;
        PyObject* v = ask_is_contiguous(o);
        if (!v) ok = false;
        if (v == Py_False) refuse("%s is not contiguous", name);
        Py_XDECREF(v);
    }
    // The tensor holds `count` elements of `size` bytes, side by side.
    void holds(PyObject* o, const char* name, int64_t count, int64_t size) {
        if (!ok || o == Py_None || PyLong_Check(o)) return;
        const int64_t bytes = attribute(o, ask_nbytes), each = attribute(o, ask_itemsize);
        if (!ok) return;
        if (each != size) refuse("%s: elements of %lld bytes, %lld expected", name, static_cast<long long>(each), static_cast<long long>(size));
        else if (bytes / size < count) refuse("%s has %lld elements, %lld needed", name, static_cast<long long>(bytes / size), static_cast<long long>(count));
        contiguous(o, name);
    }
    // The tensor is on the device, as `like` is: its maker leaves it in host memory, or another call wants it there.
    void on_device(PyObject* o, const char* name, PyObject* like) {
        if (!ok || o == Py_None || PyLong_Check(o)) return;
        if (attribute(like, ask_is_cuda) != 0 && ok && attribute(o, ask_is_cuda) == 0) refuse("%s is in host memory", name);
    }
    // Positions of T tokens, [tokens] or [axes][tokens]: their axes and the elements between those. False: an exception is set.
    bool positions(PyObject* o, int64_t T, int64_t& axes, int64_t& pos_stride) {
        if (!ok) return true;
        PyObject* shape = ask_shape(o);
        const bool several = shape && PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 2;
        Py_XDECREF(shape);
        if (!shape) return false;
        if (!several) {
            holds(o, "positions", T, 4);
            return true;
        }
        int64_t at[2] = {};
        sizes(o, 2, at);
        axes = at[0];
        pos_stride = row_stride(o, "positions", T);
        if (axes == 1 && pos_stride < T) pos_stride = T;  // (of one row it says nothing)
        if (at[1] < T) refuse("positions has %lld columns, %lld needed", static_cast<long long>(at[1]), static_cast<long long>(T));
        if (attribute(o, ask_itemsize) != 4) refuse("positions: elements of 4 bytes expected");
        return true;
    }
    // Codes and exponents of an 8-bit cache of the sizes pages, page size, heads, head dim.
    void cache8(PyObject* k_codes, PyObject* v_codes, PyObject* k_exp, PyObject* v_exp, const int64_t (&c)[4]) {
        const int64_t codes = c[0] * c[1] * c[2] * c[3], exps = c[0] * (c[1] / 16) * c[2];
        holds(k_codes, "k_codes", codes, 1);
        holds(v_codes, "v_codes", codes, 1);
        holds(k_exp, "k_exp", exps, 1);
        holds(v_exp, "v_exp", exps, 1);
    }
};

bool enough(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, want);
    return n == want;
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 3)) return nullptr;
    Reader r;
    f_slots = reinterpret_cast<decltype(f_slots)>(r.address(a[0]));
    f_qk = reinterpret_cast<decltype(f_qk)>(r.address(a[1]));
    f_attention = reinterpret_cast<decltype(f_attention)>(r.address(a[2]));
    if (!r.ok) return nullptr;
    Py_RETURN_NONE;
}

// cached, added, free_pages, used, table, q_start, kv_len, slots, positions, used_out, page_size, stream
PyObject* slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 12)) return nullptr;
    Reader r;
    int64_t table[2], n_free, n_tokens;
    r.sizes(a[4], 2, table);
    r.sizes(a[2], 1, &n_free);
    r.sizes(a[7], 1, &n_tokens);
    void* p[10];
    for (int i = 0; i < 10; ++i) p[i] = r.address(a[i]);
    const int64_t page = r.integer(a[10]);
    void* stream = r.address(a[11]);
    const int64_t R = table[0];
    r.holds(a[0], "cached", R, 4);
    r.holds(a[1], "added", R, 4);
    r.holds(a[2], "free_pages", n_free, 4);
    r.holds(a[3], "used", 1, 4);
    r.holds(a[4], "table", R * table[1], 4);
    r.holds(a[5], "q_start", R + 1, 4);
    r.holds(a[6], "kv_len", R, 4);
    r.holds(a[7], "slots", n_tokens, 8);
    r.holds(a[8], "positions", n_tokens, 4);
    r.holds(a[9], "used_out", 1, 4);
    if (!r.ok) return nullptr;
    if (r.why[0]) return PyUnicode_FromString(r.why);
    emb_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f_slots(static_cast<int32_t*>(p[0]), static_cast<int32_t*>(p[1]), table[0], static_cast<int32_t*>(p[2]), n_free,
                 static_cast<int32_t*>(p[3]), page, static_cast<int32_t*>(p[4]), table[1], static_cast<int32_t*>(p[5]),
                 static_cast<int32_t*>(p[6]), static_cast<int64_t*>(p[7]), static_cast<int32_t*>(p[8]), n_tokens,
                 static_cast<int32_t*>(p[9]), static_cast<emb_stream_t>(stream));
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

// q, k, v, q_out, k_cache, v_cache, slots, positions, q_gamma, k_gamma, eps, axis_of_pair (bytes or None), rot_dim (or
// None), base, stream
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 15)) return nullptr;
    Reader r;
    int64_t cache[4] = {}, q[2] = {}, k[2] = {}, v[2] = {};
    r.sizes(a[4], 4, cache);  // pages, page size, heads, head dim
    r.sizes(a[0], 2, q);
    r.sizes(a[1], 2, k);
    r.sizes(a[2], 2, v);
    const int64_t T = q[0], kw = cache[2] * cache[3];
    int64_t axes = 1, pos_stride = T;
    if (!r.positions(a[7], T, axes, pos_stride)) return nullptr;
    void* p[10];
    for (int i = 0; i < 10; ++i) p[i] = r.address(a[i]);
    const int64_t qs = r.row_stride(a[0], "q", q[1]), ks = r.row_stride(a[1], "k", k[1]), vs = r.row_stride(a[2], "v", v[1]);
    if (cache[3] > 0 && q[1] % cache[3] != 0) r.refuse("q: rows of %lld elements are no whole heads of %lld", static_cast<long long>(q[1]), static_cast<long long>(cache[3]));
    if (k[0] < T || k[1] < kw) r.refuse("k: fewer rows than q, or heads than the cache");
    if (v[0] < T || v[1] < kw) r.refuse("v: fewer rows than q, or heads than the cache");
    r.holds(a[3], "q_out", T * q[1], 2);
    r.holds(a[4], "k_cache", cache[0] * cache[1] * kw, 2);
    r.holds(a[5], "v_cache", cache[0] * cache[1] * kw, 2);
    r.holds(a[6], "slots", T, 8);
    r.holds(a[8], "q_gamma", cache[3], 4);
    r.holds(a[9], "k_gamma", cache[3], 4);
    const float eps = float(r.real(a[10])), base = float(r.real(a[13]));
    const int64_t d = cache[3], rot = a[12] == Py_None ? d : r.integer(a[12]);
    const uint8_t* axis = nullptr;
    if (r.ok && a[11] != Py_None) {
        char* bytes;
        Py_ssize_t len;
        if (PyBytes_AsStringAndSize(a[11], &bytes, &len) != 0) return nullptr;
        if (len != rot / 2) return PyLong_FromLong(EMB_EINVAL);
        axis = reinterpret_cast<const uint8_t*>(bytes);
    }
    void* stream = r.address(a[14]);
    if (!r.ok) return nullptr;
    if (r.why[0]) return PyUnicode_FromString(r.why);
    emb_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f_qk(static_cast<uint16_t*>(p[0]), qs, static_cast<uint16_t*>(p[1]), ks, static_cast<uint16_t*>(p[2]), vs, q[0],
              d > 0 ? q[1] / d : 0, cache[2], d, static_cast<float*>(p[8]), static_cast<float*>(p[9]), eps,
              static_cast<int32_t*>(p[7]), pos_stride, axes, axis, rot, base, static_cast<int64_t*>(p[6]),
              static_cast<uint16_t*>(p[3]), static_cast<uint16_t*>(p[4]), static_cast<uint16_t*>(p[5]), cache[0], cache[1],
              static_cast<emb_stream_t>(stream));
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

// Q, k_cache, v_cache, table, q_start, kv_len, O, workspace, prefix, scale, max_q, cap, window, ws_bytes, stream
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 15)) return nullptr;
    Reader r;
    int64_t cache[4] = {}, q[2] = {}, table[2] = {};
    r.sizes(a[1], 4, cache);
    r.sizes(a[0], 2, q);
    r.sizes(a[3], 2, table);
    void* p[9];
    for (int i = 0; i < 9; ++i) p[i] = r.address(a[i]);
    const float scale = float(r.real(a[9])), cap = float(r.real(a[11]));
    const int64_t max_q = r.integer(a[10]), window = r.integer(a[12]), bytes = r.integer(a[13]), d = cache[3];
    void* stream = r.address(a[14]);
    if (d > 0 && q[1] % d != 0) r.refuse("Q: rows of %lld elements are no whole heads of %lld", static_cast<long long>(q[1]), static_cast<long long>(d));
    r.holds(a[0], "Q", q[0] * q[1], 2);
    r.holds(a[1], "k_cache", cache[0] * cache[1] * cache[2] * d, 2);
    r.holds(a[2], "v_cache", cache[0] * cache[1] * cache[2] * d, 2);
    r.holds(a[3], "table", table[0] * table[1], 4);
    r.holds(a[4], "q_start", table[0] + 1, 4);
    r.holds(a[5], "kv_len", table[0], 4);
    r.holds(a[6], "O", q[0] * q[1], 2);
    r.holds(a[8], "prefix", table[0], 4);
    if (!r.ok) return nullptr;
    if (r.why[0]) return PyUnicode_FromString(r.why);
    emb_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f_attention(static_cast<uint16_t*>(p[0]), static_cast<uint16_t*>(p[1]), static_cast<uint16_t*>(p[2]), cache[0], cache[1],
                     static_cast<int32_t*>(p[3]), table[1], static_cast<int32_t*>(p[4]), static_cast<int32_t*>(p[5]),
                     static_cast<int32_t*>(p[8]), table[0], q[0], max_q, static_cast<uint16_t*>(p[6]), d > 0 ? q[1] / d : 0,
                     cache[2], d, scale, cap, window, p[7], size_t(bytes), static_cast<emb_stream_t>(stream));
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

// The addresses of the 8-bit cache's entry points.
PyObject* bind8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 3)) return nullptr;
    Reader r;
    f_store8 = reinterpret_cast<decltype(f_store8)>(r.address(a[0]));
    f_read8 = reinterpret_cast<decltype(f_read8)>(r.address(a[1]));
    f_attention8 = reinterpret_cast<decltype(f_attention8)>(r.address(a[2]));
    if (!r.ok) return nullptr;
    Py_RETURN_NONE;
}

// q, k, v, q_out, k_codes, v_codes, k_exp, v_exp, slots, positions, turns, q_gamma, k_gamma, axis_of_pair, eps, neighbours, factor,
// stream
PyObject* store8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 18)) return nullptr;
    Reader r;
    int64_t cache[4] = {}, q[2] = {}, k[2] = {}, v[2] = {}, pairs = 0;
    r.sizes(a[4], 4, cache);
    r.sizes(a[0], 2, q);
    r.sizes(a[1], 2, k);
    r.sizes(a[2], 2, v);
    if (a[10] != Py_None) r.sizes(a[10], 1, &pairs);
    const int64_t T = q[0], d = cache[3], kw = cache[2] * d;
    int64_t axes = 1, pos_stride = T;
    if (!r.positions(a[9], T, axes, pos_stride)) return nullptr;
    void* p[14];
    for (int i = 0; i < 14; ++i) p[i] = r.address(a[i]);
    const int64_t qs = r.row_stride(a[0], "q", q[1]), ks = r.row_stride(a[1], "k", k[1]), vs = r.row_stride(a[2], "v", v[1]);
    if (r.attribute(a[0], ask_itemsize) != 2 || r.attribute(a[1], ask_itemsize) != 2 || r.attribute(a[2], ask_itemsize) != 2)
        r.refuse("q, k, v: elements of 2 bytes expected");
    if (d > 0 && q[1] % d != 0) r.refuse("q: rows of %lld elements are no whole heads of %lld", static_cast<long long>(q[1]), static_cast<long long>(d));
    if (k[0] < T || k[1] < kw) r.refuse("k: fewer rows than q, or heads than the cache");
    if (v[0] < T || v[1] < kw) r.refuse("v: fewer rows than q, or heads than the cache");
    r.holds(a[3], "q_out", T * q[1], 2);
    r.cache8(a[4], a[5], a[6], a[7], cache);
    r.holds(a[8], "slots", T, 8);
    r.holds(a[10], "turns", pairs, 8);
    r.holds(a[11], "q_gamma", d, 4);
    r.holds(a[12], "k_gamma", d, 4);
    r.holds(a[13], "axis_of_pair", pairs, 1);
    r.on_device(a[10], "turns", a[0]);
    r.on_device(a[13], "axis_of_pair", a[0]);
    const float eps = float(r.real(a[14])), factor = float(r.real(a[16]));
    const int64_t neighbours = r.integer(a[15]);
    void* stream = r.address(a[17]);
    if (!r.ok) return nullptr;
    if (r.why[0]) return PyUnicode_FromString(r.why);
    emb_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f_store8(static_cast<uint16_t*>(p[0]), qs, static_cast<uint16_t*>(p[1]), ks, static_cast<uint16_t*>(p[2]), vs, T,
                  d > 0 ? q[1] / d : 0, cache[2], d, static_cast<float*>(p[11]), static_cast<float*>(p[12]), eps,
                  static_cast<int32_t*>(p[9]), pos_stride, axes, static_cast<uint8_t*>(p[13]), static_cast<uint64_t*>(p[10]), 2 * pairs,
                  neighbours == 0 ? 0 : 1, factor, static_cast<int64_t*>(p[8]), static_cast<uint16_t*>(p[3]), static_cast<uint8_t*>(p[4]),
                  static_cast<uint8_t*>(p[5]), static_cast<uint8_t*>(p[6]), static_cast<uint8_t*>(p[7]), cache[0], cache[1],
                  static_cast<emb_stream_t>(stream));
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

// k_codes, v_codes, k_exp, v_exp, slots, k_out, v_out, stream
PyObject* read8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 8)) return nullptr;
    Reader r;
    int64_t cache[4] = {}, rows = 0;
    r.sizes(a[0], 4, cache);
    r.sizes(a[4], 1, &rows);
    void* p[7];
    for (int i = 0; i < 7; ++i) p[i] = r.address(a[i]);
    r.cache8(a[0], a[1], a[2], a[3], cache);
    r.holds(a[4], "slots", rows, 8);
    r.holds(a[5], "k_out", rows * cache[2] * cache[3], 2);
    r.holds(a[6], "v_out", rows * cache[2] * cache[3], 2);
    void* stream = r.address(a[7]);
    if (!r.ok) return nullptr;
    if (r.why[0]) return PyUnicode_FromString(r.why);
    emb_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f_read8(static_cast<uint8_t*>(p[0]), static_cast<uint8_t*>(p[1]), static_cast<uint8_t*>(p[2]), static_cast<uint8_t*>(p[3]),
                 cache[0], cache[1], cache[2], cache[3], static_cast<int64_t*>(p[4]), rows, static_cast<uint16_t*>(p[5]),
                 static_cast<uint16_t*>(p[6]), static_cast<emb_stream_t>(stream));
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

// Q, k_codes, v_codes, k_exp, v_exp, table, q_start, kv_len, O, workspace, prefix, scale, max_q, cap, window, ws_bytes, stream
PyObject* attention8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!enough(n, 17)) return nullptr;
    Reader r;
    int64_t cache[4] = {}, q[2] = {}, table[2] = {};
    r.sizes(a[1], 4, cache);
    r.sizes(a[0], 2, q);
    r.sizes(a[5], 2, table);
    void* p[11];
    for (int i = 0; i < 11; ++i) p[i] = r.address(a[i]);
    const float scale = float(r.real(a[11])), cap = float(r.real(a[13]));
    const int64_t max_q = r.integer(a[12]), window = r.integer(a[14]), bytes = r.integer(a[15]), d = cache[3];
    void* stream = r.address(a[16]);
    if (d > 0 && q[1] % d != 0) r.refuse("Q: rows of %lld elements are no whole heads of %lld", static_cast<long long>(q[1]), static_cast<long long>(d));
    r.holds(a[0], "Q", q[0] * q[1], 2);
    r.cache8(a[1], a[2], a[3], a[4], cache);
    r.holds(a[5], "table", table[0] * table[1], 4);
    r.holds(a[6], "q_start", table[0] + 1, 4);
    r.holds(a[7], "kv_len", table[0], 4);
    r.holds(a[8], "O", q[0] * q[1], 2);
    r.holds(a[10], "prefix", table[0], 4);
    if (!r.ok) return nullptr;
    if (r.why[0]) return PyUnicode_FromString(r.why);
    emb_status st;
    Py_BEGIN_ALLOW_THREADS;
    st = f_attention8(static_cast<uint16_t*>(p[0]), static_cast<uint8_t*>(p[1]), static_cast<uint8_t*>(p[2]), static_cast<uint8_t*>(p[3]),
                      static_cast<uint8_t*>(p[4]), cache[0], cache[1], static_cast<int32_t*>(p[5]), table[1], static_cast<int32_t*>(p[6]),
                      static_cast<int32_t*>(p[7]), static_cast<int32_t*>(p[10]), table[0], q[0], max_q, static_cast<uint16_t*>(p[8]),
                      d > 0 ? q[1] / d : 0, cache[2], d, scale, cap, window, p[9], size_t(bytes), static_cast<emb_stream_t>(stream));
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(st);
}

using Fast = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyMethodDef method(const char* name, Fast f) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method("bind", bind), method("slots", slots), method("qk_norm_rope", qk_norm_rope),
                         method("attention", attention), method("bind8", bind8), method("store8", store8),
                         method("read8", read8), method("attention8", attention8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged_binding(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    s_itemsize = PyUnicode_InternFromString("itemsize");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    return PyModule_Create(&module);
}
