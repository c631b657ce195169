// The calls a training or decode loop makes, from torch tensors to libqeft's C functions without the interpreter in between:
// binding.py's functions pass their arguments here first.  The smallest calls are bound by the host: one row through a 512 x 512 layer took
// 5.9 us with ctypes (a struct of four pointers, ten conversions, two lookups of the stream), of which a bare launch of an empty kernel with as many
// arguments is 3.8; it takes 4.0 now, 0.25 of them here.  A group call 5.1 -> 3.9.
//
// Only plain cases are taken: exact tensors on one GPU, the current one, and this package's own argument objects.  Anything else - a subclass,
// host memory, a missing output - makes the functions return None, and binding.py goes the way it describes itself.  Nothing is kept
// between calls: pointers, pitches and the stream are read off the objects each time.  The interpreter's lock is released around the C call.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <cstring>

#include "qeft.h"

namespace {

struct Fns {
    decltype(&qeft_linear_fwd) fwd;
    decltype(&qeft_linear_fwd_group) fwd_group;
    decltype(&qeft_linear_bwd_dx) bwd_dx;
    decltype(&qeft_linear_bwd) bwd;
    decltype(&qeft_linear_fwd_irregular) fwd_irregular;
    decltype(&qeft_linear_bwd_dx_irregular) bwd_dx_irregular;
    decltype(&qeft_weak_grad) weak_grad;
    decltype(&qeft_cache_append) cache_append;
    decltype(&qeft_attn_decode) attn_decode;
    decltype(&qeft_cache_evict) cache_evict;
    decltype(&qeft_norm_fwd) norm_fwd;
    decltype(&qeft_norm_bwd) norm_bwd;
} fns;
constexpr int N_FNS = sizeof(Fns) / sizeof(void*);
PyTypeObject *desc_type, *weight_type, *cache_desc_type, *norm_desc_type;
PyObject *n_desc, *n_qweight, *n_scales, *n_zeros, *n_weak;

// the bytes of a ctypes object (which owns them for its lifetime)
template <class T>
const T* bytes_of(PyObject* o) {
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return nullptr;
    }
    const T* p = b.len >= (Py_ssize_t)sizeof(T) ? (const T*)b.buf : nullptr;
    PyBuffer_Release(&b);
    return p;
}

struct Call {
    int device = -1;
    bool ok = true;
    const at::Tensor* tensor(PyObject* o) {
        if (!ok || !THPVariable_CheckExact(o)) {
            ok = false;
            return nullptr;
        }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda()) ok = false;
        else if (device < 0) device = t.get_device();
        else if (device != t.get_device()) ok = false;
        return ok ? &t : nullptr;
    }
    void* ptr(PyObject* o) {
        const at::Tensor* t = tensor(o);
        return t ? t->data_ptr() : nullptr;
    }
    void* matrix(PyObject* o, int64_t& rows, int64_t& pitch) {
        const at::Tensor* t = tensor(o);
        if (!t || t->dim() != 2) {
            ok = false;
            return nullptr;
        }
        rows = t->size(0);
        pitch = t->stride(0);
        return t->data_ptr();
    }
    void* workspace(PyObject* o, size_t& n) {   // None: none
        n = 0;
        if (o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        if (!t) return nullptr;
        n = (size_t)t->numel();
        return t->data_ptr();
    }
    int number(PyObject* o) {
        const long v = PyLong_AsLong(o);
        if (v == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return (int)v;
    }
    const qeft_desc_t* desc(PyObject* o) {
        const qeft_desc_t* d = Py_TYPE(o) == desc_type ? bytes_of<qeft_desc_t>(o) : nullptr;
        if (!d) ok = false;
        return d;
    }
    template <class T>
    const T* described(PyObject* o, PyTypeObject* type) {
        const T* d = Py_TYPE(o) == type ? bytes_of<T>(o) : nullptr;
        if (!d) ok = false;
        return d;
    }
    double real(PyObject* o) {
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    int64_t whole(PyObject* o) {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
    // The calls between the linear layers check types and shapes: a tensor of this type with contiguous rows of `width` values (-1: any, which is
    // returned in it) and `rows` rows (the same), or None where it may be.  Anything else is left to binding.py, which says what is wrong.
    void* rows(PyObject* o, at::ScalarType type, int64_t& rows, int64_t& width, int64_t& pitch, bool optional = false) {
        pitch = 0;
        if (o == Py_None && optional) return nullptr;
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != type || t->dim() != 2 || t->numel() == 0) return no();
        if (rows < 0) rows = t->size(0);
        if (width < 0) width = t->size(1);
        if (t->size(0) != rows || t->size(1) != width || (width > 1 && t->stride(1) != 1)) return no();
        pitch = rows > 1 ? t->stride(0) : (width + 7) / 8 * 8;
        return t->data_ptr();
    }
    void* vec(PyObject* o, at::ScalarType type, int64_t n, bool optional = false) {
        if (o == Py_None && optional) return nullptr;
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != type || t->dim() != 1 || t->size(0) != n || n == 0 || (n > 1 && t->stride(0) != 1)) return no();
        return t->data_ptr();
    }
    // [seqs][heads][least or more], rows one pitch apart throughout (a single row's pitch: its width)
    void* planes(PyObject* o, at::ScalarType type, int64_t seqs, int64_t heads, int64_t least, int64_t& pitch, bool optional = false) {
        pitch = 0;
        if (o == Py_None && optional) return nullptr;
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != type || t->dim() != 3 || t->numel() == 0 || t->size(0) != seqs || t->size(1) != heads || t->size(2) < least) return no();
        if (t->size(2) > 1 && t->stride(2) != 1) return no();
        pitch = heads > 1 ? t->stride(1) : seqs > 1 ? t->stride(0) : t->size(2);
        if (seqs > 1 && t->stride(0) != pitch * heads) return no();
        return t->data_ptr();
    }
    void* pool(PyObject* o, const qeft_cache_desc_t* d) {
        const at::Tensor* t = tensor(o);
        if (!t || !d || t->scalar_type() != at::kHalf || t->dim() != 4) return no();
        const int64_t size[4] = {d->pages, d->kv_heads, d->page_size, d->head_dim}, stride[4] = {d->page_stride, d->head_stride, d->token_stride, 1};
        for (int i = 0; i < 4; ++i)
            if (t->size(i) != size[i] || (size[i] > 1 && t->stride(i) != stride[i])) return no();
        return t->data_ptr();
    }
    void* bytes(PyObject* o, size_t& n) {   // a workspace of uint8, or None
        n = 0;
        if (o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        if (!t || t->scalar_type() != at::kByte || t->dim() != 1 || (t->numel() > 1 && t->stride(0) != 1)) return no();
        n = (size_t)t->numel();
        return t->data_ptr();
    }
    void* no() {
        ok = false;
        return nullptr;
    }
    void weight(PyObject* o, qeft_weight_t& w) {
        w = {};
        if (!ok || Py_TYPE(o) != weight_type) {
            ok = false;
            return;
        }
        PyObject* own = PyObject_GetAttr(o, n_desc);
        const qeft_desc_t* d = own ? desc(own) : nullptr;
        auto take = [&](PyObject* name) -> void* {
            PyObject* t = ok ? PyObject_GetAttr(o, name) : nullptr;
            if (!t) {
                ok = false;
                return nullptr;
            }
            void* p = ptr(t);
            Py_DECREF(t);
            return p;
        };
        if (d && d->in_features > d->n_weak) {
            w.qweight = (decltype(w.qweight))take(n_qweight);
            w.scales = (decltype(w.scales))take(n_scales);
            w.zeros = (decltype(w.zeros))take(n_zeros);
        }
        if (d && d->n_weak > 0) w.weak = (decltype(w.weak))take(n_weak);
        if (!d) ok = false;
        Py_XDECREF(own);
        if (PyErr_Occurred()) PyErr_Clear();
    }
    // the current stream, if the tensors' GPU is the current one (binding.py takes the current GPU's)
    void* stream() {
        if (!ok || device < 0 || c10::hip::current_device() != device) {
            ok = false;
            return nullptr;
        }
        return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
    }
};

// Runs f(call) with torch's exceptions as Python's; f returns false where the call is not a plain one.
template <class F>
PyObject* guarded(F&& f) {
    int status = 0;
    try {
        Call c;
        if (!f(c, status)) Py_RETURN_NONE;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    return PyLong_FromLong(status);
}
template <class F>
int unlocked(F&& f) {
    PyThreadState* s = PyEval_SaveThread();
    const int st = f();
    PyEval_RestoreThread(s);
    return st;
}

// (desc, w, X, Y, ws)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        if (n != 5) return false;
        const qeft_desc_t* d = c.desc(a[0]);
        qeft_weight_t w;
        c.weight(a[1], w);
        if (!c.ok) return false;
        int64_t M, ldx, my, ldy;
        size_t nws;
        const void* x = c.matrix(a[2], M, ldx);
        void* y = c.matrix(a[3], my, ldy);
        void* ws = c.workspace(a[4], nws);
        void* s = c.stream();
        if (!c.ok) return false;
        if (!M) ldx = d->in_features, ldy = d->out_features;   // (an empty matrix's pitch says nothing)
        st = unlocked([&] { return fns.fwd(d, &w, x, M, ldx, y, ldy, ws, nws, s); });
        return true;
    });
}
// (n, descs, weights, X, ys, ldys): the arrays of a Group
PyObject* linear_fwd_group(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        if (n != 6) return false;
        const int layers = c.number(a[0]);
        const qeft_desc_t* d = bytes_of<qeft_desc_t>(a[1]);
        const qeft_weight_t* w = bytes_of<qeft_weight_t>(a[2]);
        void* const* ys = bytes_of<void*>(a[4]);
        const int64_t* ldy = bytes_of<int64_t>(a[5]);
        int64_t M, ldx;
        const void* x = c.matrix(a[3], M, ldx);
        void* s = c.stream();
        if (!c.ok || !d || !w || !ys || !ldy) return false;
        if (!M) ldx = d->in_features;
        st = unlocked([&] { return fns.fwd_group(layers, d, w, x, M, ldx, ys, ldy, s); });
        return true;
    });
}
// (desc, w, dY, dX, ws)
PyObject* linear_bwd_dx(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        if (n != 5) return false;
        const qeft_desc_t* d = c.desc(a[0]);
        qeft_weight_t w;
        c.weight(a[1], w);
        if (!c.ok) return false;
        int64_t M, ldy, mx, ldx;
        size_t nws;
        const void* y = c.matrix(a[2], M, ldy);
        void* x = c.matrix(a[3], mx, ldx);
        void* ws = c.workspace(a[4], nws);
        void* s = c.stream();
        if (!c.ok) return false;
        if (!M) ldy = d->out_features, ldx = d->in_features;
        st = unlocked([&] { return fns.bwd_dx(d, &w, y, M, ldy, x, ldx, ws, nws, s); });
        return true;
    });
}
// (desc, w, perm, X or dY, Y or dX, ws)
template <bool FWD>
PyObject* irregular(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        if (n != 6) return false;
        const qeft_desc_t* d = c.desc(a[0]);
        qeft_weight_t w;
        c.weight(a[1], w);
        if (!c.ok) return false;
        const int32_t* perm = (const int32_t*)c.ptr(a[2]);
        int64_t M, ldi, mo, ldo;
        size_t nws;
        const void* in = c.matrix(a[3], M, ldi);
        void* out = c.matrix(a[4], mo, ldo);
        void* ws = c.workspace(a[5], nws);
        void* s = c.stream();
        if (!c.ok) return false;
        if (!M) ldi = FWD ? d->in_features : d->out_features, ldo = FWD ? d->out_features : d->in_features;
        st = unlocked([&] { return (FWD ? fns.fwd_irregular : fns.bwd_dx_irregular)(d, &w, perm, in, M, ldi, out, ldo, ws, nws, s); });
        return true;
    });
}
// (desc, dY, Xw, dW, dtype, accumulate, ws)
PyObject* weak_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        if (n != 7) return false;
        const qeft_desc_t* d = c.desc(a[0]);
        if (!c.ok) return false;
        int64_t M, ldy, mx, ldx;
        size_t nws;
        const void* y = c.matrix(a[1], M, ldy);
        const void* x = c.matrix(a[2], mx, ldx);
        void* dw = c.ptr(a[3]);
        const int dtype = c.number(a[4]), accumulate = c.number(a[5]);
        void* ws = c.workspace(a[6], nws);
        void* s = c.stream();
        if (!c.ok || mx != M) return false;
        if (!M) ldy = d->out_features, ldx = d->n_weak > 8 ? d->n_weak : 8;
        st = unlocked([&] { return fns.weak_grad(d, y, M, ldy, x, ldx, dw, dtype, accumulate, ws, nws, s); });
        return true;
    });
}
// (desc, w, dY, dX, Xw, dW, dtype, accumulate, ws)
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        if (n != 9) return false;
        const qeft_desc_t* d = c.desc(a[0]);
        qeft_weight_t w;
        c.weight(a[1], w);
        if (!c.ok) return false;
        int64_t M, ldy, mx, ldx, mw, ldw;
        size_t nws;
        const void* y = c.matrix(a[2], M, ldy);
        void* x = c.matrix(a[3], mx, ldx);
        const void* xw = c.matrix(a[4], mw, ldw);
        void* dw = c.ptr(a[5]);
        const int dtype = c.number(a[6]), accumulate = c.number(a[7]);
        void* ws = c.workspace(a[8], nws);
        void* s = c.stream();
        if (!c.ok || mw != M) return false;
        if (!M) ldy = d->out_features, ldx = d->in_features, ldw = d->n_weak > 8 ? d->n_weak : 8;
        st = unlocked([&] { return fns.bwd(d, &w, y, M, ldy, x, ldx, xw, ldw, dw, dtype, accumulate, ws, nws, s); });
        return true;
    });
}
// What the calls on a cache have in common: (desc, pool of keys, pool of values, page table, ...)
bool cache_args(Call& c, PyObject* const* a, const qeft_cache_desc_t*& d, qeft_cache_t& pools, qeft_table_t& table) {
    d = c.described<qeft_cache_desc_t>(a[0], cache_desc_type);
    if (!d) return false;
    pools.k = c.pool(a[1], d);
    pools.v = c.pool(a[2], d);
    int64_t seqs = -1, pages = -1;
    table.table = (const int32_t*)c.rows(a[3], at::kInt, seqs, pages, table.ld_table);
    if (!c.ok || seqs > QEFT_MAX_DIM || pages > INT32_MAX) return false;
    table.table_pages = (int32_t)pages;
    table.seqs = (int32_t)seqs;
    return true;
}
// tokens that a row of the table can hold
int64_t slots(const qeft_cache_desc_t* d, const qeft_table_t& table) { return (int64_t)table.table_pages * d->page_size; }
// (desc, K, V, table, k, v, index, seq, q, q_out, rot, pos)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        const qeft_cache_desc_t* d;
        qeft_cache_t pools;
        qeft_table_t table;
        if (n != 12 || !cache_args(c, a, d, pools, table)) return false;
        qeft_append_t p;
        int64_t tokens = -1, width = (int64_t)d->kv_heads * d->head_dim, qw = -1, positions = -1, rot = -1;
        p.k = c.rows(a[4], at::kHalf, tokens, width, p.ldk);
        p.v = c.rows(a[5], at::kHalf, tokens, width, p.ldv);
        p.index = (const int32_t*)c.vec(a[6], at::kInt, tokens);
        p.seq = (const int32_t*)c.vec(a[7], at::kInt, tokens, true);
        p.q = c.rows(a[8], at::kHalf, tokens, qw, p.ldq, true);
        p.q_out = nullptr, p.ldq_out = 0;
        if (p.q) p.q_out = c.rows(a[9], at::kHalf, tokens, qw, p.ldq_out);
        p.rot = (const float*)c.rows(a[10], at::kFloat, positions, rot, p.ld_rot, true);
        p.pos = (const int32_t*)c.vec(a[11], at::kInt, tokens, true);
        void* s = c.stream();
        if (!c.ok || (p.q && (qw % d->head_dim != 0 || qw / d->head_dim > INT32_MAX)) || positions > INT32_MAX || rot > INT32_MAX) return false;
        p.heads = p.q ? (int32_t)(qw / d->head_dim) : 0;
        p.positions = p.rot ? (int32_t)positions : 0;
        p.rot_dim = p.rot ? (int32_t)rot : 0;
        p.tokens = tokens;
        st = unlocked([&] { return fns.cache_append(d, &pools, &table, &p, s); });
        return true;
    });
}
// (desc, K, V, table, lens, longest, q, out, score, accumulate, scale, ws)
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        const qeft_cache_desc_t* d;
        qeft_cache_t pools;
        qeft_table_t table;
        if (n != 12 || !cache_args(c, a, d, pools, table)) return false;
        qeft_attn_t p;
        int64_t seqs = table.seqs, width = -1;
        p.lens = (const int32_t*)c.vec(a[4], at::kInt, seqs);
        p.longest = c.whole(a[5]);
        p.q = c.rows(a[6], at::kHalf, seqs, width, p.ldq);
        p.out = c.rows(a[7], at::kHalf, seqs, width, p.ldo);
        p.score = (float*)c.planes(a[8], at::kFloat, seqs, d->kv_heads, std::min(p.longest, slots(d, table)), p.ld_score, true);
        p.accumulate = PyObject_IsTrue(a[9]) == 1;
        p.scale = (float)c.real(a[10]);
        p.ws = c.bytes(a[11], p.ws_bytes);
        void* s = c.stream();
        if (!c.ok || width % d->head_dim != 0 || width / d->head_dim > INT32_MAX) return false;
        p.heads = (int32_t)(width / d->head_dim);
        st = unlocked([&] { return fns.attn_decode(d, &pools, &table, &p, s); });
        return true;
    });
}
// (desc, K, V, table, lens, longest, budget, score, pos, seen, keep_first, keep_last, score_out, pos_out, lens_out, ws)
PyObject* cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&](Call& c, int& st) {
        const qeft_cache_desc_t* d;
        qeft_cache_t pools;
        qeft_table_t table;
        if (n != 16 || !cache_args(c, a, d, pools, table)) return false;
        qeft_evict_t p;
        const int64_t seqs = table.seqs;
        int64_t ld_pos, ld_pos_out;
        p.lens = (const int32_t*)c.vec(a[4], at::kInt, seqs);
        p.longest = c.whole(a[5]);
        p.budget = c.whole(a[6]);
        const int64_t longest = std::min(p.longest, slots(d, table));
        p.score = (const float*)c.planes(a[7], at::kFloat, seqs, d->kv_heads, longest, p.ld);
        p.pos = (const int32_t*)c.planes(a[8], at::kInt, seqs, d->kv_heads, longest, ld_pos);
        p.seen = (const int32_t*)c.vec(a[9], at::kInt, seqs);
        const int64_t first = c.whole(a[10]), last = c.whole(a[11]);
        p.score_out = (float*)c.planes(a[12], at::kFloat, seqs, d->kv_heads, std::min(p.budget, longest), p.ld_out);
        p.pos_out = (int32_t*)c.planes(a[13], at::kInt, seqs, d->kv_heads, std::min(p.budget, longest), ld_pos_out);
        p.lens_out = (int32_t*)c.vec(a[14], at::kInt, seqs);
        p.ws = c.bytes(a[15], p.ws_bytes);
        void* s = c.stream();
        if (!c.ok || ld_pos != p.ld || ld_pos_out != p.ld_out || first < 0 || first > INT32_MAX || last < 0 || last > INT32_MAX) return false;
        p.keep_first = (int32_t)first;
        p.keep_last = (int32_t)last;
        st = unlocked([&] { return fns.cache_evict(d, &pools, &table, &p, s); });
        return true;
    });
}
// the type of the residual stream, and a gate as its kind has it
at::ScalarType residual(const qeft_norm_desc_t* d) { return d->residual_dtype == QEFT_DTYPE_F32 ? at::kFloat : at::kHalf; }
void* gate_of(Call& c, PyObject* o, const qeft_norm_desc_t* d, int64_t m, int64_t n, int64_t& pitch) {
    pitch = 0;
    return d->gate == QEFT_GATE_TOKEN ? c.rows(o, at::kHalf, m, n, pitch, true) : c.vec(o, at::kHalf, n, true);
}
// (desc, r, w_pre, y, w_post, gate, h, x)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t argc) {
    return guarded([&](Call& c, int& st) {
        if (argc != 8) return false;
        const qeft_norm_desc_t* d = c.described<qeft_norm_desc_t>(a[0], norm_desc_type);
        if (!d) return false;
        qeft_norm_fwd_t p;
        int64_t m = -1, n = d->n;
        p.r = c.rows(a[1], residual(d), m, n, p.ldr);
        p.w_pre = c.vec(a[2], at::kHalf, n);
        p.y = c.rows(a[3], at::kHalf, m, n, p.ldy, true);
        p.w_post = c.vec(a[4], at::kHalf, n, true);
        p.gate = gate_of(c, a[5], d, m, n, p.ldg);
        p.h = c.rows(a[6], residual(d), m, n, p.ldh, true);
        p.x = c.rows(a[7], at::kHalf, m, n, p.ldx);
        void* s = c.stream();
        if (!c.ok) return false;
        p.m = m;
        st = unlocked([&] { return fns.norm_fwd(d, &p, s); });
        return true;
    });
}
// (desc, dx, h, w_pre, dh, y, w_post, gate, dr, dy, dw_pre, dw_post, dgate, accumulate, ws)
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t argc) {
    return guarded([&](Call& c, int& st) {
        if (argc != 15) return false;
        const qeft_norm_desc_t* d = c.described<qeft_norm_desc_t>(a[0], norm_desc_type);
        if (!d) return false;
        qeft_norm_bwd_t p;
        int64_t m = -1, n = d->n;
        p.dx = c.rows(a[1], at::kHalf, m, n, p.lddx);
        p.h = c.rows(a[2], residual(d), m, n, p.ldh);
        p.w_pre = c.vec(a[3], at::kHalf, n);
        p.dh = c.rows(a[4], residual(d), m, n, p.lddh, true);
        p.y = c.rows(a[5], at::kHalf, m, n, p.ldy, true);
        p.w_post = c.vec(a[6], at::kHalf, n, true);
        p.gate = gate_of(c, a[7], d, m, n, p.ldg);
        p.dr = c.rows(a[8], residual(d), m, n, p.lddr, true);
        p.dy = c.rows(a[9], at::kHalf, m, n, p.lddy, true);
        p.dw_pre = (float*)c.vec(a[10], at::kFloat, n, true);
        p.dw_post = (float*)c.vec(a[11], at::kFloat, n, true);
        p.lddg = 0;
        p.dgate = d->gate == QEFT_GATE_TOKEN ? c.rows(a[12], at::kHalf, m, n, p.lddg, true) : c.vec(a[12], at::kFloat, n, true);
        p.accumulate = PyObject_IsTrue(a[13]) == 1;
        p.ws = c.bytes(a[14], p.ws_bytes);
        void* s = c.stream();
        if (!c.ok) return false;
        p.m = m;
        st = unlocked([&] { return fns.norm_bwd(d, &p, s); });
        return true;
    });
}
// (addresses of the C functions in the order of Fns, qeft_desc_t, Weight, qeft_cache_desc_t, qeft_norm_desc_t)
PyObject* init(PyObject*, PyObject* args) {
    PyObject *f, *d, *w, *cd, *nd;
    if (!PyArg_ParseTuple(args, "O!O!O!O!O!", &PyTuple_Type, &f, &PyType_Type, &d, &PyType_Type, &w, &PyType_Type, &cd, &PyType_Type, &nd)) return nullptr;
    if (PyTuple_GET_SIZE(f) != N_FNS) return PyErr_Format(PyExc_ValueError, "%d functions expected", N_FNS);
    void* at[N_FNS];
    for (int i = 0; i < N_FNS; ++i) {
        at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(f, i));
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&fns, at, sizeof fns);
    for (PyObject* o : {d, w, cd, nd}) Py_INCREF(o);
    desc_type = (PyTypeObject*)d;
    weight_type = (PyTypeObject*)w;
    cache_desc_type = (PyTypeObject*)cd;
    norm_desc_type = (PyTypeObject*)nd;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", init, METH_VARARGS, nullptr},
    {"linear_fwd", (PyCFunction)(void (*)())linear_fwd, METH_FASTCALL, nullptr},
    {"linear_fwd_group", (PyCFunction)(void (*)())linear_fwd_group, METH_FASTCALL, nullptr},
    {"linear_bwd_dx", (PyCFunction)(void (*)())linear_bwd_dx, METH_FASTCALL, nullptr},
    {"linear_fwd_irregular", (PyCFunction)(void (*)())irregular<true>, METH_FASTCALL, nullptr},
    {"linear_bwd_dx_irregular", (PyCFunction)(void (*)())irregular<false>, METH_FASTCALL, nullptr},
    {"weak_grad", (PyCFunction)(void (*)())weak_grad, METH_FASTCALL, nullptr},
    {"linear_bwd", (PyCFunction)(void (*)())linear_bwd, METH_FASTCALL, nullptr},
    {"cache_append", (PyCFunction)(void (*)())cache_append, METH_FASTCALL, nullptr},
    {"attn_decode", (PyCFunction)(void (*)())attn_decode, METH_FASTCALL, nullptr},
    {"cache_evict", (PyCFunction)(void (*)())cache_evict, METH_FASTCALL, nullptr},
    {"norm_fwd", (PyCFunction)(void (*)())norm_fwd, METH_FASTCALL, nullptr},
    {"norm_bwd", (PyCFunction)(void (*)())norm_bwd, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    n_desc = PyUnicode_InternFromString("desc");
    n_qweight = PyUnicode_InternFromString("qweight");
    n_scales = PyUnicode_InternFromString("scales");
    n_zeros = PyUnicode_InternFromString("zeros");
    n_weak = PyUnicode_InternFromString("weak");
    return PyModule_Create(&module);
}
