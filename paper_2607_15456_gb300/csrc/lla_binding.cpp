// lla_binding.cpp -- native marshalling of the Python binding's calls (paper_2607_15456_gb300/lla.py).
//
// Each function takes the arguments of the Python function of the same name (with a stream handle or
// None for the current stream), fills the structs of include/lla.h straight from the objects and calls
// liblla with the GIL released.  It handles the ordinary call and nothing else: plain CUDA tensors
// (torch.nn.Parameter among them) that are contiguous, or None, Python ints in range, bf16 or fp32 data.
// Anything else (integer addresses,
// tensor subclasses, host or strided tensors, other types, wrong lengths) returns None, and the caller
// goes through its Python marshalling, which accepts or refuses it as it always did.  No reference is
// kept to any argument.
//
// A call is bound by this on the host: marshalling 24 layers in Python took 95 us beside 25 us of
// kernel, a decode call 13 us; here 5 and 2 us.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <limits>
#include <vector>

#include "lla.h"

namespace {

struct Names {
    PyObject *T, *H, *d, *r_k, *r_v, *storage, *scale;
    PyObject *codec[6];
    PyObject *pool, *num_blocks, *block_table, *max_blocks;
    PyObject *ref_count, *context_lens, *address, *count, *blocks, *device;
    PyObject *base, *pairing, *pairs, *order, *prefix[5];
} names;

struct Unusual {};  // thrown to leave for the Python path

// A new reference that is dropped at the end of its scope.
struct Ref {
    PyObject *o;
    explicit Ref(PyObject *p) : o(p) {
        if (!o) throw Unusual();
    }
    ~Ref() { Py_XDECREF(o); }
    Ref(const Ref &) = delete;
    Ref &operator=(const Ref &) = delete;
};

int64_t integer(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw Unusual();
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &over);
    if (over) throw Unusual();
    return v;
}
int32_t integer32(PyObject *o) {
    const int64_t v = integer(o);
    if (v < std::numeric_limits<int32_t>::min() || v > std::numeric_limits<int32_t>::max()) throw Unusual();
    return static_cast<int32_t>(v);
}
int32_t attr32(PyObject *o, PyObject *name) {
    const Ref r(PyObject_GetAttr(o, name));
    return integer32(r.o);
}
double real(PyObject *o) {
    if (!PyFloat_CheckExact(o)) throw Unusual();
    return PyFloat_AS_DOUBLE(o);
}

const at::Tensor &tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) throw Unusual();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || !t.is_contiguous()) throw Unusual();
    return t;
}
void *address(PyObject *o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }
void *attr_address(PyObject *o, PyObject *name) {
    const Ref r(PyObject_GetAttr(o, name));  // the object keeps the tensor alive
    return address(r.o);
}
lla_dtype dtype(const at::Tensor &t) {
    if (t.scalar_type() == at::kBFloat16) return LLA_BF16;
    if (t.scalar_type() == at::kFloat) return LLA_F32;
    throw Unusual();
}
size_t nbytes(const at::Tensor &t) { return static_cast<size_t>(t.numel()) * t.element_size(); }

lla_geometry geometry(PyObject *o) {
    lla_geometry g;
    g.T = attr32(o, names.T);
    g.H = attr32(o, names.H);
    g.d = attr32(o, names.d);
    g.r_k = attr32(o, names.r_k);
    g.r_v = attr32(o, names.r_v);
    g.block_size = LLA_BLOCK_TOKENS;
    const Ref st(PyObject_GetAttr(o, names.storage)), sc(PyObject_GetAttr(o, names.scale));
    if (!PyUnicode_CheckExact(st.o)) throw Unusual();
    g.storage = PyUnicode_CompareWithASCIIString(st.o, "bf16") == 0 ? LLA_BF16 : LLA_F32;
    if (sc.o == Py_None && g.d <= 0) throw Unusual();
    g.scale = static_cast<float>(sc.o == Py_None ? 1.0 / std::sqrt(static_cast<double>(g.d)) : real(sc.o));
    return g;
}
lla_codec codec(PyObject *o) {
    void *p[6];
    for (int i = 0; i < 6; ++i) p[i] = attr_address(o, names.codec[i]);
    return lla_codec{p[0], p[1], p[2], p[3], static_cast<const float *>(p[4]), static_cast<const float *>(p[5])};
}
lla_cache cache(PyObject *o) {
    lla_cache c;
    c.pool = attr_address(o, names.pool);
    const Ref nb(PyObject_GetAttr(o, names.num_blocks));
    c.num_blocks = integer(nb.o);
    c.block_table = static_cast<const int32_t *>(attr_address(o, names.block_table));
    c.max_blocks_per_seq = attr32(o, names.max_blocks);
    return c;
}
lla_rope rope(PyObject *base, PyObject *pairing) {
    return lla_rope{real(base), static_cast<lla_rope_pairing>(integer32(pairing))};
}
void *stream_of(PyObject *o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    return reinterpret_cast<void *>(static_cast<intptr_t>(integer(o)));
}

// Runs `body` (which marshals, then calls liblla): its status as an int, or None for the Python path.
template <typename F>
PyObject *guarded(Py_ssize_t nargs, Py_ssize_t want, F body) {
    if (nargs != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    int status = 0;
    try {
        status = body();
    } catch (...) {  // Unusual, or an exception of torch (a tensor without storage)
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}

// Releases the GIL for its scope.
struct NoGil {
    PyThreadState *s = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(s); }
};

using DecodeFn = decltype(&lla_decode_attn);
PyObject *decode(DecodeFn fn, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        const at::Tensor &q = tensor(a[6]), &ws = tensor(a[10]);
        if (q.dim() < 1) throw Unusual();
        const auto *ctx = static_cast<const int32_t *>(address(a[3]));
        const int32_t max_ctx = integer32(a[4]), loop = integer32(a[5]), B = static_cast<int32_t>(q.size(0));
        void *ck = address(a[7]), *cv = address(a[8]), *out = address(a[9]), *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[11]);
        NoGil nogil;
        return fn(&g, &cd, &ch, ctx, B, max_ctx, loop, qp, ck, cv, io, out, w, wb, st);
    });
}
PyObject *decode_attn(PyObject *, PyObject *const *a, Py_ssize_t n) { return decode(&lla_decode_attn, a, n); }
PyObject *decode_attn_2d(PyObject *, PyObject *const *a, Py_ssize_t n) { return decode(&lla_decode_attn_2d, a, n); }

PyObject *decode_attn_loops(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        const at::Tensor &q = tensor(a[5]), &ws = tensor(a[9]);
        if (q.dim() < 2) throw Unusual();
        const auto *ctx = static_cast<const int32_t *>(address(a[3]));
        const int32_t max_ctx = integer32(a[4]), B = static_cast<int32_t>(q.size(1));
        void *ck = address(a[6]), *cv = address(a[7]), *out = address(a[8]), *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[10]);
        NoGil nogil;
        return lla_decode_attn_loops(&g, &cd, &ch, ctx, B, max_ctx, qp, ck, cv, io, out, w, wb, st);
    });
}

PyObject *decode_attn_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 14, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        const lla_rope rp = rope(a[3], a[4]);
        const at::Tensor &q = tensor(a[8]), &ws = tensor(a[12]);
        if (q.dim() < 1) throw Unusual();
        const auto *ctx = static_cast<const int32_t *>(address(a[5]));
        const int32_t max_ctx = integer32(a[6]), loop = integer32(a[7]), B = static_cast<int32_t>(q.size(0));
        void *ck = address(a[9]), *cv = address(a[10]), *out = address(a[11]), *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[13]);
        NoGil nogil;
        return lla_decode_attn_rope(&g, &cd, &ch, &rp, ctx, B, max_ctx, loop, qp, ck, cv, io, out, w, wb, st);
    });
}

PyObject *decode_attn_decoupled(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 18, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        void *pool = address(a[3]);
        const int32_t dr = integer32(a[4]);
        const lla_rope rp = rope(a[5], a[6]);
        const at::Tensor &q = tensor(a[10]), &ws = tensor(a[16]);
        if (q.dim() < 1) throw Unusual();
        const auto *ctx = static_cast<const int32_t *>(address(a[7]));
        const int32_t max_ctx = integer32(a[8]), loop = integer32(a[9]), B = static_cast<int32_t>(q.size(0));
        void *qr = address(a[11]), *ck = address(a[12]), *cv = address(a[13]), *ckr = address(a[14]), *out = address(a[15]);
        void *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[17]);
        NoGil nogil;
        return lla_decode_attn_decoupled(&g, &cd, &ch, pool, dr, &rp, ctx, B, max_ctx, loop, qp, qr, ck, cv, ckr, io, out, w,
                                         wb, st);
    });
}

using EncodeFn = decltype(&lla_encode);
PyObject *encode_with(EncodeFn fn, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        const at::Tensor &x = tensor(a[3]);
        void *xk = x.data_ptr(), *xv = address(a[4]);
        const auto *slots = static_cast<const int64_t *>(address(a[5]));
        const int32_t N = x.dim() == 4 ? static_cast<int32_t>(x.size(1)) : 0;
        const lla_dtype xd = dtype(x);
        void *st = stream_of(a[6]);
        NoGil nogil;
        return fn(&g, &cd, &ch, xk, xv, xd, slots, N, st);
    });
}
PyObject *encode(PyObject *, PyObject *const *a, Py_ssize_t n) { return encode_with(&lla_encode, a, n); }
PyObject *encode_2d(PyObject *, PyObject *const *a, Py_ssize_t n) { return encode_with(&lla_encode_2d, a, n); }

PyObject *encode_layers(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const lla_geometry g = geometry(a[0]);
        for (int i = 1; i < 5; ++i)
            if (!PyList_CheckExact(a[i]) && !PyTuple_CheckExact(a[i])) throw Unusual();
        const Py_ssize_t L = PySequence_Fast_GET_SIZE(a[1]);
        if (L < 1 || L > 4096) throw Unusual();
        for (int i = 2; i < 5; ++i)
            if (PySequence_Fast_GET_SIZE(a[i]) != L) throw Unusual();
        std::vector<lla_codec> cds(L);
        std::vector<lla_cache> chs(L);
        std::vector<const void *> xk(L), xv(L);
        // an attribute could run Python code that changes a list, so each item is held while it is read
        auto item = [&](int i, Py_ssize_t l) {
            if (PySequence_Fast_GET_SIZE(a[i]) != L) throw Unusual();
            PyObject *o = PySequence_Fast_GET_ITEM(a[i], l);
            Py_INCREF(o);
            return o;
        };
        for (Py_ssize_t l = 0; l < L; ++l) {
            const Ref c(item(1, l)), h(item(2, l)), k(item(3, l)), v(item(4, l));
            cds[l] = codec(c.o);
            chs[l] = cache(h.o);
            xk[l] = address(k.o);
            xv[l] = address(v.o);
        }
        const Ref first(item(3, 0));
        const at::Tensor &x = tensor(first.o);
        const auto *slots = static_cast<const int64_t *>(address(a[5]));
        const int32_t N = x.dim() == 4 ? static_cast<int32_t>(x.size(1)) : 0;
        const lla_dtype xd = dtype(x);
        void *st = stream_of(a[6]);
        NoGil nogil;
        return lla_encode_layers(&g, static_cast<int32_t>(L), cds.data(), chs.data(), xk.data(), xv.data(), xd, slots, N, st);
    });
}

PyObject *prefill_attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        const at::Tensor &cu = tensor(a[3]), &q = tensor(a[6]);
        if (cu.dim() < 1) throw Unusual();
        const int32_t max_len = integer32(a[4]), loop = integer32(a[5]), B = static_cast<int32_t>(cu.size(0)) - 1;
        const auto *cp = static_cast<const int32_t *>(cu.data_ptr());
        void *qp = q.data_ptr(), *out = address(a[7]);
        const lla_dtype io = dtype(q);
        void *st = stream_of(a[8]);
        NoGil nogil;
        return lla_prefill_attn(&g, &cd, &ch, cp, B, max_len, loop, qp, io, out, st);
    });
}

PyObject *prefill_attn_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const lla_cache ch = cache(a[2]);
        const lla_rope rp = rope(a[3], a[4]);
        const at::Tensor &cu = tensor(a[5]), &q = tensor(a[8]), &ws = tensor(a[10]);
        if (cu.dim() < 1) throw Unusual();
        const int32_t max_len = integer32(a[6]), loop = integer32(a[7]), B = static_cast<int32_t>(cu.size(0)) - 1;
        const auto *cp = static_cast<const int32_t *>(cu.data_ptr());
        void *qp = q.data_ptr(), *out = address(a[9]), *w = ws.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[11]);
        NoGil nogil;
        return lla_prefill_attn_rope(&g, &cd, &ch, &rp, cp, B, max_len, loop, qp, io, out, w, wb, st);
    });
}

// The page and beam calls: tensors of one type and shape on the current device.
const at::Tensor &typed(PyObject *o, at::ScalarType type) {
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != type || t.get_device() != c10::cuda::current_device()) throw Unusual();
    return t;
}
template <typename P>
P *typed_ptr(PyObject *o, at::ScalarType type, int64_t n) {  // n elements in one dimension, or None
    if (o == Py_None) return nullptr;
    const at::Tensor &t = typed(o, type);
    if (t.dim() != 1 || t.size(0) != n) throw Unusual();
    return static_cast<P *>(t.data_ptr());
}
template <typename P>
P *typed_ptr(PyObject *o, at::ScalarType type, int64_t n0, int64_t n1) {
    if (o == Py_None) return nullptr;
    const at::Tensor &t = typed(o, type);
    if (t.dim() != 2 || t.size(0) != n0 || t.size(1) != n1) throw Unusual();
    return static_cast<P *>(t.data_ptr());
}
const at::Tensor &scratch(PyObject *o) {
    const at::Tensor &t = tensor(o);
    if (t.get_device() != c10::cuda::current_device()) throw Unusual();
    return t;
}
int32_t size32(int64_t n) {
    if (n > std::numeric_limits<int32_t>::max()) throw Unusual();
    return static_cast<int32_t>(n);
}
lla_pages pages(PyObject *o) {
    const Ref rc(PyObject_GetAttr(o, names.ref_count)), bt(PyObject_GetAttr(o, names.block_table)),
        cl(PyObject_GetAttr(o, names.context_lens));
    const at::Tensor &r = typed(rc.o, at::kInt), &t = typed(bt.o, at::kInt);
    if (r.dim() != 1 || t.dim() != 2) throw Unusual();
    lla_pages p;
    p.ref_count = static_cast<int32_t *>(r.data_ptr());
    p.num_blocks = r.size(0);
    p.block_table = static_cast<int32_t *>(t.data_ptr());
    p.max_blocks_per_seq = size32(t.size(1));
    p.S = size32(t.size(0));
    p.context_lens = typed_ptr<int32_t>(cl.o, at::kInt, p.S);
    return p;
}
struct PoolArray {
    const lla_pool *p;
    int32_t L;
};
PoolArray pools(PyObject *o, const lla_pages &p) {  // lla.Pools, whose array lives as long as it does
    const Ref ad(PyObject_GetAttr(o, names.address)), n(PyObject_GetAttr(o, names.count)),
        bl(PyObject_GetAttr(o, names.blocks)), dv(PyObject_GetAttr(o, names.device));
    PoolArray a = {reinterpret_cast<const lla_pool *>(static_cast<intptr_t>(integer(ad.o))), integer32(n.o)};
    if (integer(bl.o) < p.num_blocks || (a.L > 0 && integer32(dv.o) != c10::cuda::current_device())) throw Unusual();
    return a;
}

lla_rope_axes rope_axes(PyObject *o) {
    const Ref base(PyObject_GetAttr(o, names.base)), pairs(PyObject_GetAttr(o, names.pairs));
    lla_rope_axes r;
    r.base = real(base.o);
    r.pairing = static_cast<lla_rope_pairing>(attr32(o, names.pairing));
    r.order = static_cast<lla_axes_order>(attr32(o, names.order));
    if (!PyTuple_CheckExact(pairs.o) || PyTuple_GET_SIZE(pairs.o) != LLA_ROPE_AXES) throw Unusual();
    for (int i = 0; i < LLA_ROPE_AXES; ++i) r.pairs[i] = integer32(PyTuple_GET_ITEM(pairs.o, i));
    return r;
}
lla_prefix prefix(PyObject *o, int64_t B) {
    const int64_t rows = LLA_PREFIX_LEVELS * (B / 2 > 1 ? B / 2 : 1);
    const Ref a(PyObject_GetAttr(o, names.prefix[0])), b(PyObject_GetAttr(o, names.prefix[1])), c(PyObject_GetAttr(o, names.prefix[2])),
        d(PyObject_GetAttr(o, names.prefix[3])), e(PyObject_GetAttr(o, names.prefix[4]));
    return lla_prefix{typed_ptr<int32_t>(a.o, at::kInt, 1), typed_ptr<int32_t>(b.o, at::kInt, rows, 4),
                      typed_ptr<int32_t>(c.o, at::kInt, LLA_PREFIX_LEVELS * B), typed_ptr<int32_t>(d.o, at::kInt, LLA_PREFIX_LEVELS, B),
                      typed_ptr<int32_t>(e.o, at::kInt, B)};
}
// A cache whose block table has rows for B sequences.
lla_cache cache_of(PyObject *o, int64_t B) {
    const Ref bt(PyObject_GetAttr(o, names.block_table));
    const at::Tensor &t = typed(bt.o, at::kInt);
    const lla_cache c = cache(o);
    if (t.dim() != 2 || t.size(0) < B || t.size(1) != c.max_blocks_per_seq) throw Unusual();
    return c;
}
// Data of type `type`, n0 x n1 [x n2] values on the current device, or None.
void *values(PyObject *o, at::ScalarType type, int64_t n0, int64_t n1, int64_t n2 = -1) {
    if (o == Py_None) return nullptr;
    const at::Tensor &t = typed(o, type);
    if (t.dim() != (n2 < 0 ? 2 : 3) || t.size(0) != n0 || t.size(1) != n1 || (n2 >= 0 && t.size(2) != n2)) throw Unusual();
    return t.data_ptr();
}

PyObject *encode_rope_keys_axes(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        const int32_t dr = integer32(a[0]);
        const lla_rope_axes rp = rope_axes(a[1]);
        void *pool = address(a[2]);
        const int64_t nb = integer(a[3]);
        const at::Tensor &k = tensor(a[4]);
        if (k.dim() != 2 || k.size(1) != dr) throw Unusual();
        const int32_t N = size32(k.size(0));
        const lla_dtype xd = dtype(k);
        void *kp = k.data_ptr();
        const auto *pos = typed_ptr<int32_t>(a[5], at::kInt, LLA_ROPE_AXES, N);
        const auto *slots = typed_ptr<int64_t>(a[6], at::kLong, N);
        void *st = stream_of(a[7]);
        NoGil nogil;
        return lla_encode_rope_keys_axes(dr, &rp, pool, nb, kp, xd, pos, slots, N, st);
    });
}

PyObject *decode_attn_decoupled_axes(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 18, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        void *pool = address(a[3]);
        const int32_t dr = integer32(a[4]);
        const lla_rope_axes rp = rope_axes(a[5]);
        const at::Tensor &q = typed(a[10], tensor(a[10]).scalar_type()), &ws = scratch(a[16]);
        if (q.dim() != 3 || q.size(1) != g.H || q.size(2) != g.d) throw Unusual();
        const int32_t B = size32(q.size(0));
        const lla_cache ch = cache_of(a[2], B);
        const auto *pos = typed_ptr<int32_t>(a[6], at::kInt, LLA_ROPE_AXES, B), *ctx = typed_ptr<int32_t>(a[7], at::kInt, B);
        const int32_t max_ctx = integer32(a[8]), loop = integer32(a[9]);
        const at::ScalarType t = q.scalar_type();
        void *qr = values(a[11], t, B, g.H, dr), *ck = values(a[12], t, B, g.H, g.d), *cv = values(a[13], t, B, g.H, g.d);
        void *ckr = values(a[14], t, B, dr), *out = values(a[15], t, B, g.H, g.d);
        void *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[17]);
        NoGil nogil;
        return lla_decode_attn_decoupled_axes(&g, &cd, &ch, pool, dr, &rp, pos, ctx, B, max_ctx, loop, qp, qr, ck, cv, ckr, io, out, w, wb,
                                              st);
    });
}

PyObject *prefix_plan(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const at::Tensor &lens = typed(a[1], at::kInt);
        if (lens.dim() != 1) throw Unusual();
        const int32_t B = size32(lens.size(0));
        const lla_cache ch = cache_of(a[0], B);
        const int32_t max_ctx = integer32(a[2]), min_pages = integer32(a[4]);
        const lla_prefix pl = prefix(a[3], B);
        const auto *lp = static_cast<const int32_t *>(lens.data_ptr());
        void *st = stream_of(a[5]);
        NoGil nogil;
        return lla_prefix_plan(&ch, lp, B, max_ctx, min_pages, &pl, st);
    });
}

PyObject *decode_attn_prefix(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        const at::Tensor &q = typed(a[7], tensor(a[7]).scalar_type()), &ws = scratch(a[11]);
        if (q.dim() != 3 || q.size(1) != g.H || q.size(2) != g.d) throw Unusual();
        const int32_t B = size32(q.size(0));
        const lla_cache ch = cache_of(a[2], B);
        const lla_prefix pl = prefix(a[3], B);
        const auto *ctx = typed_ptr<int32_t>(a[4], at::kInt, B);
        const int32_t max_ctx = integer32(a[5]), loop = integer32(a[6]);
        const at::ScalarType t = q.scalar_type();
        void *ck = values(a[8], t, B, g.H, g.d), *cv = values(a[9], t, B, g.H, g.d), *out = values(a[10], t, B, g.H, g.d);
        void *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[12]);
        NoGil nogil;
        return lla_decode_attn_prefix(&g, &cd, &ch, &pl, ctx, B, max_ctx, loop, qp, ck, cv, io, out, w, wb, st);
    });
}

PyObject *decode_attn_prefix_decoupled(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 19, [&] {
        const lla_geometry g = geometry(a[0]);
        const lla_codec cd = codec(a[1]);
        void *pool = address(a[4]);
        const int32_t dr = integer32(a[5]);
        const lla_rope_axes rp = rope_axes(a[6]);
        const at::Tensor &q = typed(a[11], tensor(a[11]).scalar_type()), &ws = scratch(a[17]);
        if (q.dim() != 3 || q.size(1) != g.H || q.size(2) != g.d) throw Unusual();
        const int32_t B = size32(q.size(0));
        const lla_cache ch = cache_of(a[2], B);
        const lla_prefix pl = prefix(a[3], B);
        const auto *pos = typed_ptr<int32_t>(a[7], at::kInt, LLA_ROPE_AXES, B), *ctx = typed_ptr<int32_t>(a[8], at::kInt, B);
        const int32_t max_ctx = integer32(a[9]), loop = integer32(a[10]);
        const at::ScalarType t = q.scalar_type();
        void *qr = values(a[12], t, B, g.H, dr), *ck = values(a[13], t, B, g.H, g.d), *cv = values(a[14], t, B, g.H, g.d);
        void *ckr = values(a[15], t, B, dr), *out = values(a[16], t, B, g.H, g.d);
        void *w = ws.data_ptr(), *qp = q.data_ptr();
        const lla_dtype io = dtype(q);
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[18]);
        NoGil nogil;
        return lla_decode_attn_prefix_decoupled(&g, &cd, &ch, &pl, pool, dr, &rp, pos, ctx, B, max_ctx, loop, qp, qr, ck, cv, ckr, io, out, w,
                                                wb, st);
    });
}

PyObject *pages_admit(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        const lla_pages p = pages(a[0]);
        const PoolArray ps = pools(a[1], p);
        const at::Tensor &rows = typed(a[2], at::kInt), &slots = typed(a[6], at::kLong), &ws = scratch(a[9]);
        const int32_t count = size32(rows.numel()), N = size32(slots.numel());
        const auto *r = typed_ptr<int32_t>(a[2], at::kInt, count), *par = typed_ptr<int32_t>(a[3], at::kInt, count),
                   *keep = typed_ptr<int32_t>(a[4], at::kInt, count), *fresh = typed_ptr<int32_t>(a[5], at::kInt, count);
        auto *sp = static_cast<int64_t *>(slots.data_ptr());
        auto *cu = typed_ptr<int32_t>(a[7], at::kInt, static_cast<int64_t>(count) + 1), *free_blocks = typed_ptr<int32_t>(a[10], at::kInt, 1);
        auto *ok = typed_ptr<uint8_t>(a[8], at::kByte, count);
        void *w = ws.data_ptr();
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[11]);
        NoGil nogil;
        return lla_pages_admit(&p, ps.p, ps.L, r, par, keep, fresh, count, sp, N, cu, ok, free_blocks, w, wb, st);
    });
}

PyObject *pages_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 4, [&] {
        const lla_pages from = pages(a[0]), to = pages(a[1]);
        const auto *parents = typed_ptr<int32_t>(a[2], at::kInt, to.S);
        void *st = stream_of(a[3]);
        NoGil nogil;
        return lla_pages_fork(&from, &to, parents, st);
    });
}

PyObject *pages_extend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        const lla_pages p = pages(a[0]);
        const PoolArray ps = pools(a[1], p);
        const at::Tensor &slots = typed(a[2], at::kLong), &ws = scratch(a[3]);
        const int32_t N = size32(slots.numel());
        auto *sp = static_cast<int64_t *>(slots.data_ptr());
        const auto *cu = typed_ptr<int32_t>(a[4], at::kInt, p.S + 1);
        const auto *skip = typed_ptr<uint8_t>(a[5], at::kByte, p.S);
        auto *before = typed_ptr<int32_t>(a[6], at::kInt, p.S), *free_blocks = typed_ptr<int32_t>(a[7], at::kInt, 1);
        void *w = ws.data_ptr();
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[8]);
        NoGil nogil;
        return lla_pages_extend(&p, ps.p, ps.L, sp, N, cu, skip, before, free_blocks, w, wb, st);
    });
}

PyObject *pages_free(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 3, [&] {
        const lla_pages p = pages(a[0]);
        const at::Tensor &seqs = typed(a[1], at::kInt);
        const int32_t count = size32(seqs.numel());
        const auto *sp = static_cast<const int32_t *>(seqs.data_ptr());
        void *st = stream_of(a[2]);
        NoGil nogil;
        return lla_pages_free(&p, sp, count, st);
    });
}

PyObject *pages_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const lla_pages p = pages(a[0]);
        const PoolArray ps = pools(a[1], p);
        auto *remap = typed_ptr<int32_t>(a[2], at::kInt, p.num_blocks), *live = typed_ptr<int32_t>(a[3], at::kInt, 1);
        const at::Tensor &ws = scratch(a[4]);
        void *w = ws.data_ptr();
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[5]);
        NoGil nogil;
        return lla_pages_compact(&p, ps.p, ps.L, remap, live, w, wb, st);
    });
}

PyObject *beam_select(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        if (!THPVariable_CheckExact(a[0])) throw Unusual();
        const at::Tensor &z = THPVariable_Unpack(a[0]);  // rows may be padded
        if (!z.defined() || !z.is_cuda() || z.get_device() != c10::cuda::current_device() || z.dim() != 3) throw Unusual();
        const int64_t B = z.size(0), W = z.size(1), V = z.size(2);
        const int64_t rows = W > 1 ? z.stride(1) : B > 1 ? z.stride(0) : V;
        if ((V > 1 && z.stride(2) != 1) || (B > 1 && W > 1 && z.stride(0) != W * rows)) throw Unusual();
        const at::Tensor &par = typed(a[2], at::kInt), &ws = scratch(a[5]);
        if (par.dim() != 2 || par.size(0) != B) throw Unusual();
        const int64_t K = par.size(1);
        const int32_t b = size32(B), w = size32(W), v = size32(V), k = size32(K);
        const auto *scores = typed_ptr<float>(a[1], at::kFloat, B, W);
        auto *parents = static_cast<int32_t *>(par.data_ptr()), *tokens = typed_ptr<int32_t>(a[3], at::kInt, B, K);
        auto *out_scores = typed_ptr<float>(a[4], at::kFloat, B, K);
        const auto *finished = typed_ptr<uint8_t>(a[6], at::kByte, B, W);
        const auto *lengths = typed_ptr<int32_t>(a[7], at::kInt, B, W);
        auto *out_finished = typed_ptr<uint8_t>(a[8], at::kByte, B, K);
        auto *out_lengths = typed_ptr<int32_t>(a[9], at::kInt, B, K);
        const int32_t eos = integer32(a[10]);
        const float alpha = static_cast<float>(real(a[11]));
        const lla_dtype zd = dtype(z);
        void *zp = z.data_ptr(), *wp = ws.data_ptr();
        const size_t wb = nbytes(ws);
        void *st = stream_of(a[12]);
        NoGil nogil;
        return lla_beam_select(b, w, v, k, zp, rows, zd, scores, finished, lengths, eos, alpha, parents, tokens, out_scores,
                               out_finished, out_lengths, wp, wb, st);
    });
}

#define LLA_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    LLA_METHOD(decode_attn), LLA_METHOD(decode_attn_2d), LLA_METHOD(decode_attn_loops), LLA_METHOD(decode_attn_rope),
    LLA_METHOD(decode_attn_decoupled), LLA_METHOD(encode), LLA_METHOD(encode_2d), LLA_METHOD(encode_layers),
    LLA_METHOD(prefill_attn), LLA_METHOD(prefill_attn_rope), LLA_METHOD(pages_fork), LLA_METHOD(pages_extend),
    LLA_METHOD(pages_free), LLA_METHOD(pages_compact), LLA_METHOD(beam_select), LLA_METHOD(encode_rope_keys_axes),
    LLA_METHOD(decode_attn_decoupled_axes), LLA_METHOD(prefix_plan), LLA_METHOD(decode_attn_prefix),
    LLA_METHOD(decode_attn_prefix_decoupled), LLA_METHOD(pages_admit), {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lla_native", "Native marshalling of the calls of lla.py.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lla_native() {
    auto s = [](const char *t) { return PyUnicode_InternFromString(t); };
    names = Names{s("T"), s("H"), s("d"), s("r_k"), s("r_v"), s("storage"), s("scale"),
                  {s("w_down_k"), s("w_down_v"), s("w_up_k"), s("w_up_v"), s("mu_k"), s("mu_v")},
                  s("pool"), s("num_blocks"), s("block_table"), s("max_blocks_per_seq"),
                  s("ref_count"), s("context_lens"), s("address"), s("count"), s("blocks"), s("device"),
                  s("base"), s("pairing"), s("pairs"), s("order"),
                  {s("num_groups"), s("groups"), s("members"), s("column"), s("own_page")}};
    return PyModule_Create(&module);
}
