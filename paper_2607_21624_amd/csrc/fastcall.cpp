// fastcall.cpp -- the torch-tensor calls of the Python binding (fbl.py) in
// native code: argument marshalling only, the work is behind the C ABI.
//
// Why: a call through ctypes spends 10 .. 16 us in Python -- building 4 to 9
// layout descriptors, device and dtype checks, 12 to 25 argument conversions --
// and the small calls are bound by it.  Read straight from the tensors the same
// takes under 1 us beside the launches.  Host time of a pass, before and after:
// forward + backward in two launches 29 -> 6.2 us, in four 34 -> 10.4, three
// projection products 31 -> 8.5, a LoRA adapter's six 62 -> 17 (its step 64 ->
// 26 us: now the kernels'); a layer norm's two calls 30 -> 10, one linear layer 20 -> 8.5.
//
// Every function takes all arguments of its namesake by position and either
// does the whole call and returns its result, or does nothing and returns None:
// then the caller runs its own general path, which makes every check and raises
// every error.  So only plain calls are handled here -- exact torch.Tensor (or
// Parameter) arguments in strided device memory on the current device without
// wrapper or lazy-view state, plain Python numbers, the current stream -- and
// an error status of the C ABI (nothing enqueued) also goes back to the caller.
// Nothing is cached.
#include <ATen/ATen.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/hip/HIPFunctions.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "../../include/fbl.h"

#define FBL_STR2(x) #x
#define FBL_STR(x) FBL_STR2(x)
#define FBL_PYTHON FBL_STR(PY_MAJOR_VERSION) "." FBL_STR(PY_MINOR_VERSION)

namespace {

using at::Tensor;

// ------------------------------------------------------------ plain arguments
// A tensor whose memory is what its sizes and strides say: no subclass, no
// functional, batching or grad-tracking wrapper, no conjugate or negative view.
const Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const Tensor& t = THPVariable_Unpack(o);
    static const uint64_t allowed = (c10::DispatchKeySet(c10::DispatchKey::Dense) |
                                     c10::DispatchKeySet(c10::BackendComponent::CUDABit) |
                                     c10::DispatchKeySet(c10::DispatchKey::AutogradFunctionality) |
                                     c10::DispatchKeySet(c10::DispatchKey::ADInplaceOrView) |
                                     c10::DispatchKeySet(c10::DispatchKey::AutocastCUDA))
                                        .raw_repr();
    if (!t.defined() || !t.is_cuda() || (t.key_set().raw_repr() & ~allowed)) return nullptr;
    return &t;
}

// The call's arguments, read one after the other; `ok` falls at the first that is not plain.
struct Args {
    PyObject* const* a;
    bool ok = true;
    int device = -1;  // of the first tensor; all others must be on it
    const Tensor* tensor(int i) {
        const Tensor* t = ok ? plain(a[i]) : nullptr;
        if (!t) return ok = false, nullptr;
        const int d = t->device().index();
        if (device < 0) device = d;
        if (d != device) ok = false;
        return t;
    }
    const Tensor* tensor_or_none(int i) { return a[i] == Py_None ? nullptr : tensor(i); }
    int64_t integer(int i) {
        int overflow = 0;
        if (!ok || !PyLong_CheckExact(a[i])) return ok = false, 0;
        const long long v = PyLong_AsLongLongAndOverflow(a[i], &overflow);
        if (overflow || v < INT32_MIN || v > INT32_MAX) ok = false;
        return v;
    }
    bool flag(int i) {
        if (a[i] != Py_True && a[i] != Py_False) ok = false;
        return a[i] == Py_True;
    }
    float real(int i) {
        if (!PyFloat_CheckExact(a[i])) return ok = false, 0.f;
        return (float)PyFloat_AS_DOUBLE(a[i]);
    }
    // name of an activation
    uint32_t act(int i) {
        static const char* const names[] = {"none", "relu", "gelu", "gelu_tanh", "silu"};
        if (PyUnicode_CheckExact(a[i]))
            for (uint32_t k = 0; k <= FBL_ACT_SILU; ++k)
                if (PyUnicode_CompareWithASCIIString(a[i], names[k]) == 0) return k;
        return ok = false, 0;
    }
    // softmax scale: None is 1 / sqrt(D)
    float scale(int i, int64_t D) {
        if (a[i] == Py_None) return (float)(1.0 / std::sqrt((double)D));
        if (!PyFloat_CheckExact(a[i])) return ok = false, 0.f;
        return (float)PyFloat_AS_DOUBLE(a[i]);
    }
    void no_stream(int i) {
        if (a[i] != Py_None) ok = false;
    }
    bool ready() const { return ok && device >= 0 && (int)c10::hip::current_device() == device; }
    void* stream() const {
        return (void*)c10::hip::getCurrentHIPStreamMasqueradingAsCUDA((c10::DeviceIndex)device).stream();
    }
};

int dtype_code(const Tensor& t) {
    return t.scalar_type() == at::kBFloat16 ? FBL_BF16 : t.scalar_type() == at::kFloat ? FBL_F32 : -1;
}

// Descriptor of a token-major [B, S, H*D] tensor.
bool layout(const Tensor* t, int64_t H, fbl_layout* l) {
    if (!t || t->dim() != 3 || H <= 0 || t->size(2) % H || t->stride(2) != 1 || dtype_code(*t) < 0) return false;
    const int64_t B = t->size(0);
    return fbl_layout_desc(l, dtype_code(*t), B, t->size(1), H, t->size(2) / H, t->stride(1), B > 1 ? t->stride(0) : 0,
                           0) == FBL_OK;
}

// Descriptors and addresses of Q, K, V in a packed [B, S, (Hq + 2 Hkv) D] tensor.
struct Packed {
    fbl_layout q, k, v;
    char *pq, *pk, *pv;
    bool set(const Tensor* t, int64_t Hq, int64_t Hkv) {
        if (!t || t->dim() != 3 || Hq <= 0 || Hkv <= 0 || t->stride(2) != 1 || t->stride(1) != t->size(2) ||
            t->size(2) % (Hq + 2 * Hkv) || dtype_code(*t) < 0)
            return false;
        int64_t ko = 0, vo = 0;
        if (fbl_layout_packed_qkv(&q, &k, &v, &ko, &vo, dtype_code(*t), t->size(0), t->size(1), Hq, Hkv,
                                  t->size(2) / (Hq + 2 * Hkv), t->size(0) > 1 ? t->stride(0) : 0, 0) != FBL_OK)
            return false;
        pq = static_cast<char*>(t->data_ptr());
        pk = pq + ko * (int64_t)t->element_size();
        pv = pq + vo * (int64_t)t->element_size();
        return true;
    }
};

bool kv_len_fits(const Tensor* t, int64_t B) {
    return !t || (t->scalar_type() == at::kInt && t->dim() == 1 && (t->numel() <= 1 || t->stride(0) == 1) &&
                  t->numel() >= B);
}
bool lse_fits(const Tensor* t, int64_t B, int64_t Hq, int64_t S) {
    return !t || (t->scalar_type() == at::kFloat && t->dim() == 3 && t->size(0) == B && t->size(1) == Hq &&
                  t->size(2) == S && t->is_contiguous());
}
fbl_mask mask_of(bool causal, const Tensor* kv_len) {
    fbl_mask m{};
    m.kind = (causal ? FBL_MASK_CAUSAL : 0u) | (kv_len ? FBL_MASK_KEY_PADDING : 0u);
    m.kv_len = kv_len ? static_cast<const int32_t*>(kv_len->data_ptr()) : nullptr;
    return m;
}

// The library call without the interpreter lock (no tensor is read in it).
template <typename F>
fbl_status unlocked(F&& f) {
    PyThreadState* save = PyEval_SaveThread();
    const fbl_status st = f();
    PyEval_RestoreThread(save);
    return st;
}

// Result objects: the caller's own where it gave one, else the new tensor.
PyObject* object_of(PyObject* given, const Tensor& made) {
    if (given != Py_None) return Py_NewRef(given);
    return THPVariable_Wrap(made);
}
template <int N>
PyObject* tuple_of(PyObject* const (&x)[N]) {
    PyObject* t = PyTuple_New(N);
    bool bad = !t;
    for (PyObject* o : x) bad = bad || !o;
    for (int i = 0; i < N; ++i)
        if (!bad) PyTuple_SET_ITEM(t, i, x[i]);
        else Py_XDECREF(x[i]);
    if (bad) Py_CLEAR(t);
    return t;
}

Tensor empty(at::IntArrayRef size, at::ScalarType type, const Tensor& like) {
    return at::empty(size, at::TensorOptions().dtype(type).device(like.device()));
}

// ---------------------------------------------------------------------- calls
// attn_fwd(q, k, v, Hq, Hkv, scale, causal, kv_len, out, lse, stream, tile)
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Args g{a};
    const Tensor *q = g.tensor(0), *k = g.tensor(1), *v = g.tensor(2);
    const int64_t Hq = g.integer(3), Hkv = g.integer(4);
    const bool causal = g.flag(6);
    const Tensor *kv_len = g.tensor_or_none(7), *out = g.tensor_or_none(8), *lse = g.tensor_or_none(9);
    g.no_stream(10);
    const int64_t tile = g.integer(11);
    fbl_layout lq, lk, lv, lo;
    if (!g.ready() || !layout(q, Hq, &lq) || !layout(k, Hkv, &lk) || !layout(v, Hkv, &lv)) Py_RETURN_NONE;
    const float scale = g.scale(5, lq.D);
    if (!g.ok || !kv_len_fits(kv_len, lq.B) || !lse_fits(lse, lq.B, Hq, lq.S)) Py_RETURN_NONE;
    Tensor made_o, made_lse;
    if (!out) made_o = empty(q->sizes(), q->scalar_type(), *q), out = &made_o;
    if (!lse) made_lse = empty({lq.B, Hq, lq.S}, at::kFloat, *q), lse = &made_lse;
    if (!layout(out, Hq, &lo)) Py_RETURN_NONE;
    const fbl_mask m = mask_of(causal, kv_len);
    void *s = g.stream(), *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *po = out->data_ptr();
    float* pl = static_cast<float*>(lse->data_ptr());
    const fbl_status st = unlocked([&] {
        return fbl_attn_fwd_tiled(&lq, pq, &lk, pk, &lv, pv, &lo, po, pl, scale, m, (int32_t)tile, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<2>({object_of(a[8], made_o), object_of(a[9], made_lse)});
    END_HANDLE_TH_ERRORS
}

// attn_bwd(q, k, v, o, do, lse, Hq, Hkv, scale, causal, kv_len, dq, dk, dv, workspace, stream, phases, kv_tile, dq_tile)
PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 19) Py_RETURN_NONE;
    Args g{a};
    const Tensor *q = g.tensor(0), *k = g.tensor(1), *v = g.tensor(2), *o = g.tensor(3), *dO = g.tensor(4);
    const Tensor* lse = g.tensor(5);
    const int64_t Hq = g.integer(6), Hkv = g.integer(7);
    const bool causal = g.flag(9);
    const Tensor *kv_len = g.tensor_or_none(10), *dq = g.tensor_or_none(11), *dk = g.tensor_or_none(12);
    const Tensor *dv = g.tensor_or_none(13), *ws = g.tensor_or_none(14);
    g.no_stream(15);
    const int64_t phases = g.integer(16), kv_tile = g.integer(17), dq_tile = g.integer(18);
    fbl_layout lq, lk, lv, lo, ldo, ldq, ldk, ldv;
    if (!g.ready() || phases < 0 || !layout(q, Hq, &lq) || !layout(k, Hkv, &lk) || !layout(v, Hkv, &lv) ||
        !layout(o, Hq, &lo) || !layout(dO, Hq, &ldo))
        Py_RETURN_NONE;
    const float scale = g.scale(8, lq.D);
    if (!g.ok || !kv_len_fits(kv_len, lq.B) || !lse_fits(lse, lq.B, Hq, lq.S) || (ws && !ws->is_contiguous()))
        Py_RETURN_NONE;
    Tensor made_q, made_k, made_v, made_ws;
    if (!dq) made_q = empty(q->sizes(), q->scalar_type(), *q), dq = &made_q;
    if (!dk) made_k = empty(k->sizes(), k->scalar_type(), *q), dk = &made_k;
    if (!dv) made_v = empty(v->sizes(), v->scalar_type(), *q), dv = &made_v;
    if (!ws) {
        size_t need = 0;
        if (fbl_attn_bwd_workspace(&lq, &lk, &need) != FBL_OK) Py_RETURN_NONE;
        made_ws = empty({(int64_t)need}, at::kByte, *q), ws = &made_ws;
    }
    if (!layout(dq, Hq, &ldq) || !layout(dk, Hkv, &ldk) || !layout(dv, Hkv, &ldv)) Py_RETURN_NONE;
    const fbl_mask m = mask_of(causal, kv_len);
    void *s = g.stream(), *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *po = o->data_ptr();
    void *pg = dO->data_ptr(), *pdq = dq->data_ptr(), *pdk = dk->data_ptr(), *pdv = dv->data_ptr();
    void* pw = ws->data_ptr();
    const float* pl = static_cast<const float*>(lse->data_ptr());
    const size_t ws_bytes = (size_t)(ws->numel() * ws->element_size());
    const fbl_status st = unlocked([&] {
        return fbl_attn_bwd_tiled((uint32_t)phases, &lq, pq, &lk, pk, &lv, pv, &lo, po, &ldo, pg, pl, scale, m, &ldq,
                                  pdq, &ldk, pdk, &ldv, pdv, pw, ws_bytes, (int32_t)kv_tile, (int32_t)dq_tile, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<3>({object_of(a[11], made_q), object_of(a[12], made_k), object_of(a[13], made_v)});
    END_HANDLE_TH_ERRORS
}

// attn_fwd_packed(qkv, Hq, Hkv, scale, causal, kv_len, out, lse, stream)
PyObject* attn_fwd_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Args g{a};
    const Tensor* qkv = g.tensor(0);
    const int64_t Hq = g.integer(1), Hkv = g.integer(2);
    const bool causal = g.flag(4);
    const Tensor *kv_len = g.tensor_or_none(5), *out = g.tensor_or_none(6), *lse = g.tensor_or_none(7);
    g.no_stream(8);
    Packed p;
    fbl_layout lo;
    if (!g.ready() || !p.set(qkv, Hq, Hkv)) Py_RETURN_NONE;
    const float scale = g.scale(3, p.q.D);
    if (!g.ok || !kv_len_fits(kv_len, p.q.B) || !lse_fits(lse, p.q.B, Hq, p.q.S)) Py_RETURN_NONE;
    Tensor made_o, made_lse;
    if (!out) made_o = empty({p.q.B, p.q.S, Hq * p.q.D}, qkv->scalar_type(), *qkv), out = &made_o;
    if (!lse) made_lse = empty({p.q.B, Hq, p.q.S}, at::kFloat, *qkv), lse = &made_lse;
    if (!layout(out, Hq, &lo)) Py_RETURN_NONE;
    const fbl_mask m = mask_of(causal, kv_len);
    void *s = g.stream(), *po = out->data_ptr();
    float* pl = static_cast<float*>(lse->data_ptr());
    const fbl_status st = unlocked(
        [&] { return fbl_attn_fwd(&p.q, p.pq, &p.k, p.pk, &p.v, p.pv, &lo, po, pl, scale, m, s); });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<2>({object_of(a[6], made_o), object_of(a[7], made_lse)});
    END_HANDLE_TH_ERRORS
}

// attn_bwd_packed(qkv, o, do, lse, Hq, Hkv, scale, causal, kv_len, dqkv, workspace, stream)
PyObject* attn_bwd_packed(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Args g{a};
    const Tensor *qkv = g.tensor(0), *o = g.tensor(1), *dO = g.tensor(2), *lse = g.tensor(3);
    const int64_t Hq = g.integer(4), Hkv = g.integer(5);
    const bool causal = g.flag(7);
    const Tensor *kv_len = g.tensor_or_none(8), *dqkv = g.tensor_or_none(9), *ws = g.tensor_or_none(10);
    g.no_stream(11);
    Packed p, d;
    fbl_layout lo, ldo;
    if (!g.ready() || !p.set(qkv, Hq, Hkv) || !layout(o, Hq, &lo) || !layout(dO, Hq, &ldo)) Py_RETURN_NONE;
    const float scale = g.scale(6, p.q.D);
    if (!g.ok || !kv_len_fits(kv_len, p.q.B) || !lse_fits(lse, p.q.B, Hq, p.q.S) || (ws && !ws->is_contiguous()))
        Py_RETURN_NONE;
    Tensor made_d, made_ws;
    if (!dqkv) made_d = empty(qkv->sizes(), qkv->scalar_type(), *qkv), dqkv = &made_d;
    if (dqkv->sizes() != qkv->sizes() || dqkv->strides() != qkv->strides() ||
        dqkv->scalar_type() != qkv->scalar_type() || !d.set(dqkv, Hq, Hkv))
        Py_RETURN_NONE;
    if (!ws) {
        size_t need = 0;
        if (fbl_attn_bwd_workspace(&p.q, &p.k, &need) != FBL_OK) Py_RETURN_NONE;
        made_ws = empty({(int64_t)need}, at::kByte, *qkv), ws = &made_ws;
    }
    const fbl_mask m = mask_of(causal, kv_len);
    void *s = g.stream(), *po = o->data_ptr(), *pg = dO->data_ptr(), *pw = ws->data_ptr();
    const float* pl = static_cast<const float*>(lse->data_ptr());
    const size_t ws_bytes = (size_t)(ws->numel() * ws->element_size());
    const fbl_status st = unlocked([&] {
        return fbl_attn_bwd(&p.q, p.pq, &p.k, p.pk, &p.v, p.pv, &lo, po, &ldo, pg, pl, scale, m, &p.q, d.pq, &p.k, d.pk,
                            &p.v, d.pv, pw, ws_bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return object_of(a[9], made_d);
    END_HANDLE_TH_ERRORS
}

// proj(op, a, b, out, tile, stream)
PyObject* proj(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) Py_RETURN_NONE;
    Args g{a};
    const int64_t op = g.integer(0);
    const Tensor *x = g.tensor(1), *y = g.tensor(2), *out = g.tensor_or_none(3);
    const int64_t tile = g.integer(4);
    g.no_stream(5);
    const auto rows = [](const Tensor* t) { return t->dim() == 2 && t->stride(1) == 1; };
    if (!g.ready() || op < 0 || op > FBL_PROJ_BWD_WEIGHT || !rows(x) || !rows(y) || (out && !rows(out))) Py_RETURN_NONE;
    const int dt = dtype_code(*x);
    if (dt < 0 || y->scalar_type() != x->scalar_type() || (out && out->scalar_type() != x->scalar_type()))
        Py_RETURN_NONE;
    const int64_t M = x->size(0);
    const int64_t K = op == FBL_PROJ_BWD_DATA ? y->size(0) : x->size(1);
    const int64_t N = op == FBL_PROJ_BWD_DATA ? x->size(1) : y->size(1);
    // the extent that both operands state, and the result's shape: the library checks neither
    const int64_t orows = op == FBL_PROJ_BWD_WEIGHT ? K : M, ocols = op == FBL_PROJ_BWD_DATA ? K : N;
    if (op == FBL_PROJ_FWD ? y->size(0) != K : op == FBL_PROJ_BWD_DATA ? y->size(1) != N : y->size(0) != M)
        Py_RETURN_NONE;
    if (out && (out->size(0) != orows || out->size(1) != ocols)) Py_RETURN_NONE;
    Tensor made;
    if (!out) {
        made = empty({orows, ocols}, x->scalar_type(), *x);
        out = &made;
    }
    void *s = g.stream(), *px = x->data_ptr(), *py = y->data_ptr(), *pc = out->data_ptr();
    const int64_t lda = x->stride(0), ldb = y->stride(0), ldc = out->stride(0);
    const fbl_status st = unlocked([&] {
        return fbl_proj_dt((uint32_t)op, dt, M, K, N, px, lda, py, ldb, pc, ldc, (int32_t)tile, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return object_of(a[3], made);
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------- layer norm, linear layers, losses
// (the binding's _matrix, _vector, _head and _scratch)
bool matrix(const Tensor* t, int64_t rows, int64_t width, at::ScalarType type) {
    return !t || (t->dim() == 2 && t->size(0) == rows && t->size(1) == width && t->scalar_type() == type &&
                  (width <= 1 || t->stride(1) == 1));
}
int64_t row_stride(const Tensor* t) {
    return !t ? 0 : t->size(0) > 1 ? t->stride(0) : (t->size(1) + 7) / 8 * 8;
}
bool vector(const Tensor* t, int64_t n, at::ScalarType type) {
    return !t || (t->dim() == 1 && t->size(0) == n && t->scalar_type() == type && (n <= 1 || t->stride(0) == 1));
}
template <typename T = void>
T* data(const Tensor* t) {
    return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}
struct Scratch {
    Tensor made;
    void* p = nullptr;
    size_t bytes = 0;
    // false: not a plain workspace
    bool set(const Tensor* given, size_t need, const Tensor& like) {
        if (given && !given->is_contiguous()) return false;
        if (!given && need) made = empty({(int64_t)need}, at::kByte, like), given = &made;
        if (given) p = given->data_ptr(), bytes = (size_t)(given->numel() * given->element_size());
        return true;
    }
};
PyObject* object_or_none(PyObject* given, const Tensor& made) {
    return given == Py_None && !made.defined() ? Py_NewRef(Py_None) : object_of(given, made);
}

// layer_norm_fwd(x, weight, bias, eps, out, mean, rstd, stream)
PyObject* layer_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 8) Py_RETURN_NONE;
    Args g{a};
    const Tensor *x = g.tensor(0), *w = g.tensor_or_none(1), *b = g.tensor_or_none(2);
    const float eps = g.real(3);
    const Tensor *out = g.tensor_or_none(4), *mean = g.tensor_or_none(5), *rstd = g.tensor_or_none(6);
    g.no_stream(7);
    if (!g.ready() || x->dim() != 2 || dtype_code(*x) < 0) Py_RETURN_NONE;
    const int64_t M = x->size(0), N = x->size(1);
    const at::ScalarType dt = x->scalar_type();
    if (!matrix(x, M, N, dt) || !matrix(out, M, N, dt) || !vector(w, N, dt) || !vector(b, N, dt) || !vector(mean, M, at::kFloat) ||
        !vector(rstd, M, at::kFloat))
        Py_RETURN_NONE;
    Tensor mo, mm, mr;
    if (!out) mo = empty({M, N}, dt, *x), out = &mo;
    if (!mean) mm = empty({M}, at::kFloat, *x), mean = &mm;
    if (!rstd) mr = empty({M}, at::kFloat, *x), rstd = &mr;
    void *s = g.stream(), *px = data(x), *pw = data(w), *pb = data(b), *po = data(out);
    float *pm = data<float>(mean), *pr = data<float>(rstd);
    const int64_t ldx = row_stride(x), ldo = row_stride(out);
    const int code = dtype_code(*x);
    const fbl_status st =
        unlocked([&] { return fbl_layer_norm_fwd(code, M, N, px, ldx, pw, pb, eps, po, ldo, pm, pr, s); });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<3>({object_of(a[4], mo), object_of(a[5], mm), object_of(a[6], mr)});
    END_HANDLE_TH_ERRORS
}

// layer_norm_bwd(dy, x, mean, rstd, weight, dx, dweight, dbias, workspace, stream, need_weight, need_bias)
PyObject* layer_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Args g{a};
    const Tensor *dy = g.tensor(0), *x = g.tensor(1), *mean = g.tensor(2), *rstd = g.tensor(3), *w = g.tensor_or_none(4);
    const Tensor *dx = g.tensor_or_none(5), *dw = g.tensor_or_none(6), *db = g.tensor_or_none(7), *ws = g.tensor_or_none(8);
    g.no_stream(9);
    const bool need_w = g.flag(10), need_b = g.flag(11);
    if (!g.ready() || x->dim() != 2 || dtype_code(*x) < 0) Py_RETURN_NONE;
    const int64_t M = x->size(0), N = x->size(1);
    const at::ScalarType dt = x->scalar_type();
    const int code = dtype_code(*x);
    if (!matrix(x, M, N, dt) || !matrix(dy, M, N, dt) || !matrix(dx, M, N, dt) || !vector(mean, M, at::kFloat) ||
        !vector(rstd, M, at::kFloat) || !vector(w, N, dt) || !vector(dw, N, dt) || !vector(db, N, dt))
        Py_RETURN_NONE;
    Tensor mx, mw, mb;
    if (!dx) mx = empty({M, N}, dt, *x), dx = &mx;
    if (!dw && need_w) mw = empty({N}, dt, *x), dw = &mw;
    if (!db && need_b) mb = empty({N}, dt, *x), db = &mb;
    Scratch sc;
    size_t need = 0;
    if (dw || db) {
        if (!ws && fbl_layer_norm_bwd_workspace(code, M, N, &need) != FBL_OK) Py_RETURN_NONE;
        if (!sc.set(ws, need, *x)) Py_RETURN_NONE;
    }
    void *s = g.stream(), *py = data(dy), *px = data(x), *pw = data(w), *pdx = data(dx), *pdw = data(dw), *pdb = data(db);
    float *pm = data<float>(mean), *pr = data<float>(rstd);
    const int64_t ldy = row_stride(dy), ldx = row_stride(x), lddx = row_stride(dx);
    const fbl_status st = unlocked([&] {
        return fbl_layer_norm_bwd(code, M, N, py, ldy, px, ldx, pw, pm, pr, pdx, lddx, pdw, pdb, sc.p, sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<3>({object_of(a[5], mx), object_or_none(a[6], mw), object_or_none(a[7], mb)});
    END_HANDLE_TH_ERRORS
}

// linear_fwd(x, w, bias, act, residual, out, z, tile, workspace, stream)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) Py_RETURN_NONE;
    Args g{a};
    const Tensor *x = g.tensor(0), *w = g.tensor(1), *b = g.tensor_or_none(2);
    const uint32_t act = g.act(3);
    const Tensor *res = g.tensor_or_none(4), *out = g.tensor_or_none(5), *z = g.tensor_or_none(6);
    const int64_t tile = g.integer(7);
    const Tensor* ws = g.tensor_or_none(8);
    g.no_stream(9);
    if (!g.ready() || x->dim() != 2 || w->dim() != 2 || dtype_code(*x) < 0) Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1), N = w->size(1);
    const at::ScalarType dt = x->scalar_type();
    const int code = dtype_code(*x);
    if (!matrix(x, M, K, dt) || !matrix(w, K, N, dt) || !vector(b, N, dt) || !matrix(res, M, N, dt) || !matrix(out, M, N, dt) ||
        !matrix(z, M, N, dt))
        Py_RETURN_NONE;
    Tensor mo;
    if (!out) mo = empty({M, N}, dt, *x), out = &mo;
    Scratch sc;
    size_t need = 0;
    if (!ws && tile == FBL_GEMM_TILE_AUTO && M <= 128 && fbl_linear_fwd_workspace(code, M, K, N, &need) != FBL_OK) Py_RETURN_NONE;
    if (!sc.set(ws, need, *x)) Py_RETURN_NONE;
    void *s = g.stream(), *px = data(x), *pw = data(w), *pb = data(b), *pr = data(res), *po = data(out), *pz = data(z);
    const int64_t ldx = row_stride(x), ldw = row_stride(w), ldr = row_stride(res), ldo = row_stride(out), ldz = row_stride(z);
    const fbl_status st = unlocked([&] {
        return fbl_linear_fwd(code, act, M, K, N, px, ldx, pw, ldw, pb, pr, ldr, po, ldo, pz, ldz, (int32_t)tile, sc.p, sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return object_of(a[5], mo);
    END_HANDLE_TH_ERRORS
}

// linear_bwd(dy, x, w, z, act, dx, dw, dbias, workspace, stream, need_dx, need_dw, need_bias, x_act, x_z, dxbias)
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 16) Py_RETURN_NONE;
    Args g{a};
    const Tensor *dy = g.tensor(0), *x = g.tensor(1), *w = g.tensor(2), *z = g.tensor_or_none(3);
    const uint32_t act = g.act(4), xact = g.act(13);
    const Tensor *dx = g.tensor_or_none(5), *dw = g.tensor_or_none(6), *db = g.tensor_or_none(7), *ws = g.tensor_or_none(8);
    g.no_stream(9);
    const bool need_x = g.flag(10), need_w = g.flag(11), need_b = g.flag(12);
    const Tensor *xz = g.tensor_or_none(14), *dxb = g.tensor_or_none(15);
    if (!g.ready() || x->dim() != 2 || w->dim() != 2 || dtype_code(*x) < 0) Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1), N = w->size(1);
    const at::ScalarType dt = x->scalar_type();
    const int code = dtype_code(*x);
    if (!matrix(x, M, K, dt) || !matrix(w, K, N, dt) || !matrix(dy, M, N, dt) || !matrix(z, M, N, dt) || !matrix(xz, M, K, dt) ||
        !matrix(dx, M, K, dt) || !matrix(dw, K, N, dt) || !vector(db, N, dt) || !vector(dxb, K, dt))
        Py_RETURN_NONE;
    Tensor mx, mw, mb;
    if (!dx && need_x) mx = empty({M, K}, dt, *x), dx = &mx;
    if (!dw && need_w) mw = empty({K, N}, dt, *x), dw = &mw;
    if (!db && need_b) mb = empty({N}, dt, *x), db = &mb;
    Scratch sc;
    size_t need = 0;
    if (act != FBL_ACT_NONE || db || dxb || ws || (dx && M <= 128) || (dw && K * N <= 1 << 19)) {
        if (!ws && fbl_linear_bwd_workspace(code, M, K, N, &need) != FBL_OK) Py_RETURN_NONE;
        if (!sc.set(ws, need, *x)) Py_RETURN_NONE;
    }
    void *s = g.stream(), *py = data(dy), *px = data(x), *pw = data(w), *pz = data(z), *pxz = data(xz), *pdx = data(dx),
         *pdw = data(dw), *pdb = data(db), *pdxb = data(dxb);
    const int64_t ldy = row_stride(dy), ldx = row_stride(x), ldw = row_stride(w), ldz = row_stride(z), ldxz = row_stride(xz),
                  lddx = row_stride(dx), lddw = row_stride(dw);
    const fbl_status st = unlocked([&] {
        return fbl_linear_bwd(code, act, M, K, N, py, ldy, px, ldx, pw, ldw, pz, ldz, xact, pxz, ldxz, pdx, lddx, pdxb, pdw, lddw,
                              pdb, sc.p, sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<3>({object_or_none(a[5], mx), object_or_none(a[6], mw), object_or_none(a[7], mb)});
    END_HANDLE_TH_ERRORS
}

// A head's weight [K, V]: the way it is stored and its row stride.
bool head(const Tensor* w, const Tensor* x, uint32_t* order, int64_t* ld) {
    if (w->dim() != 2 || w->scalar_type() != x->scalar_type() || w->size(0) != x->size(1)) return false;
    const int64_t K = w->size(0), V = w->size(1);
    if (w->stride(1) == 1 && (K == 1 || w->stride(0) >= V)) {
        *order = FBL_HEAD_KV, *ld = K > 1 ? w->stride(0) : std::max(w->stride(0), V);
        return true;
    }
    if (w->stride(0) != 1 && K != 1) return false;
    *order = FBL_HEAD_VK, *ld = V > 1 ? w->stride(1) : std::max(w->stride(1), K);
    return true;
}
// x [M, K] and w of a loss, their arguments and workspace
struct HeadCall {
    int64_t M, K, V, ldx, ldw;
    uint32_t order;
    int code;
    Scratch sc;
    bool set(const Tensor* x, const Tensor* w, const Tensor* ws, int64_t top) {
        if (x->dim() != 2 || dtype_code(*x) < 0 || !matrix(x, x->size(0), x->size(1), x->scalar_type())) return false;
        if (!head(w, x, &order, &ldw)) return false;
        M = x->size(0), K = x->size(1), V = w->size(1), ldx = row_stride(x), code = dtype_code(*x);
        size_t need = 0;
        if (!ws && fbl_linear_loss_workspace(code, order, M, K, V, top, ldw, &need) != FBL_OK) return false;
        return sc.set(ws, need, *x);
    }
};
// The gradients' tensors: the given ones or new ones
struct HeadGrads {
    Tensor mx, mw;
    const Tensor *dx, *dw;
    int64_t lddx = 0, lddw = 0;
    bool set(const HeadCall& h, const Tensor* x, const Tensor* gx, const Tensor* gw, bool need_x, bool need_w) {
        dx = gx, dw = gw;
        const at::ScalarType dt = x->scalar_type();
        if (!matrix(dx, h.M, h.K, dt)) return false;
        if (!dx && need_x) mx = empty({h.M, h.K}, dt, *x), dx = &mx;
        if (!dw && need_w) mw = h.order == FBL_HEAD_VK ? empty({h.V, h.K}, dt, *x).t() : empty({h.K, h.V}, dt, *x), dw = &mw;
        uint32_t order = h.order;
        if (dw && (!head(dw, x, &order, &lddw) || order != h.order || dw->size(1) != h.V)) return false;
        lddx = row_stride(dx);
        return true;
    }
};
// the loss' gradient: one number, or one a row
bool loss_grad(const Tensor* t, int64_t M, int64_t* stride) {
    if (t->scalar_type() != at::kFloat) return false;
    if (t->dim() == 0) return *stride = 0, true;
    if (t->dim() != 1 || t->size(0) != M) return false;
    return *stride = t->stride(0), true;
}
float* mean_of(const Tensor* t) { return data<float>(t); }
bool mean_fits(const Tensor* t) { return !t || (t->scalar_type() == at::kFloat && t->numel() == 1); }

// linear_ce_fwd(x, w, labels, ignore_index, loss, lse, total, mean, workspace, stream)
PyObject* linear_ce_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 10) Py_RETURN_NONE;
    Args g{a};
    const Tensor *x = g.tensor(0), *w = g.tensor(1), *labels = g.tensor(2);
    const int64_t ignore = g.integer(3);
    const Tensor *loss = g.tensor_or_none(4), *lse = g.tensor_or_none(5), *total = g.tensor_or_none(6), *mean = g.tensor_or_none(7),
                 *ws = g.tensor_or_none(8);
    g.no_stream(9);
    HeadCall h;
    if (!g.ready() || !h.set(x, w, ws, 1) || !vector(labels, h.M, at::kLong) || !vector(loss, h.M, at::kFloat) ||
        !vector(lse, h.M, at::kFloat) || !vector(total, 2, at::kFloat) || !mean_fits(mean))
        Py_RETURN_NONE;
    Tensor ml, me, mt;
    if (!loss) ml = empty({h.M}, at::kFloat, *x), loss = &ml;
    if (!lse) me = empty({h.M}, at::kFloat, *x), lse = &me;
    if (!total) mt = empty({2}, at::kFloat, *x), total = &mt;
    void *s = g.stream(), *px = data(x), *pw = data(w);
    const int64_t* pl = data<int64_t>(labels);
    float *po = data<float>(loss), *pe = data<float>(lse), *pt = data<float>(total), *pm = mean_of(mean);
    const fbl_status st = unlocked([&] {
        return fbl_linear_ce_fwd(h.code, h.order, h.M, h.K, h.V, px, h.ldx, pw, h.ldw, pl, ignore, po, pe, pt, pm, h.sc.p, h.sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<3>({object_of(a[4], ml), object_of(a[5], me), object_of(a[6], mt)});
    END_HANDLE_TH_ERRORS
}

// linear_ce_bwd(dloss, x, w, labels, lse, total, ignore_index, dx, dw, workspace, stream, need_dx, need_dw)
PyObject* linear_ce_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 13) Py_RETURN_NONE;
    Args g{a};
    const Tensor *dl = g.tensor(0), *x = g.tensor(1), *w = g.tensor(2), *labels = g.tensor(3), *lse = g.tensor(4),
                 *total = g.tensor_or_none(5);
    const int64_t ignore = g.integer(6);
    const Tensor *dx = g.tensor_or_none(7), *dw = g.tensor_or_none(8), *ws = g.tensor_or_none(9);
    g.no_stream(10);
    const bool need_x = g.flag(11), need_w = g.flag(12);
    HeadCall h;
    HeadGrads d;
    int64_t ldl = 0;
    if (!g.ready() || !h.set(x, w, ws, 1) || !vector(labels, h.M, at::kLong) || !vector(lse, h.M, at::kFloat) ||
        !vector(total, 2, at::kFloat) || !loss_grad(dl, h.M, &ldl) || !d.set(h, x, dx, dw, need_x, need_w))
        Py_RETURN_NONE;
    void *s = g.stream(), *px = data(x), *pw = data(w), *pdx = data(d.dx), *pdw = data(d.dw);
    const int64_t* pl = data<int64_t>(labels);
    const float *pg = data<float>(dl), *pe = data<float>(lse), *pt = data<float>(total);
    const fbl_status st = unlocked([&] {
        return fbl_linear_ce_bwd(h.code, h.order, h.M, h.K, h.V, pg, ldl, pt, px, h.ldx, pw, h.ldw, pl, ignore, pe, pdx, d.lddx, pdw,
                                 d.lddw, h.sc.p, h.sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<2>({object_or_none(a[7], d.mx), object_or_none(a[8], d.mw)});
    END_HANDLE_TH_ERRORS
}

// linear_kd_fwd(x, w, index, logits, temperature, loss, lse, prob, total, mean, workspace, stream)
PyObject* linear_kd_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 12) Py_RETURN_NONE;
    Args g{a};
    const Tensor *x = g.tensor(0), *w = g.tensor(1), *index = g.tensor(2), *logits = g.tensor(3);
    const float T = g.real(4);
    const Tensor *loss = g.tensor_or_none(5), *lse = g.tensor_or_none(6), *prob = g.tensor_or_none(7), *total = g.tensor_or_none(8),
                 *mean = g.tensor_or_none(9), *ws = g.tensor_or_none(10);
    g.no_stream(11);
    if (!g.ready() || index->dim() != 2 || dtype_code(*logits) < 0) Py_RETURN_NONE;
    const int64_t top = index->size(1);
    HeadCall h;
    if (!h.set(x, w, ws, top) || !matrix(index, h.M, top, at::kLong) || !matrix(logits, h.M, top, logits->scalar_type()) ||
        !vector(loss, h.M, at::kFloat) || !vector(lse, h.M, at::kFloat) || !vector(total, 2, at::kFloat) || !mean_fits(mean) ||
        !matrix(prob, h.M, top, at::kFloat) || (prob && !prob->is_contiguous()))
        Py_RETURN_NONE;
    Tensor ml, me, mp, mt;
    if (!loss) ml = empty({h.M}, at::kFloat, *x), loss = &ml;
    if (!lse) me = empty({h.M}, at::kFloat, *x), lse = &me;
    if (!prob) mp = empty({h.M, top}, at::kFloat, *x), prob = &mp;
    if (!total) mt = empty({2}, at::kFloat, *x), total = &mt;
    void *s = g.stream(), *px = data(x), *pw = data(w), *pz = data(logits);
    const int64_t* pi = data<int64_t>(index);
    float *pp = data<float>(prob), *po = data<float>(loss), *pe = data<float>(lse), *pt = data<float>(total), *pm = mean_of(mean);
    const int64_t ldi = row_stride(index), ldz = row_stride(logits);
    const int zcode = dtype_code(*logits);
    const fbl_status st = unlocked([&] {
        return fbl_linear_kd_fwd(h.code, h.order, h.M, h.K, h.V, top, px, h.ldx, pw, h.ldw, pi, ldi, zcode, pz, ldz, T, pp, po, pe, pt,
                                 pm, h.sc.p, h.sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<4>({object_of(a[5], ml), object_of(a[6], me), object_of(a[7], mp), object_of(a[8], mt)});
    END_HANDLE_TH_ERRORS
}

// linear_kd_bwd(dloss, x, w, index, prob, lse, temperature, total, dx, dw, workspace, stream, need_dx, need_dw)
PyObject* linear_kd_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 14) Py_RETURN_NONE;
    Args g{a};
    const Tensor *dl = g.tensor(0), *x = g.tensor(1), *w = g.tensor(2), *index = g.tensor(3), *prob = g.tensor(4), *lse = g.tensor(5);
    const float T = g.real(6);
    const Tensor *total = g.tensor_or_none(7), *dx = g.tensor_or_none(8), *dw = g.tensor_or_none(9), *ws = g.tensor_or_none(10);
    g.no_stream(11);
    const bool need_x = g.flag(12), need_w = g.flag(13);
    if (!g.ready() || index->dim() != 2) Py_RETURN_NONE;
    const int64_t top = index->size(1);
    HeadCall h;
    HeadGrads d;
    int64_t ldl = 0;
    if (!h.set(x, w, ws, top) || !matrix(index, h.M, top, at::kLong) || !matrix(prob, h.M, top, at::kFloat) || !prob->is_contiguous() ||
        !vector(lse, h.M, at::kFloat) || !vector(total, 2, at::kFloat) || !loss_grad(dl, h.M, &ldl) ||
        !d.set(h, x, dx, dw, need_x, need_w))
        Py_RETURN_NONE;
    void *s = g.stream(), *px = data(x), *pw = data(w), *pdx = data(d.dx), *pdw = data(d.dw);
    const int64_t* pi = data<int64_t>(index);
    const float *pg = data<float>(dl), *pp = data<float>(prob), *pe = data<float>(lse), *pt = data<float>(total);
    const int64_t ldi = row_stride(index);
    const fbl_status st = unlocked([&] {
        return fbl_linear_kd_bwd(h.code, h.order, h.M, h.K, h.V, top, pg, ldl, pt, px, h.ldx, pw, h.ldw, pi, ldi, T, pp, pe, pdx, d.lddx,
                                 pdw, d.lddw, h.sc.p, h.sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<2>({object_or_none(a[8], d.mx), object_or_none(a[9], d.mw)});
    END_HANDLE_TH_ERRORS
}

// ---------------------- norms and rotation of queries and keys, gated layers, clipping
// How a call turns and norms: its arguments from `turns` to `eps` (seven), as the binding's _rotary and _head_norm
// read them.
struct Turning {
    fbl_rotary rot{};
    fbl_head_norm norm{};
    const fbl_rotary* prot = nullptr;
    const fbl_head_norm* pnorm = nullptr;
    const Tensor *wq = nullptr, *wk = nullptr;
    bool set(Args& g, int i, int64_t B, int64_t S, int64_t D, at::ScalarType dt) {
        const Tensor *turns = g.tensor_or_none(i), *pos = g.tensor_or_none(i + 1);
        PyObject* axes = g.a[i + 2];
        const bool neighbours = g.flag(i + 3);
        wq = g.tensor_or_none(i + 4), wk = g.tensor_or_none(i + 5);
        const bool has_norm = g.a[i + 6] != Py_None;
        const float eps = has_norm ? g.real(i + 6) : 0.f;
        if (!g.ok || !vector(wq, D, dt) || !vector(wk, D, dt) || (!has_norm && (wq || wk))) return false;
        if (has_norm) {
            norm.q_weight = data(wq), norm.k_weight = data(wk), norm.eps = eps;
            pnorm = &norm;
        }
        if (!turns) return !pos && axes == Py_None;
        const int64_t pairs = turns->numel();
        if (turns->scalar_type() != at::kLong || turns->dim() != 1 || !turns->is_contiguous() || pairs < 1 || pairs > 64) return false;
        rot.turns = static_cast<const uint64_t*>(turns->data_ptr()), rot.dims = (int32_t)(2 * pairs), rot.neighbours = neighbours;
        rot.num_axes = 1;
        prot = &rot;
        if (!pos) return axes == Py_None;
        const int64_t dim = pos->dim();
        if (pos->scalar_type() != at::kLong || dim < 1 || dim > 3 || pos->size(dim - 1) != S || (dim > 1 && pos->size(dim - 2) != B))
            return false;
        rot.positions = static_cast<const int64_t*>(pos->data_ptr());
        rot.stride_token = pos->stride(dim - 1), rot.stride_batch = dim > 1 ? pos->stride(dim - 2) : 0;
        if (dim == 3) {
            const int64_t n = pos->size(0);
            if (n < 1 || n > FBL_ROTARY_MAX_AXES || (n > 1 && axes == Py_None)) return false;
            rot.num_axes = (int32_t)n, rot.stride_axis = pos->stride(0);
        }
        if (axes == Py_None) return true;
        if (dim != 3 || !PyTuple_CheckExact(axes) || PyTuple_GET_SIZE(axes) != pairs) return false;
        for (int64_t k = 0; k < pairs; ++k) {
            PyObject* o = PyTuple_GET_ITEM(axes, k);
            const long v = PyLong_CheckExact(o) ? PyLong_AsLong(o) : -1;
            if (v == -1 && PyErr_Occurred()) PyErr_Clear();
            if (v < 0 || v >= rot.num_axes) return false;
            rot.axes[k] = (uint8_t)v;
        }
        return true;
    }
};

// qk_norm_rotary_fwd(q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps, q_out, k_out, stream)
PyObject* qk_norm_rotary_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 14) Py_RETURN_NONE;
    Args g{a};
    const Tensor *q = g.tensor(0), *k = g.tensor_or_none(1);
    const int64_t Hq = g.integer(2), Hkv = g.integer(3);
    const Tensor *qo = g.tensor_or_none(11), *ko = g.tensor_or_none(12);
    g.no_stream(13);
    fbl_layout lq, lk, lqo, lko;
    if (!g.ready() || !layout(q, Hq, &lq) || (k && !layout(k, Hkv, &lk)) || (!k && ko)) Py_RETURN_NONE;
    Turning t;
    if (!t.set(g, 4, lq.B, lq.S, lq.D, q->scalar_type()) || !g.ready()) Py_RETURN_NONE;
    Tensor mq, mk;
    if (!qo) mq = empty(q->sizes(), q->scalar_type(), *q), qo = &mq;
    if (k && !ko) mk = empty(k->sizes(), k->scalar_type(), *q), ko = &mk;
    if (!layout(qo, Hq, &lqo) || (k && !layout(ko, Hkv, &lko))) Py_RETURN_NONE;
    void *s = g.stream(), *pq = data(q), *pk = data(k), *pqo = data(qo), *pko = data(ko);
    const fbl_status st = unlocked([&] {
        return fbl_qk_norm_rotary_fwd(&lq, pq, k ? &lk : nullptr, pk, t.prot, t.pnorm, &lqo, pqo, k ? &lko : nullptr, pko, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<2>({object_of(a[11], mq), object_or_none(a[12], mk)});
    END_HANDLE_TH_ERRORS
}

// qk_norm_rotary_bwd(dq_out, dk_out, q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps, dq, dk,
//                    dq_weight, dk_weight, workspace, stream, need_weights)
PyObject* qk_norm_rotary_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 20) Py_RETURN_NONE;
    Args g{a};
    const Tensor *gq = g.tensor(0), *gk = g.tensor_or_none(1);
    const int64_t Hq = g.integer(4), Hkv = g.integer(5);
    const bool norm = a[12] != Py_None;
    const Tensor *q = norm ? g.tensor(2) : nullptr, *k = norm ? g.tensor_or_none(3) : nullptr;
    const Tensor *dq = g.tensor_or_none(13), *dk = g.tensor_or_none(14), *dqw = g.tensor_or_none(15), *dkw = g.tensor_or_none(16);
    const Tensor* ws = g.tensor_or_none(17);
    g.no_stream(18);
    const bool need = g.flag(19);
    fbl_layout lgq, lgk, lq, lk, ldq, ldk;
    if (!g.ready() || !layout(gq, Hq, &lgq) || (gk && !layout(gk, Hkv, &lgk)) || (!gk && dk)) Py_RETURN_NONE;
    if (norm && (!layout(q, Hq, &lq) || !k != !gk || (k && !layout(k, Hkv, &lk)))) Py_RETURN_NONE;
    Turning t;
    const at::ScalarType dt = gq->scalar_type();
    if (!t.set(g, 6, lgq.B, lgq.S, lgq.D, dt) || !vector(dqw, lgq.D, dt) || !vector(dkw, lgq.D, dt) || !g.ready()) Py_RETURN_NONE;
    Tensor mq, mk, mqw, mkw;
    if (!dq) mq = empty(gq->sizes(), dt, *gq), dq = &mq;
    if (gk && !dk) mk = empty(gk->sizes(), gk->scalar_type(), *gq), dk = &mk;
    if (need && !dqw && t.wq) mqw = empty({lgq.D}, dt, *gq), dqw = &mqw;
    if (need && !dkw && t.wk && gk) mkw = empty({lgq.D}, dt, *gq), dkw = &mkw;
    if (!layout(dq, Hq, &ldq) || (gk && !layout(dk, Hkv, &ldk))) Py_RETURN_NONE;
    Scratch sc;
    size_t bytes = 0;
    if (dqw || dkw) {
        if (!ws && fbl_qk_norm_rotary_bwd_workspace(&lgq, gk ? &lgk : nullptr, &bytes) != FBL_OK) Py_RETURN_NONE;
        if (!sc.set(ws, bytes, *gq)) Py_RETURN_NONE;
    }
    void *s = g.stream(), *pgq = data(gq), *pgk = data(gk), *pq = data(q), *pk = data(k), *pdq = data(dq), *pdk = data(dk),
         *pdqw = data(dqw), *pdkw = data(dkw);
    const fbl_status st = unlocked([&] {
        return fbl_qk_norm_rotary_bwd(&lgq, pgq, gk ? &lgk : nullptr, pgk, q ? &lq : nullptr, pq, k ? &lk : nullptr, pk, t.prot, t.pnorm,
                                      &ldq, pdq, gk ? &ldk : nullptr, pdk, pdqw, pdkw, sc.p, sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<4>({object_of(a[13], mq), object_or_none(a[14], mk), object_or_none(a[15], mqw), object_or_none(a[16], mkw)});
    END_HANDLE_TH_ERRORS
}

// gated_fwd(x, w, bias, act, out, factors, tile, workspace, stream)
PyObject* gated_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Args g{a};
    const Tensor *x = g.tensor(0), *w = g.tensor(1), *b = g.tensor_or_none(2);
    const uint32_t act = g.act(3);
    const Tensor *out = g.tensor_or_none(4), *f = g.tensor_or_none(5);
    const int64_t tile = g.integer(6);
    const Tensor* ws = g.tensor_or_none(7);
    g.no_stream(8);
    if (!g.ready() || x->dim() != 2 || w->dim() != 2 || w->size(1) % 2 || dtype_code(*x) < 0) Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1), F = w->size(1) / 2;
    const at::ScalarType dt = x->scalar_type();
    const int code = dtype_code(*x);
    if (!matrix(x, M, K, dt) || !matrix(w, K, 2 * F, dt) || !vector(b, 2 * F, dt) || !matrix(out, M, F, dt) || !matrix(f, M, 2 * F, dt))
        Py_RETURN_NONE;
    Tensor mo;
    if (!out) mo = empty({M, F}, dt, *x), out = &mo;
    Scratch sc;
    size_t need = 0;
    if (!ws && tile == FBL_GEMM_TILE_AUTO && M <= 128 && fbl_gated_fwd_workspace(code, M, K, F, &need) != FBL_OK) Py_RETURN_NONE;
    if (!sc.set(ws, need, *x)) Py_RETURN_NONE;
    void *s = g.stream(), *px = data(x), *pw = data(w), *pb = data(b), *po = data(out), *pf = data(f);
    const int64_t ldx = row_stride(x), ldw = row_stride(w), ldo = row_stride(out), ldf = row_stride(f);
    const fbl_status st = unlocked([&] {
        return fbl_gated_fwd(code, act, M, K, F, px, ldx, pw, ldw, pb, po, ldo, pf, ldf, (int32_t)tile, sc.p, sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return object_of(a[4], mo);
    END_HANDLE_TH_ERRORS
}

// gated_bwd(dy, w_down, factors, dz, dbias, tile, workspace, stream, need_bias)
PyObject* gated_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 9) Py_RETURN_NONE;
    Args g{a};
    const Tensor *dy = g.tensor(0), *wd = g.tensor(1), *f = g.tensor(2);
    const Tensor *dz = g.tensor_or_none(3), *db = g.tensor_or_none(4);
    const int64_t tile = g.integer(5);
    const Tensor* ws = g.tensor_or_none(6);
    g.no_stream(7);
    const bool need_b = g.flag(8);
    if (!g.ready() || dy->dim() != 2 || wd->dim() != 2 || dtype_code(*dy) < 0) Py_RETURN_NONE;
    const int64_t M = dy->size(0), N = dy->size(1), F = wd->size(0);
    const at::ScalarType dt = dy->scalar_type();
    const int code = dtype_code(*dy);
    if (!matrix(dy, M, N, dt) || !matrix(wd, F, N, dt) || !matrix(f, M, 2 * F, dt) || !matrix(dz, M, 2 * F, dt) || !vector(db, 2 * F, dt))
        Py_RETURN_NONE;
    Tensor mz, mb;
    if (!dz) mz = empty({M, 2 * F}, dt, *dy), dz = &mz;
    if (!db && need_b) mb = empty({2 * F}, dt, *dy), db = &mb;
    Scratch sc;
    size_t need = 0;
    if (db || ws || M <= 128) {
        if (!ws && fbl_gated_bwd_workspace(code, M, F, N, &need) != FBL_OK) Py_RETURN_NONE;
        if (!sc.set(ws, need, *dy)) Py_RETURN_NONE;
    }
    void *s = g.stream(), *py = data(dy), *pwd = data(wd), *pf = data(f), *pdz = data(dz), *pdb = data(db);
    const int64_t ldy = row_stride(dy), ldwd = row_stride(wd), ldf = row_stride(f), lddz = row_stride(dz);
    const fbl_status st = unlocked([&] {
        return fbl_gated_bwd(code, M, F, N, py, ldy, pwd, ldwd, pf, ldf, pdz, lddz, pdb, (int32_t)tile, sc.p, sc.bytes, s);
    });
    if (st != FBL_OK) Py_RETURN_NONE;
    return tuple_of<2>({object_of(a[3], mz), object_or_none(a[4], mb)});
    END_HANDLE_TH_ERRORS
}

// A list (or tuple) of gradients and of the tensors that receive them, as the binding's _grad_list reads it.
struct Grads {
    std::vector<fbl_grad> list;
    const Tensor* first = nullptr;
    static Py_ssize_t size(PyObject* o) {
        return PyList_CheckExact(o) ? PyList_GET_SIZE(o) : PyTuple_CheckExact(o) ? PyTuple_GET_SIZE(o) : -1;
    }
    static PyObject* item(PyObject* o, Py_ssize_t i) { return PyList_CheckExact(o) ? PyList_GET_ITEM(o, i) : PyTuple_GET_ITEM(o, i); }
    bool set(Args& g, PyObject* grads, PyObject* out) {
        const Py_ssize_t n = size(grads);
        if (n < 1 || (out != Py_None && size(out) != n)) return false;
        list.resize((size_t)n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject* const given = item(grads, i);
            const Tensor* t = plain(given);
            if (!t || t->layout() != c10::kStrided || dtype_code(*t) < 0 || !t->is_non_overlapping_and_dense()) return false;
            if (g.device < 0) g.device = t->device().index();
            if (t->device().index() != g.device) return false;
            if (!first) first = t;
            fbl_grad& e = list[(size_t)i];
            e = fbl_grad{t->data_ptr(), t->data_ptr(), t->numel(), dtype_code(*t), 0};
            if (out == Py_None) continue;
            const Tensor* o = plain(item(out, i));
            if (!o || o->scalar_type() != t->scalar_type() || o->sizes() != t->sizes() || o->strides() != t->strides() ||
                o->device().index() != g.device)
                return false;
            e.out = o->data_ptr();
        }
        return true;
    }
};
bool one_float(const Tensor* t) { return !t || (t->scalar_type() == at::kFloat && t->numel() == 1); }

// grad_norm(grads, norm, workspace, stream)
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 4) Py_RETURN_NONE;
    Args g{a};
    const Tensor *norm = g.tensor_or_none(1), *ws = g.tensor_or_none(2);
    g.no_stream(3);
    Grads l;
    if (!g.ok || !l.set(g, a[0], Py_None) || !g.ready() || !one_float(norm)) Py_RETURN_NONE;
    Tensor made;
    if (!norm) made = empty({}, at::kFloat, *l.first), norm = &made;
    Scratch sc;
    size_t need = 0;
    const int64_t count = (int64_t)l.list.size();
    if ((!ws && fbl_grad_norm_workspace(count, &need) != FBL_OK) || !sc.set(ws, need, *l.first)) Py_RETURN_NONE;
    void* s = g.stream();
    float* pn = data<float>(norm);
    const fbl_status st = unlocked([&] { return fbl_grad_norm(count, l.list.data(), pn, sc.p, sc.bytes, s); });
    if (st != FBL_OK) Py_RETURN_NONE;
    return object_of(a[1], made);
    END_HANDLE_TH_ERRORS
}

// clip_grad_norm(grads, limit, out, norm, workspace, stream)
PyObject* clip_grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6) Py_RETURN_NONE;
    Args g{a};
    const float limit = g.real(1);
    const Tensor *norm = g.tensor_or_none(3), *ws = g.tensor_or_none(4);
    g.no_stream(5);
    Grads l;
    if (!g.ok || !l.set(g, a[0], a[2]) || !g.ready() || !one_float(norm)) Py_RETURN_NONE;
    Tensor made;
    if (!norm) made = empty({}, at::kFloat, *l.first), norm = &made;
    Scratch sc;
    size_t need = 0;
    const int64_t count = (int64_t)l.list.size();
    if ((!ws && fbl_grad_norm_workspace(count, &need) != FBL_OK) || !sc.set(ws, need, *l.first)) Py_RETURN_NONE;
    void* s = g.stream();
    float* pn = data<float>(norm);
    const fbl_status st = unlocked([&] { return fbl_clip_grad_norm(count, l.list.data(), limit, pn, sc.p, sc.bytes, s); });
    if (st != FBL_OK) Py_RETURN_NONE;
    return object_of(a[3], made);
    END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {
    {"attn_fwd", (PyCFunction)(void (*)())attn_fwd, METH_FASTCALL, nullptr},
    {"attn_bwd", (PyCFunction)(void (*)())attn_bwd, METH_FASTCALL, nullptr},
    {"attn_fwd_packed", (PyCFunction)(void (*)())attn_fwd_packed, METH_FASTCALL, nullptr},
    {"attn_bwd_packed", (PyCFunction)(void (*)())attn_bwd_packed, METH_FASTCALL, nullptr},
    {"proj", (PyCFunction)(void (*)())proj, METH_FASTCALL, nullptr},
    {"layer_norm_fwd", (PyCFunction)(void (*)())layer_norm_fwd, METH_FASTCALL, nullptr},
    {"layer_norm_bwd", (PyCFunction)(void (*)())layer_norm_bwd, METH_FASTCALL, nullptr},
    {"linear_fwd", (PyCFunction)(void (*)())linear_fwd, METH_FASTCALL, nullptr},
    {"linear_bwd", (PyCFunction)(void (*)())linear_bwd, METH_FASTCALL, nullptr},
    {"linear_ce_fwd", (PyCFunction)(void (*)())linear_ce_fwd, METH_FASTCALL, nullptr},
    {"linear_ce_bwd", (PyCFunction)(void (*)())linear_ce_bwd, METH_FASTCALL, nullptr},
    {"linear_kd_fwd", (PyCFunction)(void (*)())linear_kd_fwd, METH_FASTCALL, nullptr},
    {"linear_kd_bwd", (PyCFunction)(void (*)())linear_kd_bwd, METH_FASTCALL, nullptr},
    {"qk_norm_rotary_fwd", (PyCFunction)(void (*)())qk_norm_rotary_fwd, METH_FASTCALL, nullptr},
    {"qk_norm_rotary_bwd", (PyCFunction)(void (*)())qk_norm_rotary_bwd, METH_FASTCALL, nullptr},
    {"gated_fwd", (PyCFunction)(void (*)())gated_fwd, METH_FASTCALL, nullptr},
    {"gated_bwd", (PyCFunction)(void (*)())gated_bwd, METH_FASTCALL, nullptr},
    {"grad_norm", (PyCFunction)(void (*)())grad_norm, METH_FASTCALL, nullptr},
    {"clip_grad_norm", (PyCFunction)(void (*)())clip_grad_norm, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and Python versions, for the binding to compare before it
// makes a call here (their headers' struct layouts are compiled in).
PyMODINIT_FUNC PyInit__fastcall(void) {
    PyObject* m = PyModule_Create(&kModule);
    PyObject* v = m ? Py_BuildValue("(ss)", TORCH_VERSION, FBL_PYTHON) : nullptr;
    if (v && PyModule_AddObject(m, "built_for", v) == 0) return m;
    Py_XDECREF(v);
    Py_XDECREF(m);
    return nullptr;
}
