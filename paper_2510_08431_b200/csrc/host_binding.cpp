// Tensor checks, output allocation and the call into the C ABI for the entry points whose kernels take microseconds: a
// CPython module, because there the marshalling in Python took several times as long as the kernel (a call of the fused
// adaLN step 14 us of host time, half of it in attribute reads, allocations and ctypes).  Nothing is computed here, and the
// library's functions come in as addresses (bind()), so that this module depends on no particular build of it.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <stdexcept>
#include <vector>

#include "attn_jvp.h"

namespace {

decltype(&attn_jvp_adaln_fwd) f_adaln_fwd = nullptr;
decltype(&attn_jvp_adaln_bwd) f_adaln_bwd = nullptr;
decltype(&attn_jvp_adaln_bwd_workspace_bytes) f_adaln_bwd_bytes = nullptr;
decltype(&attn_jvp_block_select) f_block_select = nullptr;
decltype(&attn_jvp_block_select_workspace_bytes) f_block_select_bytes = nullptr;
decltype(&attn_jvp_block_lists) f_block_lists = nullptr;
decltype(&attn_jvp_sparse_fwd) f_sparse_fwd = nullptr;
decltype(&attn_jvp_sparse_bwd) f_sparse_bwd = nullptr;
decltype(&attn_jvp_sparse_bwd_workspace_bytes) f_sparse_bwd_bytes = nullptr;
decltype(&attn_jvp_fwd_stream) f_fwd_stream = nullptr;
decltype(&attn_jvp_fwd_mu) f_fwd_mu = nullptr;
decltype(&attn_jvp_attention_fwd) f_attention_fwd = nullptr;
decltype(&attn_jvp_attention_bwd) f_attention_bwd = nullptr;
decltype(&attn_jvp_attention_bwd_workspace_bytes) f_attention_bwd_bytes = nullptr;
decltype(&attn_jvp_rotary_table) f_rotary_table = nullptr;
decltype(&attn_jvp_qk_rotary_fwd) f_qk_rotary_fwd = nullptr;
decltype(&attn_jvp_qk_rotary_bwd) f_qk_rotary_bwd = nullptr;
decltype(&attn_jvp_qk_rotary_bwd_workspace_bytes) f_qk_rotary_bwd_bytes = nullptr;

// An argument that does not fit: becomes a ValueError.
struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };
[[noreturn]] void refuse(const char* format, ...) {
    char text[256];
    va_list args;
    va_start(args, format);
    vsnprintf(text, sizeof text, format, args);
    va_end(args);
    throw Refused(text);
}

// The tensor behind an argument; undefined for None.
at::Tensor tensor(PyObject* o, const char* name) {
    if (o == Py_None) return at::Tensor();
    if (!THPVariable_Check(o)) refuse("%s must be a tensor or None", name);
    return THPVariable_Unpack(o);
}
at::Tensor required(PyObject* o, const char* name) {
    at::Tensor t = tensor(o, name);
    if (!t.defined()) refuse("%s is required", name);
    return t;
}
PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
// A contiguous tensor of this type, shape and device.
void expect(const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape, const at::Device& device) {
    if (t.device() != device || t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
        refuse("%s must be a contiguous %s tensor on %s of the shape that the other arguments give", name, c10::toString(type), device.str().c_str());
}
void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
template <typename T>
T* ptr(const at::Tensor& t) { return static_cast<T*>(ptr(t)); }
at::Tensor like(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType type) { return at::empty(shape, t.options().dtype(type).requires_grad(false)); }
at::Tensor same(const at::Tensor& t) { return like(t, t.sizes(), t.scalar_type()); }
// A caller's workspace, or one of `need` bytes.
at::Tensor scratch(PyObject* o, const at::Tensor& on, size_t need) {
    at::Tensor w = tensor(o, "workspace");
    if (!w.defined()) return like(on, {static_cast<int64_t>(need)}, at::kByte);
    if (w.device() != on.device() || !w.is_contiguous()) refuse("workspace must be contiguous and on %s", on.device().str().c_str());
    return w;
}
int size32(int64_t v) { return v > 0x7fffffff ? 0x7fffffff : static_cast<int>(v); }      // (sizes that large are refused by the library)

// What every function does around its body: exceptions become Python's (torch's own those that it raises for them, as
// torch.OutOfMemoryError), and nothing gets past this point.
template <typename F>
PyObject* guarded(F&& body) {
    try {
        return body();
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}
bool count(Py_ssize_t n, Py_ssize_t want, const char* name) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%s takes %zd arguments", name, want);
    return n == want;
}
PyObject* result(int rc, std::initializer_list<at::Tensor> out) {
    PyObject* t = PyTuple_New(1 + static_cast<Py_ssize_t>(out.size()));
    PyTuple_SET_ITEM(t, 0, PyLong_FromLong(rc));
    Py_ssize_t i = 1;
    for (const at::Tensor& o : out) PyTuple_SET_ITEM(t, i++, wrap(o));
    return t;
}
// Without the interpreter's lock: a launch waits where the stream's queue is full.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F>
int unlocked(F&& call) {
    Unlocked u;
    return call();
}
double number(PyObject* o, const char* name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse("%s must be a number", name);
    }
    return v;
}
int whole(PyObject* o, const char* name) {
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if ((v == -1 && PyErr_Occurred()) || overflow) {
        PyErr_Clear();
        refuse("%s must be a whole number", name);
    }
    return v > 0x7fffffffL ? 0x7fffffff : v < -0x7fffffffL ? -0x7fffffff : static_cast<int>(v);
}

// ---- adaln ----
// args: x, h, gate, scale, shift, weight, post_weight, norm, post_norm, eps
struct Adaln {
    at::Tensor x, h, gate, scale, shift, w, wp;
    attn_jvp_adaln_t a = {};
    explicit Adaln(PyObject* const* p) {
        x = required(p[0], "x");
        if (!x.is_cuda() || x.dim() != 3) refuse("x must be a CUDA tensor [B][L][C]");
        const auto type = x.scalar_type();
        if ((type != at::kBFloat16 && type != at::kFloat) || !x.is_contiguous()) refuse("x must be contiguous, bf16 or fp32");
        h = tensor(p[1], "h");
        gate = tensor(p[2], "gate");
        scale = tensor(p[3], "scale");
        shift = tensor(p[4], "shift");
        w = tensor(p[5], "weight");
        wp = tensor(p[6], "post_weight");
        a.B = size32(x.size(0));
        a.L = size32(x.size(1));
        a.C = size32(x.size(2));
        a.x_dtype = type == at::kFloat ? ATTN_JVP_FP32 : ATTN_JVP_BF16;
        a.norm = whole(p[7], "norm");
        a.post_norm = whole(p[8], "post_norm");
        a.eps = static_cast<float>(number(p[9], "eps"));
        if (!h.defined() && (gate.defined() || wp.defined() || a.post_norm != ATTN_JVP_NORM_NONE)) refuse("gate, post_norm and post_weight act on h, which is None");
        if (a.norm == ATTN_JVP_NORM_NONE && (scale.defined() || shift.defined() || w.defined())) refuse("scale, shift and weight act on the norm's result, and norm is None");
        if (h.defined()) expect(h, "h", at::kBFloat16, x.sizes(), x.device());
        for (auto* v : {&w, &wp}) if (v->defined()) expect(*v, v == &w ? "weight" : "post_weight", at::kFloat, {x.size(2)}, x.device());
        a.x = ptr(x);
        a.h = ptr(h);
        row(gate, "gate", a.gate, a.gate_stride);
        row(scale, "scale", a.scale, a.scale_stride);
        row(shift, "shift", a.shift, a.shift_stride);
        a.weight = ptr<float>(w);
        a.post_weight = ptr<float>(wp);
    }
    // a modulation row per batch
    void row(const at::Tensor& t, const char* name, const float*& p, long long& stride) const {
        if (!t.defined()) return;
        if (t.device() != x.device() || t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != x.size(0) || t.size(1) != x.size(2) ||
            (t.stride(1) != 1 && t.size(1) > 1))
            refuse("%s must be fp32 of shape [%d][%d] on %s with contiguous rows", name, a.B, a.C, x.device().str().c_str());
        p = ptr<float>(t);
        stride = a.B > 1 ? t.stride(0) : 0;
    }
};

// ... , tx, th, tgate, tscale, tshift -> (rc, x', y, tx', ty); x' and tx' None without h
PyObject* adaln_fwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 15, "adaln_fwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Adaln c(p);
        at::Tensor tx = tensor(p[10], "tx"), th = tensor(p[11], "th"), tg = tensor(p[12], "tgate"), ts = tensor(p[13], "tscale"), tb = tensor(p[14], "tshift");
        const bool jvp = tx.defined() || th.defined() || tg.defined() || ts.defined() || tb.defined();
        const bool norm = c.a.norm != ATTN_JVP_NORM_NONE;
        if (!c.h.defined() && !norm) refuse("neither h nor norm: nothing to compute");
        if (jvp) {
            if (!tx.defined() || th.defined() != c.h.defined()) refuse("with tangents tx is required, and th exactly where h is given");
            if ((!c.h.defined() && tg.defined()) || (!norm && (ts.defined() || tb.defined()))) refuse("a tangent of something that does not act");
            expect(tx, "tx", c.x.scalar_type(), c.x.sizes(), c.x.device());
            if (th.defined()) expect(th, "th", at::kBFloat16, c.x.sizes(), c.x.device());
            c.a.tx = ptr(tx);
            c.a.th = ptr(th);
            c.row(tg, "tgate", c.a.tgate, c.a.tgate_stride);
            c.row(ts, "tscale", c.a.tscale, c.a.tscale_stride);
            c.row(tb, "tshift", c.a.tshift, c.a.tshift_stride);
        }
        at::Tensor xn, y, txn, ty;
        if (c.h.defined()) xn = same(c.x);
        if (norm) y = like(c.x, c.x.sizes(), at::kBFloat16);
        if (jvp && c.h.defined()) txn = same(c.x);
        if (jvp && norm) ty = like(c.x, c.x.sizes(), at::kBFloat16);
        const c10::cuda::CUDAGuard guard(c.x.device());
        const int rc = unlocked([&] { return f_adaln_fwd(&c.a, ptr(xn), ptr(y), ptr(txn), ptr(ty), c10::cuda::getCurrentCUDAStream(c.x.device().index()).stream()); });
        return result(rc, {xn, y, txn, ty});
    });
}

// dx_new, dy, (the ten of Adaln), workspace -> (rc, dx, dh, dgate, dscale, dshift, dweight, dpost_weight)
PyObject* adaln_bwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 13, "adaln_bwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        at::Tensor dxn = tensor(p[0], "dx_new"), dy = tensor(p[1], "dy");
        Adaln c(p + 2);
        const at::Device dev = c.x.device();
        if (dxn.defined()) expect(dxn, "dx_new", c.x.scalar_type(), c.x.sizes(), dev);
        if (dy.defined()) {
            if (c.a.norm == ATTN_JVP_NORM_NONE) refuse("dy given, but norm is None");
            expect(dy, "dy", at::kBFloat16, c.x.sizes(), dev);
        }
        const int64_t B = c.x.size(0), C = c.x.size(2);
        at::Tensor dx = same(c.x), dh, dg, ds, db, dw, dwp;
        if (c.h.defined()) dh = same(c.h);
        if (c.gate.defined()) dg = like(c.x, {B, C}, at::kFloat);
        if (c.scale.defined()) ds = like(c.x, {B, C}, at::kFloat);
        if (c.shift.defined()) db = like(c.x, {B, C}, at::kFloat);
        if (c.w.defined()) dw = like(c.x, {C}, at::kFloat);
        if (c.wp.defined()) dwp = like(c.x, {C}, at::kFloat);
        at::Tensor ws = scratch(p[12], c.x, f_adaln_bwd_bytes(c.a.B, c.a.L, c.a.C));
        const c10::cuda::CUDAGuard guard(dev);
        const int rc = unlocked([&] { return f_adaln_bwd(&c.a, ptr(dxn), ptr(dy), ptr(dx), ptr(dh), ptr<float>(dg), ptr<float>(ds), ptr<float>(db), ptr<float>(dw), ptr<float>(dwp),
                                   ptr(ws), ws.nbytes(), c10::cuda::getCurrentCUDAStream(dev.index()).stream()); });
        return result(rc, {dx, dh, dg, ds, db, dw, dwp});
    });
}

// ---- attention over selected key blocks ----
struct Qkv {
    at::Tensor q, k, v;
    int B, H, Lq, Lk, D;
    Qkv(PyObject* pq, PyObject* pk, PyObject* pv) : q(required(pq, "q")), k(required(pk, "k")) {
        if (!q.is_cuda() || q.dim() != 4 || k.dim() != 4) refuse("q and k must be CUDA tensors [B][L][H][D]");
        expect(q, "q", at::kBFloat16, q.sizes(), q.device());
        expect(k, "k", at::kBFloat16, {q.size(0), k.size(1), q.size(2), q.size(3)}, q.device());
        if (pv) {
            v = required(pv, "v");
            expect(v, "v", at::kBFloat16, k.sizes(), q.device());
        }
        B = size32(q.size(0));
        Lq = size32(q.size(1));
        H = size32(q.size(2));
        D = size32(q.size(3));
        Lk = size32(k.size(1));
    }
    int64_t n_q() const { return (q.size(1) + ATTN_JVP_SELECT_BLOCK - 1) / ATTN_JVP_SELECT_BLOCK; }
    int64_t n_k() const { return (k.size(1) + ATTN_JVP_SELECT_BLOCK - 1) / ATTN_JVP_SELECT_BLOCK; }
    // a selection for these sizes: mask, index, tiles, order (or None), Lq, Lk
    void selection(PyObject* const* p, at::Tensor& mask, at::Tensor& index, at::Tensor& tiles, at::Tensor& order) const {
        mask = required(p[0], "selection");
        index = required(p[1], "selection");
        tiles = required(p[2], "selection");
        order = tensor(p[3], "selection");
        const at::Device dev = q.device();
        if (whole(p[4], "Lq") != Lq || whole(p[5], "Lk") != Lk || mask.dim() != 4 || mask.size(0) != B || mask.size(1) != H || mask.device() != dev)
            refuse("the selection is for other sizes or another device than q and k (B=%d, H=%d, Lq=%d, Lk=%d)", B, H, Lq, Lk);
        expect(mask, "selection.mask", at::kBool, {q.size(0), q.size(2), n_q(), n_k()}, dev);
        expect(index, "selection.index", at::kInt, {q.size(0), q.size(2), n_q(), n_k()}, dev);
        expect(tiles, "selection.tiles", at::kInt, {q.size(0), q.size(2), n_q()}, dev);
        if (order.defined()) expect(order, "selection.order", at::kInt, tiles.sizes(), dev);
    }
    cudaStream_t stream() const { return c10::cuda::getCurrentCUDAStream(q.device().index()).stream(); }
};

// q, k, topk, workspace -> (rc, mask, index, tiles)
PyObject* block_select(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 4, "block_select")) return nullptr;
    return guarded([&]() -> PyObject* {
        Qkv c(p[0], p[1], nullptr);
        const int topk = whole(p[2], "topk");
        at::Tensor mask = like(c.q, {c.q.size(0), c.q.size(2), c.n_q(), c.n_k()}, at::kBool), index = like(c.q, mask.sizes(), at::kInt);
        at::Tensor tiles = like(c.q, {c.q.size(0), c.q.size(2), c.n_q()}, at::kInt);
        at::Tensor ws = scratch(p[3], c.q, f_block_select_bytes(c.B, c.H, c.Lq, c.Lk, c.D));
        const c10::cuda::CUDAGuard guard(c.q.device());
        const int rc = unlocked([&] { return f_block_select(ptr(c.q), ptr(c.k), c.B, c.H, c.Lq, c.Lk, c.D, topk, ptr<unsigned char>(mask), ptr<int>(index), ptr<int>(tiles), ptr(ws),
                                      ws.nbytes(), c.stream()); });
        return result(rc, {mask, index, tiles});
    });
}

// mask, Lq, Lk -> (rc, index, tiles, order)
PyObject* block_lists(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 3, "block_lists")) return nullptr;
    return guarded([&]() -> PyObject* {
        at::Tensor mask = required(p[0], "mask");
        if (!mask.is_cuda() || mask.scalar_type() != at::kBool || mask.dim() != 4 || !mask.is_contiguous()) refuse("mask must be a contiguous CUDA bool tensor [B][H][n_q][n_k]");
        const int Lq = whole(p[1], "Lq"), Lk = whole(p[2], "Lk"), blk = ATTN_JVP_SELECT_BLOCK;
        if (mask.size(2) != (Lq + (int64_t)blk - 1) / blk || mask.size(3) != (Lk + (int64_t)blk - 1) / blk) refuse("mask must have a block for every 128 of %d queries and of %d keys", Lq, Lk);
        at::Tensor index = like(mask, mask.sizes(), at::kInt);
        at::Tensor tiles = like(mask, {mask.size(0), mask.size(1), mask.size(2)}, at::kInt), order = like(mask, tiles.sizes(), at::kInt);
        const c10::cuda::CUDAGuard guard(mask.device());
        const int rc = unlocked([&] { return f_block_lists(ptr<unsigned char>(mask), size32(mask.size(0)), size32(mask.size(1)), Lq, Lk, ptr<int>(index), ptr<int>(tiles),
                                     ptr<int>(order), c10::cuda::getCurrentCUDAStream(mask.device().index()).stream()); });
        return result(rc, {index, tiles, order});
    });
}

// q, k, v, mask, index, tiles, order, Lq, Lk, tq, tk, tv, scale (None: 1/sqrt D), fwd_only, return_mu, o, to, lse (outputs, or None)
// -> (rc, o, to, lse, mu)
PyObject* sparse_fwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 18, "sparse_fwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Qkv c(p[0], p[1], p[2]);
        at::Tensor mask, index, tiles, order, tq, tk, tv;
        c.selection(p + 3, mask, index, tiles, order);
        p += 9;                                                  // (the arguments behind the selection)
        const bool fwd_only = p[4] == Py_True;
        unsigned flags = ATTN_JVP_FWD_ONLY;
        if (!fwd_only) {
            tq = tensor(p[0], "tq");
            tk = tensor(p[1], "tk");
            tv = tensor(p[2], "tv");
            if (!tq.defined()) refuse("tq is required unless fwd_only");
            expect(tq, "tq", at::kBFloat16, c.q.sizes(), c.q.device());
            if (tk.defined() != tv.defined()) refuse("tk and tv must both be given or both be None");
            flags = tk.defined() ? 0u : ATTN_JVP_KV_TANGENT_FREE;
            if (tk.defined()) {
                expect(tk, "tk", at::kBFloat16, c.k.sizes(), c.q.device());
                expect(tv, "tv", at::kBFloat16, c.k.sizes(), c.q.device());
            }
        }
        const float scale = p[3] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(c.D))) : static_cast<float>(number(p[3], "scale"));
        const int64_t rows[3] = {c.q.size(0), c.q.size(2), c.q.size(1)};
        at::Tensor o = tensor(p[6], "o"), to = tensor(p[7], "to"), lse = tensor(p[8], "lse"), mu;
        if (o.defined()) expect(o, "o", at::kBFloat16, c.q.sizes(), c.q.device()); else o = same(c.q);
        if (!fwd_only) {
            if (to.defined()) expect(to, "to", at::kBFloat16, c.q.sizes(), c.q.device()); else to = same(c.q);
        } else {
            to = at::Tensor();
        }
        if (lse.defined()) expect(lse, "lse", at::kFloat, rows, c.q.device()); else lse = like(c.q, rows, at::kFloat);
        if (p[5] == Py_True) mu = like(c.q, rows, at::kFloat);
        const c10::cuda::CUDAGuard guard(c.q.device());
        const int rc = unlocked([&] { return f_sparse_fwd(ptr(c.q), ptr(c.k), ptr(c.v), ptr(tq), ptr(tk), ptr(tv), ptr<int>(index), ptr<int>(tiles), ptr<int>(order), ptr(o), ptr(to), ptr<float>(lse),
                                    ptr<float>(mu), c.B, c.H, c.Lq, c.Lk, c.D, scale, flags, c.stream()); });
        return result(rc, {o, to, lse, mu});
    });
}

// d_o, q, k, v, o, lse, mask, index, tiles, order, Lq, Lk, scale, workspace -> (rc, dq, dk, dv)
PyObject* sparse_bwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 14, "sparse_bwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Qkv c(p[1], p[2], p[3]);
        at::Tensor d_o = required(p[0], "d_o"), o = required(p[4], "o"), lse = required(p[5], "lse"), mask, index, tiles, order;
        const at::Device dev = c.q.device();
        expect(d_o, "d_o", at::kBFloat16, c.q.sizes(), dev);
        expect(o, "o", at::kBFloat16, c.q.sizes(), dev);
        expect(lse, "lse", at::kFloat, {c.q.size(0), c.q.size(2), c.q.size(1)}, dev);
        c.selection(p + 6, mask, index, tiles, order);
        const float scale = p[12] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(c.D))) : static_cast<float>(number(p[12], "scale"));
        at::Tensor ws = scratch(p[13], c.q, f_sparse_bwd_bytes(c.B, c.H, c.Lq, c.Lk, c.D));
        at::Tensor dq = same(c.q), dk = same(c.k), dv = same(c.k);
        const c10::cuda::CUDAGuard guard(dev);
        const int rc = unlocked([&] { return f_sparse_bwd(ptr(d_o), ptr(c.q), ptr(c.k), ptr(c.v), ptr(o), ptr<float>(lse), ptr<unsigned char>(mask), ptr<int>(index), ptr<int>(tiles), ptr<int>(order), ptr(dq),
                                    ptr(dk), ptr(dv), c.B, c.H, c.Lq, c.Lk, c.D, scale, ptr(ws), ws.nbytes(), c.stream()); });
        return result(rc, {dq, dk, dv});
    });
}

// Strides of batch, token and head of a tensor whose heads are contiguous.
void heads_of(const at::Tensor& t, const char* name, at::IntArrayRef shape, const at::Device& device, long long* stride) {
    if (t.device() != device || t.scalar_type() != at::kBFloat16 || t.sizes() != shape || t.stride(3) != 1)
        refuse("%s must be a bf16 tensor on %s of the shape that the other arguments give, with contiguous heads", name, device.str().c_str());
    for (int i = 0; i < 3; ++i) {
        stride[i] = t.stride(i);
        if (t.size(i) > 1 && stride[i] % 8 != 0 && !t.is_contiguous()) refuse("%s: strides must be multiples of 8 elements", name);     // (else: a head dimension that the library refuses)
    }
}

// ---- dense attention with masks, shared heads and strides ----
// args: q, k, v, scale (None: 1/sqrt D), causal, k_lengths
struct Attention {
    at::Tensor q, k, v, lengths;
    attn_jvp_attention_t a = {};
    explicit Attention(PyObject* const* p) : q(required(p[0], "q")), k(required(p[1], "k")), v(required(p[2], "v")), lengths(tensor(p[5], "k_lengths")) {
        if (!q.is_cuda() || q.dim() != 4 || k.dim() != 4) refuse("q and k must be CUDA tensors [B][L][H][D]");
        const at::Device dev = q.device();
        heads_of(q, "q", q.sizes(), dev, a.q_stride);
        heads_of(k, "k", {q.size(0), k.size(1), k.size(2), q.size(3)}, dev, a.k_stride);
        heads_of(v, "v", k.sizes(), dev, a.v_stride);
        if (k.size(2) == 0 ? q.size(2) != 0 : q.size(2) % k.size(2) != 0) refuse("%lld query heads cannot share %lld key heads evenly", (long long)q.size(2), (long long)k.size(2));
        if (lengths.defined()) expect(lengths, "k_lengths", at::kInt, {q.size(0)}, dev);
        a.q = ptr(q);
        a.k = ptr(k);
        a.v = ptr(v);
        a.k_lengths = ptr<int>(lengths);
        a.B = size32(q.size(0));
        a.Lq = size32(q.size(1));
        a.H = size32(q.size(2));
        a.D = size32(q.size(3));
        a.Lk = size32(k.size(1));
        a.Hk = size32(k.size(2));
        a.scale = p[3] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(a.D))) : static_cast<float>(number(p[3], "scale"));
        a.causal = p[4] == Py_True;
    }
    // what the calls without masks, shared heads and strides take
    bool plain() const { return !a.causal && !a.k_lengths && a.H == a.Hk && q.is_contiguous() && k.is_contiguous() && v.is_contiguous(); }
    cudaStream_t stream() const { return c10::cuda::getCurrentCUDAStream(q.device().index()).stream(); }
};

// ... , tq, tk, tv, fwd_only, return_mu, o, to, lse (outputs, or None) -> (rc, o, to, lse, mu)
PyObject* attention_fwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 14, "attention_fwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Attention c(p);
        p += 6;
        const at::Device dev = c.q.device();
        const bool fwd_only = p[3] == Py_True;
        unsigned flags = ATTN_JVP_FWD_ONLY;
        at::Tensor tq, tk, tv;
        if (!fwd_only) {
            tq = required(p[0], "tq");
            tk = tensor(p[1], "tk");
            tv = tensor(p[2], "tv");
            expect(tq, "tq", at::kBFloat16, c.q.sizes(), dev);
            if (tk.defined() != tv.defined()) refuse("tk and tv must both be given or both be None");
            flags = tk.defined() ? 0u : ATTN_JVP_KV_TANGENT_FREE;
            if (tk.defined()) {
                expect(tk, "tk", at::kBFloat16, c.k.sizes(), dev);
                expect(tv, "tv", at::kBFloat16, c.k.sizes(), dev);
            }
            c.a.tq = ptr(tq);
            c.a.tk = ptr(tk);
            c.a.tv = ptr(tv);
        }
        const int64_t rows[3] = {c.q.size(0), c.q.size(2), c.q.size(1)};
        at::Tensor o = tensor(p[5], "o"), to = fwd_only ? at::Tensor() : tensor(p[6], "to"), lse = tensor(p[7], "lse"), mu;
        if (o.defined()) expect(o, "o", at::kBFloat16, c.q.sizes(), dev); else o = same(c.q);
        if (to.defined()) expect(to, "to", at::kBFloat16, c.q.sizes(), dev); else if (!fwd_only) to = same(c.q);
        if (lse.defined()) expect(lse, "lse", at::kFloat, rows, dev); else lse = like(c.q, rows, at::kFloat);
        if (p[4] == Py_True) mu = like(c.q, rows, at::kFloat);
        const c10::cuda::CUDAGuard guard(dev);
        const int rc = unlocked([&] {
            const attn_jvp_attention_t& a = c.a;
            if (c.plain() && mu.defined())
                return f_fwd_mu(a.q, a.k, a.v, a.tq, a.tk, a.tv, ptr(o), ptr(to), ptr<float>(lse), ptr<float>(mu), a.B, a.H, a.Lq, a.Lk, a.D, a.scale, flags, c.stream());
            if (c.plain()) return f_fwd_stream(a.q, a.k, a.v, a.tq, a.tk, a.tv, ptr(o), ptr(to), ptr<float>(lse), a.B, a.H, a.Lq, a.Lk, a.D, a.scale, flags, c.stream());
            return f_attention_fwd(&c.a, ptr(o), ptr(to), ptr<float>(lse), ptr<float>(mu), flags, c.stream());
        });
        return result(rc, {o, to, lse, mu});
    });
}

// d_o, (the six of Attention), o, lse, workspace -> (rc, dq, dk, dv)
PyObject* attention_bwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 10, "attention_bwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        at::Tensor d_o = required(p[0], "d_o"), o = required(p[7], "o"), lse = required(p[8], "lse");
        Attention c(p + 1);
        const at::Device dev = c.q.device();
        expect(d_o, "d_o", at::kBFloat16, c.q.sizes(), dev);
        expect(o, "o", at::kBFloat16, c.q.sizes(), dev);
        expect(lse, "lse", at::kFloat, {c.q.size(0), c.q.size(2), c.q.size(1)}, dev);
        at::Tensor ws = scratch(p[9], c.q, f_attention_bwd_bytes(c.a.B, c.a.H, c.a.Hk, c.a.Lq, c.a.Lk, c.a.D));
        at::Tensor dq = same(c.q), dk = same(c.k), dv = same(c.k);
        const c10::cuda::CUDAGuard guard(dev);
        const int rc = unlocked([&] { return f_attention_bwd(&c.a, ptr(d_o), ptr(o), ptr<float>(lse), ptr(dq), ptr(dk), ptr(dv), ptr(ws), ws.nbytes(), c.stream()); });
        return result(rc, {dq, dk, dv});
    });
}

// ---- rotary positions ----
// The numbers of a sequence (a tuple or list), one per axis.
int numbers(PyObject* o, const char* name, double* out, int most) {
    if (!PyTuple_Check(o) && !PyList_Check(o)) refuse("%s must be a tuple or list", name);
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
    if (n < 1 || n > most) refuse("%s must have 1 to %d entries", name, most);
    for (Py_ssize_t i = 0; i < n; ++i) out[i] = number(PySequence_Fast_GET_ITEM(o, i), name);
    return static_cast<int>(n);
}

// positions, dims, base, scaling, factor, original_length -> (rc, table)
PyObject* rotary_table(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 6, "rotary_table")) return nullptr;
    return guarded([&]() -> PyObject* {
        constexpr int kMost = 8;
        at::Tensor pos = required(p[0], "positions");
        double d[kMost], base[kMost], factor[kMost];
        int dims[kMost], channels = 0;
        const int axes = numbers(p[1], "dims", d, kMost);
        if (numbers(p[2], "base", base, kMost) != axes || numbers(p[4], "factor", factor, kMost) != axes) refuse("base and factor must have an entry for each of the %d axes", axes);
        for (int a = 0; a < axes; ++a) {
            if (!(d[a] >= 2 && d[a] <= 1024) || d[a] != std::floor(d[a])) refuse("dims must be even numbers of channels");
            channels += dims[a] = static_cast<int>(d[a]);
        }
        const auto type = pos.scalar_type();
        if (!pos.is_cuda() || !pos.is_contiguous() || (type != at::kInt && type != at::kLong && type != at::kFloat)) refuse("positions must be a contiguous CUDA tensor of int32, int64 or fp32");
        std::vector<int64_t> shape(pos.sizes().begin(), pos.sizes().end());
        if (axes > 1) {
            if (shape.empty() || shape.back() != axes) refuse("positions must have shape [...][%d], one coordinate per axis", axes);
            shape.pop_back();
        }
        shape.push_back(channels / 2);
        shape.push_back(2);
        at::Tensor table = like(pos, shape, at::kFloat);
        const int scaling = whole(p[3], "scaling"), kind = type == at::kInt ? ATTN_JVP_INT32 : type == at::kLong ? ATTN_JVP_INT64 : ATTN_JVP_FP32;
        const double original = p[5] == Py_None ? 0.0 : number(p[5], "original_length");
        const c10::cuda::CUDAGuard guard(pos.device());
        const int rc = unlocked([&] { return f_rotary_table(ptr(pos), kind, pos.numel() / axes, axes, dims, base, scaling, factor, original, ptr<float>(table),
                                       c10::cuda::getCurrentCUDAStream(pos.device().index()).stream()); });
        return result(rc, {table});
    });
}

// args: q, k, table, index, norm, layout, eps, q_weight, k_weight, q_bias, k_bias
struct Rotary {
    at::Tensor q, k, table, index, w[4];
    attn_jvp_qk_rotary_t a = {};
    explicit Rotary(PyObject* const* p) : q(required(p[0], "q")), k(tensor(p[1], "k")), table(required(p[2], "table")), index(tensor(p[3], "index")) {
        if (!q.is_cuda() || q.dim() != 4 || q.numel() == 0) refuse("q must be a CUDA tensor [B][L][H][D] that is not empty");
        const at::Device dev = q.device();
        heads_of(q, "q", q.sizes(), dev, a.q_stride);
        if (k.defined()) {
            if (k.dim() != 4 || k.numel() == 0) refuse("k must have shape [B][L][Hk][D] and not be empty");
            heads_of(k, "k", {q.size(0), q.size(1), k.size(2), q.size(3)}, dev, a.k_stride);
        }
        a.B = size32(q.size(0));
        a.L = size32(q.size(1));
        a.H = size32(q.size(2));
        a.Hk = k.defined() ? size32(k.size(2)) : 0;
        a.D = size32(q.size(3));
        const int64_t td = table.dim();
        if (table.device() != dev || table.scalar_type() != at::kFloat || !table.is_contiguous() || (td != 3 && td != 4) || table.size(td - 1) != 2 ||
            (td == 4 && table.size(0) != q.size(0)))
            refuse("table must be a contiguous fp32 tensor [rows][R / 2][2] or [B][rows][R / 2][2] on %s", dev.str().c_str());
        a.R = size32(2 * table.size(td - 2));
        a.table_rows = table.size(td - 3);
        a.table_batch = td == 4 ? a.table_rows : 0;
        if (index.defined()) {
            const int64_t id = index.dim();
            if (index.device() != dev || index.scalar_type() != at::kInt || !index.is_contiguous() || (id != 1 && id != 2) || index.size(id - 1) != q.size(1) ||
                (id == 2 && index.size(0) != q.size(0)))
                refuse("index must be a contiguous int32 tensor [L] or [B][L] on %s", dev.str().c_str());
            a.index_batch = id == 2 ? q.size(1) : 0;
        } else if (a.table_rows < a.L) {
            refuse("the table has %lld rows for %d tokens", a.table_rows, a.L);
        }
        a.norm = whole(p[4], "norm");
        a.layout = whole(p[5], "layout");
        a.eps = static_cast<float>(number(p[6], "eps"));
        static const char* const names[4] = {"q_weight", "k_weight", "q_bias", "k_bias"};
        for (int i = 0; i < 4; ++i) {
            w[i] = tensor(p[7 + i], names[i]);
            if (!w[i].defined()) continue;
            if (i % 2 == 1 && !k.defined()) refuse("%s acts on k, which is None", names[i]);
            expect(w[i], names[i], at::kFloat, {q.size(3)}, dev);
        }
        a.q = ptr(q);
        a.k = ptr(k);
        a.q_weight = ptr<float>(w[0]);
        a.k_weight = ptr<float>(w[1]);
        a.q_bias = ptr<float>(w[2]);
        a.k_bias = ptr<float>(w[3]);
        a.table = ptr<float>(table);
        a.index = ptr<int>(index);
    }
    at::Tensor out(const at::Tensor& t) const { return t.defined() ? like(t, t.sizes(), at::kBFloat16) : at::Tensor(); }
    cudaStream_t stream() const { return c10::cuda::getCurrentCUDAStream(q.device().index()).stream(); }
};

// ... , tq, tk -> (rc, q', k', tq', tk')
PyObject* qk_rotary_fwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 13, "qk_rotary_fwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        Rotary c(p);
        at::Tensor tq = tensor(p[11], "tq"), tk = tensor(p[12], "tk"), q = c.out(c.q), k = c.out(c.k), tqn, tkn;
        if (tq.defined() || tk.defined()) {
            if (!tq.defined() || tk.defined() != c.k.defined()) refuse("with tangents tq is required, and tk exactly where k is given");
            heads_of(tq, "tq", c.q.sizes(), c.q.device(), c.a.tq_stride);
            if (tk.defined()) heads_of(tk, "tk", c.k.sizes(), c.q.device(), c.a.tk_stride);
            c.a.tq = ptr(tq);
            c.a.tk = ptr(tk);
            tqn = c.out(c.q);
            tkn = c.out(c.k);
        }
        const c10::cuda::CUDAGuard guard(c.q.device());
        const int rc = unlocked([&] { return f_qk_rotary_fwd(&c.a, ptr(q), ptr(k), ptr(tqn), ptr(tkn), c.stream()); });
        return result(rc, {q, k, tqn, tkn});
    });
}

// dq_new, dk_new, (the eleven of Rotary), workspace -> (rc, dq, dk, dq_weight, dk_weight, dq_bias, dk_bias)
PyObject* qk_rotary_bwd(PyObject*, PyObject* const* p, Py_ssize_t n) {
    if (!count(n, 14, "qk_rotary_bwd")) return nullptr;
    return guarded([&]() -> PyObject* {
        at::Tensor dqn = required(p[0], "dq_new"), dkn = tensor(p[1], "dk_new");
        Rotary c(p + 2);
        if (dkn.defined() != c.k.defined()) refuse("dk_new is required exactly where k is given");
        expect(dqn, "dq_new", at::kBFloat16, c.q.sizes(), c.q.device());
        if (dkn.defined()) expect(dkn, "dk_new", at::kBFloat16, c.k.sizes(), c.q.device());
        at::Tensor dq = c.out(c.q), dk = c.out(c.k), d[4], ws;
        bool sums = false;
        for (int i = 0; i < 4; ++i) if (c.w[i].defined()) {
            d[i] = like(c.q, {c.q.size(3)}, at::kFloat);
            sums = true;
        }
        if (sums) ws = scratch(p[13], c.q, f_qk_rotary_bwd_bytes(c.a.B, c.a.L, c.a.H, c.a.Hk, c.a.D));
        const c10::cuda::CUDAGuard guard(c.q.device());
        const int rc = unlocked([&] { return f_qk_rotary_bwd(&c.a, ptr(dqn), ptr(dkn), ptr(dq), ptr(dk), ptr<float>(d[0]), ptr<float>(d[1]), ptr<float>(d[2]), ptr<float>(d[3]), ptr(ws),
                                       ws.defined() ? ws.nbytes() : 0, c.stream()); });
        return result(rc, {dq, dk, d[0], d[1], d[2], d[3]});
    });
}

// The library's functions, by address and in this order.
PyObject* bind(PyObject*, PyObject* const* p, Py_ssize_t n) {
    void** slots[] = {reinterpret_cast<void**>(&f_adaln_fwd), reinterpret_cast<void**>(&f_adaln_bwd), reinterpret_cast<void**>(&f_adaln_bwd_bytes),
                      reinterpret_cast<void**>(&f_block_select), reinterpret_cast<void**>(&f_block_select_bytes), reinterpret_cast<void**>(&f_block_lists),
                      reinterpret_cast<void**>(&f_sparse_fwd), reinterpret_cast<void**>(&f_sparse_bwd), reinterpret_cast<void**>(&f_sparse_bwd_bytes),
                      reinterpret_cast<void**>(&f_fwd_stream), reinterpret_cast<void**>(&f_fwd_mu), reinterpret_cast<void**>(&f_attention_fwd), reinterpret_cast<void**>(&f_attention_bwd), reinterpret_cast<void**>(&f_attention_bwd_bytes),
                      reinterpret_cast<void**>(&f_rotary_table), reinterpret_cast<void**>(&f_qk_rotary_fwd), reinterpret_cast<void**>(&f_qk_rotary_bwd),
                      reinterpret_cast<void**>(&f_qk_rotary_bwd_bytes)};
    constexpr Py_ssize_t slots_n = sizeof slots / sizeof slots[0];
    if (!count(n, slots_n, "bind")) return nullptr;
    for (Py_ssize_t i = 0; i < slots_n; ++i) {
        void* at = PyLong_AsVoidPtr(p[i]);
        if (at == nullptr) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: a null address");
            return nullptr;
        }
        *slots[i] = at;
    }
    Py_RETURN_NONE;
}

#define HOST_FN(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HOST_FN(bind), HOST_FN(adaln_fwd), HOST_FN(adaln_bwd), HOST_FN(block_select), HOST_FN(block_lists),
                         HOST_FN(sparse_fwd), HOST_FN(sparse_bwd), HOST_FN(attention_fwd), HOST_FN(attention_bwd), HOST_FN(rotary_table), HOST_FN(qk_rotary_fwd),
                         HOST_FN(qk_rotary_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "Tensor checks and calls into the C ABI.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
