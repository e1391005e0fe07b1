// CPython module behind binding.py: takes torch tensors, checks them, makes the outputs and the
// scratch, and calls the C entry point of the same name on the current stream.
//
// Every call here is on the critical path of a small decode or prefill step: marshalling the same
// arguments through ctypes (a Python object per pointer, attribute look-ups per tensor, a stream
// object) took ~15 us of host time per call where the kernels behind it run 3 to 20 us, so a rollout
// layer of 12 launches was bound by the host.  Nothing is kept between calls except the
// per-device library context.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <mutex>
#include <string>
#include <vector>

#include "../../include/tik.h"

namespace {

PyObject* g_error = nullptr;                 // binding.TikError

// A Python exception is set; unwinds to the entry point.
struct PyError {};

[[noreturn]] void raise(PyObject* type, const std::string& msg) {
    PyErr_SetString(type, msg.c_str());
    throw PyError{};
}
[[noreturn]] void raise_tik(const std::string& msg) { raise(g_error, msg); }

// ---------------------------------------------------------------- per-device context
constexpr int MAX_DEVICES = 64;
std::mutex g_ctx_mutex;
std::atomic<tik_ctx*> g_ctx[MAX_DEVICES];

tik_ctx* context(int device) {
    if (device < 0 || device >= MAX_DEVICES) raise_tik("device ordinal out of range");
    tik_ctx* c = g_ctx[device].load(std::memory_order_acquire);
    if (c) return c;
    std::lock_guard<std::mutex> lock(g_ctx_mutex);
    c = g_ctx[device].load(std::memory_order_acquire);
    if (c) return c;
    const tik_status rc = tik_create(&c, device);
    if (rc != TIK_OK) raise_tik(std::string("tik_create failed: ") + tik_status_str(rc));
    g_ctx[device].store(c, std::memory_order_release);
    return c;
}

int current_device() {
    if (c10::cuda::device_count() < 1) raise_tik("tik needs a CUDA device; there is no CPU path");
    return static_cast<int>(c10::cuda::current_device());
}

// ---------------------------------------------------------------- arguments
struct Args {
    PyObject* const* a;
    Py_ssize_t n;
    Py_ssize_t i = 0;
    PyObject* next() {
        if (i >= n) raise(PyExc_TypeError, "too few arguments");
        return a[i++];
    }
    const at::Tensor& tensor() {
        PyObject* o = next();
        if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string("expected a tensor, got ") + Py_TYPE(o)->tp_name);
        return THPVariable_Unpack(o);
    }
    // nullptr for None
    const at::Tensor* opt() {
        if (i < n && a[i] == Py_None) {
            ++i;
            return nullptr;
        }
        return &tensor();
    }
    int64_t integer() {
        const long long v = PyLong_AsLongLong(next());
        if (v == -1 && PyErr_Occurred()) throw PyError{};
        return v;
    }
    int int32() {
        const int64_t v = integer();
        if (v < INT32_MIN || v > INT32_MAX) raise(PyExc_OverflowError, "integer argument out of range");
        return static_cast<int>(v);
    }
    double dbl() {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw PyError{};
        return v;
    }
    float real() { return static_cast<float>(dbl()); }
};

void* ptr(const at::Tensor& t) {
    if (!t.is_cuda() || !t.is_contiguous()) raise_tik("tensors must be contiguous CUDA tensors");
    return t.data_ptr();
}
void* ptr(const at::Tensor& t, at::ScalarType type) {
    void* p = ptr(t);
    if (t.scalar_type() != type)
        raise_tik(std::string("expected dtype ") + at::toString(type) + ", got " + at::toString(t.scalar_type()));
    return p;
}
void* ptr(const at::Tensor* t, at::ScalarType type) { return t ? ptr(*t, type) : nullptr; }
void* bf(const at::Tensor& t) { return ptr(t, at::kBFloat16); }
void* bf(const at::Tensor* t) { return ptr(t, at::kBFloat16); }
float* f32(const at::Tensor* t) { return static_cast<float*>(ptr(t, at::kFloat)); }
int32_t* i32(const at::Tensor& t) { return static_cast<int32_t*>(ptr(t, at::kInt)); }
int32_t* i32(const at::Tensor* t) { return t ? i32(*t) : nullptr; }

void want_rank(const at::Tensor& t, int64_t rank) {
    if (t.dim() != rank)
        raise(PyExc_ValueError, "expected a tensor with " + std::to_string(rank) + " dimensions, got " + std::to_string(t.dim()));
}
// an argument of which only one axis' size is read
void want_axis(const at::Tensor& t, int64_t axis) {
    if (t.dim() <= axis) raise(PyExc_IndexError, "axis " + std::to_string(axis) + " of a tensor with " + std::to_string(t.dim()) + " dimensions");
}
int dim(const at::Tensor& t, int64_t i) {
    const int64_t v = t.size(i);
    if (v > INT32_MAX) raise(PyExc_OverflowError, "tensor dimension out of range");
    return static_cast<int>(v);
}

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
    if (!like.is_cuda()) raise_tik("tensors must be contiguous CUDA tensors");
    return at::detail::empty_cuda(sizes, type, like.device(), std::nullopt);
}

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

void check(tik_status rc, const tik_ctx* ctx) {
    if (rc != TIK_OK) raise_tik(std::string(tik_status_str(rc)) + ": " + tik_last_error(ctx));
}

// Runs a C entry point without the interpreter lock (a launch blocks while the launch queue is full).  f reads
// plain values only: whatever inspects a tensor or may raise happens before, under the lock.  An exception that
// leaves f all the same passes with the lock taken back, so that its handler may set a Python error.
template <class F>
tik_status unlocked(F&& f) {
    struct Unlock {
        PyThreadState* state = PyEval_SaveThread();
        ~Unlock() { PyEval_RestoreThread(state); }
    } unlock;
    return f();
}

struct Scratch {
    at::Tensor own;
    void* p = nullptr;
    size_t bytes = 0;
    void use(const at::Tensor& t) {
        p = ptr(t);
        bytes = t.nbytes();
    }
    void make(size_t need, const at::Tensor& like) {
        own = empty({static_cast<int64_t>(need)}, at::kByte, like);
        p = own.data_ptr();
        bytes = need;
    }
};

// Scratch of the full-sequence kernels: None = what the op asks for, False = none, a tensor = that one.
Scratch plan_ws(PyObject* ws, int op, int64_t S, int64_t max_positions, const at::Tensor& like) {
    Scratch s;
    if (ws == Py_False) return s;
    if (ws != Py_None) {
        if (!THPVariable_Check(ws)) raise(PyExc_TypeError, "ws must be a tensor, None or False");
        s.use(THPVariable_Unpack(ws));
        return s;
    }
    const size_t need = tik_workspace_bytes(op, S, 0, 0, 0, max_positions, 0, 0);
    if (need > 0) s.make(need, like);
    return s;
}
Scratch sized_ws(const at::Tensor* ws, size_t need, const at::Tensor& like) {
    Scratch s;
    if (ws) s.use(*ws);
    else s.make(need > 16 ? need : 16, like);
    return s;
}

PyObject* wrap(const at::Tensor* given, at::Tensor& made) {
    return THPVariable_Wrap(given ? *given : made);
}
// `given` or a new tensor of those sizes
const at::Tensor& out_or(const at::Tensor* given, at::Tensor& made, at::IntArrayRef sizes, at::ScalarType type,
                         const at::Tensor& like) {
    if (given) return *given;
    made = empty(sizes, type, like);
    return made;
}

// ---------------------------------------------------------------- entry points (positional, in binding.py's order)

PyObject* attn_train_fwd(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &q = a.tensor(), &k = a.tensor();
    const at::Tensor* v = a.opt();
    const at::Tensor& cu = a.tensor();
    const int max_seqlen = a.int32();
    const float scale = a.real();
    const at::Tensor *o_in = a.opt(), *lse = a.opt();
    PyObject* ws_in = a.next();
    want_rank(q, 3);
    want_axis(k, 1);
    at::Tensor made;
    const at::Tensor& o = out_or(o_in, made, q.sizes(), q.scalar_type(), q);
    const int S = static_cast<int>(cu.numel() - 1);
    const Scratch ws = plan_ws(ws_in, TIK_OP_ATTN_TRAIN_FWD, S, max_seqlen, q);
    void *qp = bf(q), *kp = bf(k), *vp = bf(v), *op = bf(o), *st = stream();
    float* lp = f32(lse);
    int32_t* cp = i32(cu);
    const int Hq = dim(q, 1), Hkv = dim(k, 1), d = dim(q, 2);
    const int64_t tot = q.size(0);
    check(unlocked([&] { return tik_attn_train_fwd(ctx, qp, kp, vp, op, lp, cp, S, tot, max_seqlen, Hq, Hkv, d, scale, ws.p,
                                                   ws.bytes, st); }), ctx);
    return wrap(o_in, made);
}

PyObject* attn_train_bwd(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &q = a.tensor(), &k = a.tensor(), &v = a.tensor();
    const at::Tensor *o = a.opt(), *d_o = a.opt(), *lse = a.opt();
    const at::Tensor& cu = a.tensor();
    const int max_seqlen = a.int32();
    const float scale = a.real();
    const at::Tensor* ws_in = a.opt();
    want_rank(q, 3);
    want_axis(k, 1);
    const int64_t tot = q.size(0);
    const int Hq = dim(q, 1), Hkv = dim(k, 1), d = dim(q, 2), S = static_cast<int>(cu.numel() - 1);
    const Scratch ws = sized_ws(ws_in, tik_workspace_bytes(TIK_OP_ATTN_TRAIN_BWD, tot, Hq, Hkv, d, 0, 0, 0), q);
    at::Tensor dq = empty(q.sizes(), q.scalar_type(), q), dk = empty(k.sizes(), k.scalar_type(), k),
               dv = empty(v.sizes(), v.scalar_type(), v);
    void *qp = bf(q), *kp = bf(k), *vp = bf(v), *op = bf(o), *gp = bf(d_o), *dqp = bf(dq), *dkp = bf(dk), *dvp = bf(dv), *st = stream();
    float* lp = f32(lse);
    int32_t* cp = i32(cu);
    check(unlocked([&] { return tik_attn_train_bwd(ctx, qp, kp, vp, op, gp, lp, dqp, dkp, dvp, cp, S, tot, max_seqlen, Hq, Hkv,
                                                   d, scale, ws.p, ws.bytes, st); }), ctx);
    PyObject *a0 = THPVariable_Wrap(dq), *a1 = THPVariable_Wrap(dk), *a2 = THPVariable_Wrap(dv);
    return Py_BuildValue("(NNN)", a0, a1, a2);
}

// caches, block table and what they say about the layout
struct Cache {
    void *k, *v;
    int32_t* table;
    int max_blocks, num_pages, Hkv, page, d;
};
Cache cache_of(const at::Tensor& kc, const at::Tensor& vc, const at::Tensor& table) {
    want_rank(kc, 4);
    want_axis(table, 1);
    return {bf(kc), bf(vc), i32(table), dim(table, 1), dim(kc, 0), dim(kc, 1), dim(kc, 2), dim(kc, 3)};
}

PyObject* kv_cache_write(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor& k = a.tensor();
    const at::Tensor *v = a.opt(), *cu = a.opt();
    const at::Tensor &lens = a.tensor(), &kc = a.tensor(), &vc = a.tensor(), &table = a.tensor();
    want_axis(k, 0);
    const Cache c = cache_of(kc, vc, table);
    void *kp = bf(k), *vp = bf(v), *st = stream();
    int32_t *cp = i32(cu), *lp = i32(lens);
    const int S = static_cast<int>(lens.numel());
    const int64_t n = k.size(0);
    check(unlocked([&] { return tik_kv_cache_write(ctx, kp, vp, cp, lp, c.k, c.v, c.table, c.max_blocks, S, n, c.Hkv, c.d,
                                                   c.page, c.num_pages, st); }), ctx);
    Py_RETURN_NONE;
}

PyObject* qk_norm_rope_kv_write(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &q = a.tensor(), &k = a.tensor();
    const at::Tensor *v = a.opt(), *wq = a.opt(), *wk = a.opt();
    const float eps = a.real();
    const at::Tensor &cs = a.tensor(), &cu = a.tensor();
    const at::Tensor *lens = a.opt(), *kc = a.opt(), *vc = a.opt(), *table = a.opt();
    want_rank(q, 3);
    want_axis(k, 1);
    want_axis(cs, 0);
    if (kc) want_axis(*kc, 2);
    if (table) want_axis(*table, 1);
    const int Hq = dim(q, 1), Hkv = dim(k, 1), d = dim(q, 2), page = kc ? dim(*kc, 2) : 0, pages = kc ? dim(*kc, 0) : 0;
    const int max_blocks = table ? dim(*table, 1) : 0, S = static_cast<int>(cu.numel() - 1);
    void *qp = bf(q), *kp = bf(k), *vp = bf(v), *wqp = bf(wq), *wkp = bf(wk), *kcp = bf(kc), *vcp = bf(vc), *st = stream();
    const float* csp = f32(&cs);
    int32_t *cp = i32(cu), *lp = i32(lens), *tp = i32(table);
    const int64_t n = q.size(0);
    const int max_pos = dim(cs, 0);
    check(unlocked([&] { return tik_qk_norm_rope_kv_write(ctx, qp, kp, vp, wqp, wkp, eps, csp, max_pos, cp, lp, kcp, vcp, tp,
                                                          max_blocks, S, n, Hq, Hkv, d, page, pages, st); }), ctx);
    Py_RETURN_NONE;
}

PyObject* rmsnorm(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &x = a.tensor(), &w = a.tensor();
    const float eps = a.real();
    const at::Tensor *res = a.opt(), *y_in = a.opt();
    want_rank(x, 2);
    at::Tensor made;
    const at::Tensor& y = out_or(y_in, made, x.sizes(), x.scalar_type(), x);
    void *xp = bf(x), *rp = bf(res), *wp = bf(w), *yp = bf(y), *st = stream();
    const int64_t T = x.size(0);
    const int H = dim(x, 1);
    check(unlocked([&] { return tik_rmsnorm(ctx, xp, rp, wp, yp, eps, T, H, st); }), ctx);
    return wrap(y_in, made);
}

PyObject* swiglu(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor& gu = a.tensor();
    const at::Tensor* out_in = a.opt();
    want_rank(gu, 2);
    at::Tensor made;
    const int64_t T = gu.size(0);
    const int inter = dim(gu, 1) / 2;
    const at::Tensor& out = out_or(out_in, made, {T, inter}, at::kBFloat16, gu);
    void *gp = bf(gu), *op = bf(out), *st = stream();
    check(unlocked([&] { return tik_swiglu(ctx, gp, op, T, inter, st); }), ctx);
    return wrap(out_in, made);
}

PyObject* linear(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &x = a.tensor(), &w = a.tensor();
    const at::Tensor* y_in = a.opt();
    want_rank(x, 2);
    want_axis(w, 0);
    at::Tensor made;
    const int64_t T = x.size(0);
    const int K = dim(x, 1), N = dim(w, 0);
    const at::Tensor& y = out_or(y_in, made, {T, N}, at::kBFloat16, x);
    void *xp = bf(x), *wp = bf(w), *yp = bf(y), *st = stream();
    check(unlocked([&] { return tik_linear(ctx, xp, wp, yp, T, K, N, st); }), ctx);
    return wrap(y_in, made);
}

// a tensor of the current device
const at::Tensor& on(int device, const at::Tensor& t) {
    if (!t.is_cuda() || t.get_device() != device) raise_tik("tensors must be on the current CUDA device");
    return t;
}
const at::Tensor* on(int device, const at::Tensor* t) { return t ? &on(device, *t) : nullptr; }
void want_sizes(const at::Tensor& t, at::IntArrayRef sizes, const char* what) {
    if (t.sizes() != sizes) raise(PyExc_ValueError, std::string(what) + " has the wrong shape");
}
void want_sizes(const at::Tensor* t, at::IntArrayRef sizes, const char* what) {
    if (t) want_sizes(*t, sizes, what);
}

// A contiguous tensor over a part of another one's storage, `at` elements in (a view without the dispatcher: ~0.1 us of host
// time where an allocation takes 0.8).
at::Tensor part_of(const at::Tensor& whole, int64_t at, at::IntArrayRef sizes, at::ScalarType type) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), c10::scalarTypeToTypeMeta(type));
    impl->set_storage_offset(at);
    impl->set_sizes_contiguous(sizes);
    return at::Tensor(std::move(impl));
}
// What a call makes -- results and scratch -- as parts of one allocation where it is small: host time is what such a call costs
// (block norm 64 x 3584 4.8 -> 4.5 us, its gradient 256 x 256 9.8 -> 8.4).  A result then keeps its neighbours' memory alive, so
// larger ones have allocations of their own.
struct Pool {
    static constexpr int64_t MOST = 1 << 20;
    at::Tensor whole;
    int64_t used = 0;
    static int64_t room(int64_t bytes) { return (bytes + 127) / 128 * 128; }
    Pool(int64_t total, const at::Tensor& like) {
        if (total > 0 && total <= MOST) whole = empty({total}, at::kByte, like);
    }
    at::Tensor take(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
        if (!whole.defined()) return empty(sizes, type, like);
        const int64_t size = static_cast<int64_t>(c10::elementSize(type)), at = used;
        int64_t n = size;
        for (const int64_t s : sizes) n *= s;
        used += room(n);
        return part_of(whole, at / size, sizes, type);
    }
};

PyObject* embedding(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const at::Tensor &ids = on(dev, a.tensor()), &table = on(dev, a.tensor());
    const float scale = a.real();
    const at::Tensor* y_in = on(dev, a.opt());
    want_rank(ids, 1);
    want_rank(table, 2);
    at::Tensor made;
    const int64_t T = ids.size(0);
    const int V = dim(table, 0), H = dim(table, 1);
    want_sizes(y_in, {T, H}, "y");
    const at::Tensor& y = out_or(y_in, made, {T, H}, at::kBFloat16, table);
    void *tp = bf(table), *yp = bf(y), *st = stream();
    const int32_t* ip = i32(ids);
    check(unlocked([&] { return tik_embedding(ctx, ip, tp, yp, scale, T, V, H, st); }), ctx);
    return wrap(y_in, made);
}

int element_type(const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return TIK_DTYPE_BF16;
    if (t.scalar_type() == at::kFloat) return TIK_DTYPE_FP32;
    raise_tik(std::string("expected bf16 or fp32, got ") + at::toString(t.scalar_type()));
}

PyObject* embedding_bwd(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const at::Tensor &dy = on(dev, a.tensor()), &ids = on(dev, a.tensor());
    const int V = a.int32();
    const float scale = a.real();
    const at::Tensor* table_in = on(dev, a.opt());
    const int accumulate = a.int32();
    const at::Tensor* ws_in = on(dev, a.opt());
    want_rank(dy, 2);
    const int64_t T = dy.size(0);
    const int H = dim(dy, 1);
    want_sizes(ids, {T}, "ids");
    if (V <= 0) raise(PyExc_ValueError, "vocab must be positive");
    want_sizes(table_in, {V, H}, "d_table");
    if (accumulate && !table_in) raise(PyExc_ValueError, "accumulate needs d_table");
    const Scratch ws = sized_ws(ws_in, tik_workspace_bytes(TIK_OP_EMBEDDING_BWD, T, 0, 0, 0, 0, H, V), dy);
    at::Tensor made;
    const at::Tensor& table = out_or(table_in, made, {V, H}, at::kBFloat16, dy);
    const int type = element_type(table);
    void *gp = bf(dy), *tp = ptr(table), *st = stream();
    const int32_t* ip = i32(ids);
    check(unlocked([&] { return tik_embedding_bwd(ctx, gp, ip, tp, type, accumulate, scale, T, V, H, ws.p, ws.bytes, st); }), ctx);
    return wrap(table_in, made);
}

// TIK_GATE_* of a gate [H] or [T,1]
int gate_kind(const at::Tensor* gate, int64_t T, int64_t H) {
    if (!gate) return TIK_GATE_NONE;
    if (gate->dim() == 2) {
        want_sizes(*gate, {T, 1}, "gate");
        return TIK_GATE_TOKEN;
    }
    want_sizes(*gate, {H}, "gate");
    return TIK_GATE_CHANNEL;
}

PyObject* block_norm(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const at::Tensor &x = on(dev, a.tensor()), &res = on(dev, a.tensor());
    const at::Tensor* w = on(dev, a.opt());
    const float eps = a.real();
    const at::Tensor *post = on(dev, a.opt()), *gate = on(dev, a.opt());
    const float branch_scale = a.real();
    const at::Tensor *s_in = on(dev, a.opt()), *y_in = on(dev, a.opt());
    want_rank(x, 2);
    const int64_t T = x.size(0);
    const int H = dim(x, 1), kind = gate_kind(gate, T, H);
    want_sizes(res, {T, H}, "residual");
    want_sizes(w, {H}, "weight");
    want_sizes(post, {H}, "post_weight");
    want_sizes(s_in, {T, H}, "s");
    want_sizes(y_in, {T, H}, "y");
    if (y_in && !w) raise(PyExc_ValueError, "y needs weight");
    at::Tensor made_s, made_y;
    const int64_t rows = Pool::room(2 * T * H);
    Pool pool((s_in ? 0 : rows) + (w && !y_in ? rows : 0), x);
    if (!s_in) made_s = pool.take({T, H}, at::kBFloat16, x);
    if (w && !y_in) made_y = pool.take({T, H}, at::kBFloat16, x);
    const at::Tensor &s = s_in ? *s_in : made_s, *y = !w ? nullptr : y_in ? y_in : &made_y;
    void *xp = bf(x), *rp = bf(res), *wp = bf(w), *pp = bf(post), *gp = bf(gate), *sp = bf(s), *yp = bf(y), *st = stream();
    check(unlocked([&] { return tik_block_norm(ctx, xp, rp, pp, gp, kind, branch_scale, wp, sp, yp, eps, T, H, st); }), ctx);
    PyObject* a0 = Py_None;
    if (w) a0 = wrap(y_in, made_y);
    else Py_INCREF(Py_None);
    PyObject* a1 = wrap(s_in, made_s);
    return Py_BuildValue("(NN)", a0, a1);
}

PyObject* block_norm_bwd(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const at::Tensor *dy = on(dev, a.opt()), *ds = on(dev, a.opt()), *x = on(dev, a.opt());
    const at::Tensor& s = on(dev, a.tensor());
    const at::Tensor* w = on(dev, a.opt());
    const float eps = a.real();
    const at::Tensor *post = on(dev, a.opt()), *gate = on(dev, a.opt());
    const float branch_scale = a.real();
    const at::Tensor* ws_in = on(dev, a.opt());
    want_rank(s, 2);
    const int64_t T = s.size(0);
    const int H = dim(s, 1), kind = gate_kind(gate, T, H);
    want_sizes(dy, {T, H}, "d_y");
    want_sizes(ds, {T, H}, "d_s");
    want_sizes(x, {T, H}, "x");
    want_sizes(w, {H}, "weight");
    want_sizes(post, {H}, "post_weight");
    if (!dy != !w) raise(PyExc_ValueError, "d_y and weight go together");
    if (!dy && !ds) raise(PyExc_ValueError, "neither d_y nor d_s");
    if (!x && (post || gate)) raise(PyExc_ValueError, "post_weight and gate need x");
    const size_t need = tik_workspace_bytes(TIK_OP_BLOCK_NORM_BWD, T, 0, 0, 0, 0, H, 0);
    const int64_t rows = Pool::room(2 * T * H), scratch = ws_in ? 0 : static_cast<int64_t>(need);
    // the fp32 gradients are parts of one allocation in any case, each at a multiple of 16 bytes
    const int64_t part[3] = {w ? H : 0, post ? H : 0, gate ? gate->numel() : 0}, parts = part[0] + part[1] + part[2];
    Pool pool((x ? 2 : 1) * rows + Pool::room(4 * parts) + Pool::room(scratch), s);
    at::Tensor made[5];
    made[1] = pool.take({T, H}, at::kBFloat16, s);
    if (x) made[0] = pool.take({T, H}, at::kBFloat16, s);
    if (parts > 0) {
        const at::Tensor whole = pool.take({parts}, at::kFloat, s);
        const int64_t at = whole.storage_offset();
        if (w) made[2] = part_of(whole, at, {H}, at::kFloat);
        if (post) made[3] = part_of(whole, at + part[0], {H}, at::kFloat);
        if (gate) made[4] = part_of(whole, at + part[0] + part[1], gate->sizes(), at::kFloat);
    }
    Scratch ws;
    if (ws_in) {
        ws.use(*ws_in);
    } else if (need > 0) {
        ws.own = pool.take({scratch}, at::kByte, s);
        ws.p = ws.own.data_ptr();
        ws.bytes = need;
    }
    auto opt = [](const at::Tensor& t) { return t.defined() ? &t : nullptr; };
    void *dyp = bf(dy), *dsp = bf(ds), *xp = bf(x), *sp = bf(s), *wp = bf(w), *pp = bf(post), *gp = bf(gate), *dxp = bf(opt(made[0])),
         *drp = bf(made[1]), *st = stream();
    float *dwp = f32(opt(made[2])), *dpp = f32(opt(made[3])), *dgp = f32(opt(made[4]));
    check(unlocked([&] { return tik_block_norm_bwd(ctx, dyp, dsp, xp, sp, pp, gp, kind, branch_scale, wp, eps, dxp, drp, dwp, dpp, dgp,
                                                   T, H, ws.p, ws.bytes, st); }), ctx);
    PyObject* out[5];
    for (int i = 0; i < 5; ++i) {
        out[i] = Py_None;
        if (made[i].defined()) out[i] = THPVariable_Wrap(made[i]);
        else Py_INCREF(Py_None);
    }
    return Py_BuildValue("(NNNNN)", out[0], out[1], out[2], out[3], out[4]);
}

// A Python list or tuple of gradients as the arrays of the C interface.
struct GradArgs {
    std::vector<void*> ptrs;
    std::vector<int64_t> numel;
    std::vector<int> types;
    int n = 0;
    GradArgs(PyObject* list, int device) {
        if (!PyList_Check(list) && !PyTuple_Check(list)) raise(PyExc_TypeError, "expected a list or tuple of tensors");
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(list);
        if (count > INT32_MAX) raise(PyExc_OverflowError, "too many tensors");
        n = static_cast<int>(count);
        ptrs.reserve(n);
        numel.reserve(n);
        types.reserve(n);
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* o = PySequence_Fast_GET_ITEM(list, i);
            if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string("expected a tensor, got ") + Py_TYPE(o)->tp_name);
            const at::Tensor& t = on(device, THPVariable_Unpack(o));
            types.push_back(element_type(t));
            ptrs.push_back(ptr(t));
            numel.push_back(t.numel());
        }
    }
};

// The norm's own tensor and the scratch of a gradient call, given or made; both made are parts of one allocation.
struct GradNorm {
    at::Tensor made;
    float* norm = nullptr;
    Scratch ws;
    GradNorm(const at::Tensor* norm_in, const at::Tensor* ws_in, int n, int device, bool scratch) {
        const size_t need = scratch ? tik_workspace_bytes(TIK_OP_GRAD_NORM, n, 0, 0, 0, 0, 0, 0) : 0;
        if (ws_in) ws.use(*ws_in);
        if (norm_in) {
            want_sizes(*norm_in, {1}, "norm");
            norm = f32(norm_in);
            if (!ws_in && need > 0) ws.make(need, *norm_in);
            return;
        }
        constexpr int64_t SKIP = 4;                          // floats, so that the scratch keeps its alignment
        const at::Tensor whole = at::detail::empty_cuda({SKIP + (ws_in ? 0 : static_cast<int64_t>(need / sizeof(float)))}, at::kFloat,
                                                        at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(device)), std::nullopt);
        made = part_of(whole, 0, {1}, at::kFloat);
        norm = f32(&made);
        if (!ws_in) {
            ws.p = norm + SKIP;
            ws.bytes = need;
        }
    }
};

PyObject* grad_norm(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const GradArgs g(a.next(), dev);
    const at::Tensor *norm_in = on(dev, a.opt()), *ws_in = on(dev, a.opt());
    GradNorm n(norm_in, ws_in, g.n, dev, true);
    void* st = stream();
    check(unlocked([&] { return tik_grad_norm(ctx, g.ptrs.data(), g.numel.data(), g.types.data(), g.n, n.norm, n.ws.p, n.ws.bytes, st); }), ctx);
    return wrap(norm_in, n.made);
}

PyObject* grad_clip(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const GradArgs g(a.next(), dev);
    const float max_norm = a.real();
    const at::Tensor* norm_in = on(dev, a.opt());
    PyObject* out_list = a.next();
    const at::Tensor* ws_in = on(dev, a.opt());
    std::vector<void*> to;
    if (out_list != Py_None) {
        GradArgs out(out_list, dev);
        if (out.numel != g.numel || out.types != g.types) raise(PyExc_ValueError, "out has other types or sizes than grads");
        to.swap(out.ptrs);
    }
    GradNorm n(norm_in, ws_in, g.n, dev, norm_in == nullptr);
    void* st = stream();
    check(unlocked([&] { return tik_grad_clip(ctx, g.ptrs.data(), out_list != Py_None ? to.data() : nullptr, g.numel.data(), g.types.data(),
                                              g.n, max_norm, n.norm, norm_in != nullptr, n.ws.p, n.ws.bytes, st); }), ctx);
    return wrap(norm_in, n.made);
}

PyObject* attn_prefill(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor& q = a.tensor();
    const at::Tensor* cu = a.opt();
    const at::Tensor &lens = a.tensor(), &kc = a.tensor(), &vc = a.tensor(), &table = a.tensor();
    const int max_q = a.int32(), max_ctx = a.int32();
    const float scale = a.real();
    const at::Tensor *o_in = a.opt(), *lse = a.opt();
    PyObject* ws_in = a.next();
    want_rank(q, 3);
    const Cache c = cache_of(kc, vc, table);
    at::Tensor made;
    const at::Tensor& o = out_or(o_in, made, q.sizes(), q.scalar_type(), q);
    const int64_t tot = q.size(0);
    const int S = static_cast<int>(lens.numel()), Hq = dim(q, 1), d = dim(q, 2);
    const Scratch ws = plan_ws(ws_in, TIK_OP_ATTN_PREFILL, S, max_ctx, q);
    void *qp = bf(q), *op = bf(o), *st = stream();
    float* lp = f32(lse);
    int32_t *cp = i32(cu), *np = i32(lens);
    check(unlocked([&] { return tik_attn_prefill(ctx, qp, op, lp, cp, np, c.k, c.v, c.table, c.max_blocks, S, tot, max_q,
                                                 max_ctx, Hq, c.Hkv, d, c.page, c.num_pages, scale, ws.p, ws.bytes, st); }), ctx);
    return wrap(o_in, made);
}

PyObject* attn_prefill_kv(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor& q = a.tensor();
    const at::Tensor *k = a.opt(), *v = a.opt(), *cu = a.opt();
    const at::Tensor &lens = a.tensor(), &kc = a.tensor(), &vc = a.tensor(), &table = a.tensor();
    const int max_q = a.int32(), max_ctx = a.int32();
    const float scale = a.real();
    const at::Tensor *o_in = a.opt(), *lse = a.opt();
    PyObject* ws_in = a.next();
    want_rank(q, 3);
    const Cache c = cache_of(kc, vc, table);
    at::Tensor made;
    const at::Tensor& o = out_or(o_in, made, q.sizes(), q.scalar_type(), q);
    const int64_t tot = q.size(0);
    const int S = static_cast<int>(lens.numel()), Hq = dim(q, 1), d = dim(q, 2);
    const Scratch ws = plan_ws(ws_in, TIK_OP_ATTN_PREFILL, S, max_ctx, q);
    void *qp = bf(q), *kp = bf(k), *vp = bf(v), *op = bf(o), *st = stream();
    float* lp = f32(lse);
    int32_t *cp = i32(cu), *np = i32(lens);
    check(unlocked([&] { return tik_attn_prefill_kv(ctx, qp, kp, vp, op, lp, cp, np, c.k, c.v, c.table, c.max_blocks, S,
                                                    tot, max_q, max_ctx, Hq, c.Hkv, d, c.page, c.num_pages, scale, ws.p,
                                                    ws.bytes, st); }), ctx);
    return wrap(o_in, made);
}

PyObject* attn_decode(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &q = a.tensor(), &lens = a.tensor(), &kc = a.tensor(), &vc = a.tensor(), &table = a.tensor();
    const int max_ctx = a.int32();
    const float scale = a.real();
    const at::Tensor *ws_in = a.opt(), *o_in = a.opt(), *lse = a.opt();
    want_rank(q, 3);
    const Cache c = cache_of(kc, vc, table);
    const int B = dim(q, 0), Hq = dim(q, 1), d = dim(q, 2);
    const Scratch ws = sized_ws(ws_in, tik_workspace_bytes(TIK_OP_ATTN_DECODE, B, Hq, c.Hkv, d, max_ctx, 0, 0), q);
    at::Tensor made;
    const at::Tensor& o = out_or(o_in, made, q.sizes(), q.scalar_type(), q);
    void *qp = bf(q), *op = bf(o), *st = stream();
    float* lp = f32(lse);
    int32_t* np = i32(lens);
    check(unlocked([&] { return tik_attn_decode(ctx, qp, op, lp, np, c.k, c.v, c.table, c.max_blocks, B, max_ctx, Hq, c.Hkv, d,
                                                c.page, c.num_pages, scale, ws.p, ws.bytes, st); }), ctx);
    return wrap(o_in, made);
}

PyObject* attn_decode_static(Args a) {
    const at::Tensor &q = a.tensor(), &lens = a.tensor(), &kc = a.tensor(), &vc = a.tensor(), &table = a.tensor();
    const int max_ctx = a.int32();
    const float scale = a.real();
    const at::Tensor& o = a.tensor();
    const at::Tensor *lse = a.opt(), *flags = a.opt();
    want_rank(q, 3);
    const Cache c = cache_of(kc, vc, table);
    const int B = dim(q, 0), Hq = dim(q, 1), d = dim(q, 2);
    void *qp = bf(q), *op = bf(o), *st = stream();
    float* lp = f32(lse);
    int32_t *np = i32(lens), *fp = i32(flags);
    const tik_status rc = unlocked([&] { return tik_attn_decode_static(qp, op, lp, np, c.k, c.v, c.table, c.max_blocks, B, max_ctx,
                                                                       Hq, c.Hkv, d, c.page, c.num_pages, scale, fp, st); });
    return PyLong_FromLong(rc);
}

PyObject* token_logprob(Args a) {
    tik_ctx* ctx = context(current_device());
    const at::Tensor &x = a.tensor(), &w = a.tensor(), &ids = a.tensor();
    const float inv_temperature = a.real();
    const at::Tensor *ws_in = a.opt(), *lp_in = a.opt(), *lse = a.opt();
    want_rank(x, 2);
    want_axis(w, 0);
    const int64_t T = x.size(0);
    const int H = dim(x, 1), V = dim(w, 0);
    const Scratch ws = sized_ws(ws_in, tik_workspace_bytes(TIK_OP_TOKEN_LOGPROB, T, 0, 0, 0, 0, H, V), x);
    at::Tensor made;
    const at::Tensor& lp = out_or(lp_in, made, {T}, at::kFloat, x);
    void *xp = bf(x), *wp = bf(w), *st = stream();
    int32_t* ip = i32(ids);
    float *op = f32(&lp), *sp = f32(lse);
    check(unlocked([&] { return tik_token_logprob(ctx, xp, wp, ip, op, sp, T, H, V, inv_temperature, ws.p, ws.bytes, st); }), ctx);
    return wrap(lp_in, made);
}

PyObject* token_logprob_bwd(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const at::Tensor &g = on(dev, a.tensor()), &x = on(dev, a.tensor()), &w = on(dev, a.tensor()), &ids = on(dev, a.tensor()),
                     &lse = on(dev, a.tensor());
    const float inv_temperature = a.real();
    const int need_hidden = a.int32(), need_table = a.int32();
    const at::Tensor *dx_in = on(dev, a.opt()), *dw_in = on(dev, a.opt());
    const int accumulate = a.int32();
    const at::Tensor* ws_in = on(dev, a.opt());
    want_rank(x, 2);
    want_rank(w, 2);
    const int64_t T = x.size(0);
    const int H = dim(x, 1), V = dim(w, 0);
    want_sizes(w, {V, H}, "lm_head");
    want_sizes(g, {T}, "d_logprob");
    want_sizes(ids, {T}, "target_ids");
    want_sizes(lse, {T}, "lse");
    want_sizes(dx_in, {T, H}, "d_hidden");
    want_sizes(dw_in, {V, H}, "d_lm_head");
    if ((dx_in && !need_hidden) || (dw_in && !need_table)) raise(PyExc_ValueError, "an output that is not needed is given");
    if (!need_hidden && !need_table) raise(PyExc_ValueError, "neither d_hidden nor d_lm_head");
    if (accumulate && !dw_in) raise(PyExc_ValueError, "accumulate needs d_lm_head");
    at::Tensor made_x, made_w;
    const at::Tensor *dx = need_hidden ? &out_or(dx_in, made_x, {T, H}, at::kBFloat16, x) : nullptr;
    const at::Tensor *dw = need_table ? &out_or(dw_in, made_w, {V, H}, at::kBFloat16, x) : nullptr;
    const Scratch ws = sized_ws(ws_in, tik_workspace_bytes(TIK_OP_TOKEN_LOGPROB_BWD, T, 0, 0, 0, 0, H, V), x);
    const int type = dw ? element_type(*dw) : TIK_DTYPE_BF16;
    void *xp = bf(x), *wp = bf(w), *dxp = bf(dx), *dwp = dw ? ptr(*dw) : nullptr, *st = stream();
    const float *gp = f32(&g), *lp = f32(&lse);
    const int32_t* ip = i32(ids);
    check(unlocked([&] { return tik_token_logprob_bwd(ctx, gp, xp, wp, ip, lp, dxp, dwp, type, accumulate, T, H, V, inv_temperature, ws.p,
                                                      ws.bytes, st); }), ctx);
    PyObject *a0 = Py_None, *a1 = Py_None;
    if (dx) a0 = wrap(dx_in, made_x);
    else Py_INCREF(Py_None);
    if (dw) a1 = wrap(dw_in, made_w);
    else Py_INCREF(Py_None);
    return Py_BuildValue("(NN)", a0, a1);
}

PyObject* policy_loss(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const at::Tensor &lp = on(dev, a.tensor()), &old = on(dev, a.tensor()), &adv = on(dev, a.tensor());
    const at::Tensor *weight = on(dev, a.opt()), *ref = on(dev, a.opt()), *cu = on(dev, a.opt());
    const float low = a.real(), high = a.real(), dual = a.real(), kl = a.real();
    const int reduction = a.int32();
    const float scale = a.real();
    const int grad = a.int32();
    const at::Tensor *d_in = on(dev, a.opt()), *ws_in = on(dev, a.opt());
    want_rank(lp, 1);
    const int64_t T = lp.size(0);
    int S = 0;
    if (cu) {
        want_rank(*cu, 1);
        S = dim(*cu, 0) - 1;
        if (S < 0) raise(PyExc_ValueError, "cu_seqlens needs an element at least");
    }
    const bool per_sequence = adv.dim() == 2;
    want_sizes(old, {T}, "old_logprob");
    if (per_sequence) want_sizes(adv, {S, 1}, "advantage");
    else want_sizes(adv, {T}, "advantage");
    want_sizes(weight, {T}, "weight");
    want_sizes(ref, {T}, "ref_logprob");
    want_sizes(d_in, {T}, "d_logprob");
    if (d_in && !grad) raise(PyExc_ValueError, "an output that is not needed is given");
    const size_t need = tik_workspace_bytes(TIK_OP_POLICY_LOSS, T, 0, 0, 0, S, 0, 0);
    // loss and stats are parts of one storage, with the gradient and the scratch where those are small
    constexpr int64_t STATS = 5, SKIP = 4;                   // floats
    const int64_t rows = Pool::room(4 * T), small = Pool::room(4 * (SKIP + STATS)), scratch = ws_in ? 0 : Pool::room(static_cast<int64_t>(need));
    Pool pool((grad && !d_in ? rows : 0) + small + scratch, lp);
    const at::Tensor both = pool.take({SKIP + STATS}, at::kFloat, lp);
    const at::Tensor loss = part_of(both, both.storage_offset(), {1}, at::kFloat);
    const at::Tensor stats = part_of(both, both.storage_offset() + SKIP, {STATS}, at::kFloat);
    at::Tensor made;
    if (grad && !d_in) made = pool.take({T}, at::kFloat, lp);
    const at::Tensor* d = !grad ? nullptr : d_in ? d_in : &made;
    Scratch ws;
    if (ws_in) {
        ws.use(*ws_in);
    } else {
        ws.own = pool.take({static_cast<int64_t>(need)}, at::kByte, lp);
        ws.p = ws.own.data_ptr();
        ws.bytes = need;
    }
    const float *lpp = f32(&lp), *op = f32(&old), *ap = f32(&adv), *wp = f32(weight), *rp = f32(ref);
    float *lossp = f32(&loss), *dp = f32(d), *sp = f32(&stats);
    const int32_t* cp = i32(cu);
    void* st = stream();
    check(unlocked([&] { return tik_policy_loss(ctx, lpp, op, ap, per_sequence, wp, rp, cp, S, T, low, high, dual, kl, reduction, scale, lossp,
                                                dp, sp, ws.p, ws.bytes, st); }), ctx);
    PyObject *a0 = THPVariable_Wrap(loss), *a1 = Py_None, *a2 = THPVariable_Wrap(stats);
    if (d) a1 = wrap(d_in, made);
    else Py_INCREF(Py_None);
    return Py_BuildValue("(NNN)", a0, a1, a2);
}

// A Python list or tuple of tensors of one of some types, as a C array of their addresses.
struct ListArgs {
    std::vector<void*> ptrs;
    ListArgs(PyObject* list, int device, const char* name, const std::vector<int64_t>& numel, std::initializer_list<at::ScalarType> types,
             int64_t per, bool may_lack) {
        if (!PyList_Check(list) && !PyTuple_Check(list)) raise(PyExc_TypeError, std::string(name) + ": expected a list or tuple of tensors");
        if (PySequence_Fast_GET_SIZE(list) != static_cast<Py_ssize_t>(numel.size()))
            raise(PyExc_ValueError, std::string(name) + " has another length than params");
        ptrs.reserve(numel.size());
        for (size_t i = 0; i < numel.size(); ++i) {
            PyObject* o = PySequence_Fast_GET_ITEM(list, static_cast<Py_ssize_t>(i));
            if (may_lack && o == Py_None) {
                ptrs.push_back(nullptr);
                continue;
            }
            if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string("expected a tensor, got ") + Py_TYPE(o)->tp_name);
            const at::Tensor& t = on(device, THPVariable_Unpack(o));
            bool known = false;
            for (const at::ScalarType type : types) known = known || t.scalar_type() == type;
            if (!known) raise_tik(std::string(name) + ": unexpected dtype " + at::toString(t.scalar_type()));
            if (t.numel() != (numel[i] + per - 1) / per) raise(PyExc_ValueError, std::string(name) + " has other sizes than params");
            ptrs.push_back(ptr(t));
        }
    }
};

PyObject* adamw(Args a) {
    const int dev = current_device();
    tik_ctx* ctx = context(dev);
    const GradArgs p(a.next(), dev), g(a.next(), dev);
    if (p.numel != g.numel) raise(PyExc_ValueError, "grads has other sizes than params");
    PyObject *m_list = a.next(), *v_list = a.next();
    auto number = [&](double& value, const at::Tensor*& tensor, at::ScalarType type, const char* name) {
        PyObject* o = a.next();
        if (THPVariable_Check(o)) {
            tensor = &on(dev, THPVariable_Unpack(o));
            want_sizes(*tensor, {1}, name);
            ptr(*tensor, type);
            return;
        }
        value = PyFloat_AsDouble(o);
        if (value == -1.0 && PyErr_Occurred()) throw PyError{};
    };
    double lr = 0.0, step = 1.0;
    const at::Tensor *lr_t = nullptr, *step_t = nullptr;
    number(lr, lr_t, at::kFloat, "lr");
    number(step, step_t, at::kInt, "step");
    if (!(step >= 0.0 && step < 9.0e15) || step != static_cast<double>(static_cast<int64_t>(step))) raise(PyExc_ValueError, "step must be a whole number");
    const double beta1 = a.dbl(), beta2 = a.dbl(), eps = a.dbl(), decay = a.dbl();
    PyObject *master_list = a.next(), *ms_list = a.next(), *vs_list = a.next();
    const at::Tensor* norm = on(dev, a.opt());
    want_sizes(norm, {1}, "norm");
    const float max_norm = a.real();
    PyObject* seed_in = a.next();
    uint32_t seed = 0;
    const bool stochastic = seed_in != Py_None;
    if (stochastic) {
        seed = static_cast<uint32_t>(PyLong_AsUnsignedLongLongMask(seed_in));
        if (PyErr_Occurred()) throw PyError{};
    }
    if ((ms_list == Py_None) != (vs_list == Py_None)) raise(PyExc_ValueError, "the moments' scales go together");
    const bool state8 = ms_list != Py_None;
    const at::ScalarType state = state8 ? at::kFloat8_e4m3fn : at::kFloat;
    const std::vector<int64_t>& n = p.numel;
    const ListArgs m(m_list, dev, "exp_avg", n, {state}, 1, false), v(v_list, dev, "exp_avg_sq", n, {state}, 1, false);
    std::vector<void*> master, ms, vs;
    if (master_list != Py_None) master = ListArgs(master_list, dev, "master", n, {at::kFloat}, 1, true).ptrs;
    if (state8) {
        ms = ListArgs(ms_list, dev, "exp_avg_scale", n, {at::kFloat8_e8m0fnu, at::kByte}, 32, false).ptrs;
        vs = ListArgs(vs_list, dev, "exp_avg_sq_scale", n, {at::kFloat8_e8m0fnu, at::kByte}, 32, false).ptrs;
    }
    auto floats = [](const std::vector<void*>& l) { return l.empty() ? nullptr : reinterpret_cast<float* const*>(l.data()); };
    auto bytes = [](const std::vector<void*>& l) { return l.empty() ? nullptr : reinterpret_cast<uint8_t* const*>(l.data()); };
    const float *lrp = f32(lr_t), *np = f32(norm);
    const int32_t* stp = i32(step_t);
    void* st = stream();
    check(unlocked([&] { return tik_adamw(ctx, p.ptrs.data(), p.types.data(), g.ptrs.data(), g.types.data(), floats(master), m.ptrs.data(),
                                          v.ptrs.data(), bytes(ms), bytes(vs), state8 ? TIK_DTYPE_E4M3 : TIK_DTYPE_FP32, n.data(), p.n, lr, beta1,
                                          beta2, eps, decay, static_cast<int64_t>(step), lrp, stp, np, max_norm, stochastic, seed, st); }), ctx);
    Py_RETURN_NONE;
}

PyObject* context_handle(Args a) {           // device ordinal (or None: the current device) -> the context's address
    PyObject* o = a.next();
    int device = current_device();
    if (o != Py_None) {
        --a.i;
        device = a.int32();
    }
    return PyLong_FromVoidPtr(context(device));
}

PyObject* init(Args a) {
    PyObject* e = a.next();
    Py_INCREF(e);
    Py_XSETREF(g_error, e);
    Py_RETURN_NONE;
}

template <PyObject* (*F)(Args)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS                         // torch's own errors (out of memory among them) keep their types
    try {
        return F(Args{args, n});
    } catch (const PyError&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

#define TIK_DEF(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    TIK_DEF(init), TIK_DEF(context_handle), TIK_DEF(attn_train_fwd), TIK_DEF(attn_train_bwd), TIK_DEF(kv_cache_write),
    TIK_DEF(qk_norm_rope_kv_write), TIK_DEF(rmsnorm), TIK_DEF(swiglu), TIK_DEF(linear), TIK_DEF(attn_prefill),
    TIK_DEF(attn_prefill_kv), TIK_DEF(attn_decode), TIK_DEF(attn_decode_static), TIK_DEF(token_logprob), TIK_DEF(embedding),
    TIK_DEF(embedding_bwd), TIK_DEF(block_norm), TIK_DEF(block_norm_bwd), TIK_DEF(grad_norm), TIK_DEF(grad_clip),
    TIK_DEF(token_logprob_bwd), TIK_DEF(policy_loss), TIK_DEF(adamw),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_tikbind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tikbind(void) { return PyModule_Create(&module_def); }
