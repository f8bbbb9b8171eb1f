// swr_binding.cpp -- the Python binding's fast path: tensors to pointers and
// strides, outputs allocated, one call of the C ABI, in native code.
//
// Host time binds small calls: checking, allocating and marshalling one call
// in Python and ctypes took about 17 us, twice what its kernel takes on a
// problem of a few MB.  Each function here takes one entry point's arguments in
// a fixed order and handles the ordinary call: plain strided GPU tensors that
// pass every check.  It returns None for anything else, and the caller then
// runs the Python path, which raises what there is to raise and which serves
// every call where this module cannot be built or loaded; a status of the C
// ABI comes back as an int.  Nothing is kept between calls: the C ABI's entry
// points are the only state, bound when the library is loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/swr.h"
#include "../../include/swr_hybrid.h"

// What this module was built from and for; the build looks for it in the file.
extern "C" __attribute__((used)) const char swr_binding_key[] = "swr-binding-key:" SWR_BINDING_KEY;

namespace {

// The C ABI's entry points (the addresses that the loaded library has).
struct Abi {
    decltype(&swr_forward) forward;
    decltype(&swr_backward) backward;
    decltype(&swr_exact_workspace_bytes) exact_workspace_bytes;
    decltype(&swr_exact_forward) exact_forward;
    decltype(&swr_exact_backward) exact_backward;
    decltype(&swr_step) step;
    decltype(&swr_exact_step) exact_step;
    decltype(&swr_decode_state) decode_state;
    decltype(&swr_uniform_forward) uniform_forward;
    decltype(&swr_uniform_backward) uniform_backward;
    decltype(&swr_forward_shared_gates) forward_shared_gates;
    decltype(&swr_backward_shared_gates) backward_shared_gates;
    decltype(&swr_shared_gates_workspace_bytes) shared_gates_workspace_bytes;
};
constexpr int kEntries = sizeof(Abi) / sizeof(void*);
union {
    Abi fn;
    void* address[kEntries];
} abi;

// Those of the hybrid model's operators.
struct HybridAbi {
    decltype(&swr_rms_norm) rms_norm;
    decltype(&swr_rms_norm_workspace_bytes) rms_norm_workspace_bytes;
    decltype(&swr_rms_norm_backward) rms_norm_backward;
    decltype(&swr_fp4_linear) fp4_linear;
    decltype(&swr_block_tables) block_tables;
    decltype(&swr_cache_append) cache_append;
    decltype(&swr_paged_workspace_bytes) paged_workspace_bytes;
    decltype(&swr_paged_attention) paged_attention;
};
constexpr int kHybridEntries = sizeof(HybridAbi) / sizeof(void*);
union {
    HybridAbi fn;
    void* address[kHybridEntries];
} hybrid;

// Arguments of one call, taken in order; ok turns false at the first that is
// not what the fast path handles.
struct Args {
    PyObject* const* v;
    bool ok = true;

    const at::Tensor& tensor() {   // a plain torch.Tensor or Parameter
        static const at::Tensor undefined;
        PyObject* o = *v++;
        if (!THPVariable_CheckExact(o)) { ok = false; return undefined; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || t.layout() != c10::kStrided) ok = false;
        return t;
    }
    at::Tensor optional() {        // None or a tensor
        if (*v == Py_None) { ++v; return {}; }
        return tensor();
    }
    int64_t integer() {
        PyObject* o = *v++;
        if (!PyLong_Check(o)) { ok = false; return 0; }
        const int64_t r = PyLong_AsLongLong(o);
        if (r == -1 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return r;
    }
    bool truth() { return *v++ == Py_True; }
    double real() {
        PyObject* o = *v++;
        if (!PyFloat_Check(o)) { ok = false; return 0; }
        return PyFloat_AS_DOUBLE(o);
    }
};

bool same_layout(const at::Tensor& x, const at::Tensor& t) {
    return t.scalar_type() == x.scalar_type() && t.device() == x.device() && t.sizes() == x.sizes() &&
           t.strides() == x.strides();
}

bool float_state(const at::Tensor& t, const at::Tensor& x, at::IntArrayRef shape) {
    return t.scalar_type() == at::kFloat && t.device() == x.device() && t.sizes() == shape && t.is_contiguous();
}

// The problem of x, a and the scalars, with every check of the Python path.
bool problem(const at::Tensor& x, const at::Tensor& a, int64_t block, int64_t flags, int64_t run_len,
             swr_problem_t* p) {
    if (x.dim() != 4 || !x.is_cuda() || a.device() != x.device() || a.scalar_type() != x.scalar_type()) return false;
    const bool pc = a.dim() == 4;
    if (pc ? a.sizes() != x.sizes() || a.strides() != x.strides()
           : a.dim() != 3 || a.sizes() != x.sizes().slice(0, 3))
        return false;
    if (x.stride(3) != 1 && x.size(3) > 1) return false;
    if (x.scalar_type() != at::kBFloat16 && x.scalar_type() != at::kFloat) return false;
    if (block <= 0) return false;
    *p = swr_problem_t{};
    p->abi_version = SWR_ABI_VERSION;
    p->dtype = x.scalar_type() == at::kBFloat16 ? SWR_DTYPE_BF16 : SWR_DTYPE_F32;
    p->B = x.size(0); p->T = x.size(1); p->H = x.size(2); p->D = x.size(3);
    p->block = block;
    p->flags = (uint32_t)flags | (pc ? SWR_FLAG_PER_CHANNEL_DECAY : 0);
    p->sx_b = x.stride(0); p->sx_t = x.stride(1); p->sx_h = x.stride(2);
    p->sa_b = a.stride(0); p->sa_t = a.stride(1); p->sa_h = a.stride(2);
    p->run_len = run_len;
    return true;
}

// Allocating and launching run without the interpreter's lock, so that other
// Python threads go on where one waits for the allocator or a full queue.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

template <typename F, typename... A>
int call(F entry, A... args) {
    const Unlocked unlocked;
    return entry(args...);
}

void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* fptr(const at::Tensor& t) { return (float*)ptr(t); }

at::Tensor like(const at::Tensor& x) {
    const Unlocked unlocked;
    return at::empty_strided(x.sizes(), x.strides(), x.options().requires_grad(false));
}
at::Tensor floats(const at::Tensor& x, at::IntArrayRef shape) {
    const Unlocked unlocked;
    return at::empty(shape, x.options().dtype(at::kFloat).requires_grad(false));
}
at::Tensor decay_gradient(const at::Tensor& a) {
    const Unlocked unlocked;
    return at::empty_strided(a.sizes(), a.strides(), a.options().dtype(at::kFloat).requires_grad(false));
}

std::array<int64_t, 4> carrier_shape(const swr_problem_t& p) {
    return {p.B, p.H, (p.T + p.block - 1) / p.block, p.D};
}

// The stream argument (an address, or None: x's device's current stream).
void* stream_of(PyObject* o, const at::Tensor& x, bool* ok) {
    if (o == Py_None) return (void*)c10::hip::getCurrentHIPStream(x.device().index()).stream();
    if (!PyLong_Check(o)) { *ok = false; return nullptr; }
    return PyLong_AsVoidPtr(o);
}

// n floats that only one call's kernels use, on its stream (o, st: the stream
// argument and its address).  The tensor is let go when the call returns, so
// it is taken from that stream's memory: whoever gets it next is ordered
// behind those kernels there, and it has no other stream's work pending.
at::Tensor workspace(const at::Tensor& x, int64_t n, PyObject* o, void* st) {
    if (o == Py_None) return floats(x, {n});
    struct On {
        const c10::hip::HIPStream before;
        On(c10::DeviceIndex d, void* s) : before(c10::hip::getCurrentHIPStream(d)) {
            c10::hip::setCurrentHIPStream(s ? c10::hip::getStreamFromExternal((hipStream_t)s, d)
                                            : c10::hip::getDefaultHIPStream(d));
        }
        ~On() { c10::hip::setCurrentHIPStream(before); }
    } on(x.device().index(), st);
    return floats(x, {n});
}

PyObject* none() { Py_RETURN_NONE; }

PyObject* results(int rc, std::initializer_list<at::Tensor> ts) {
    if (rc != 0) return PyLong_FromLong(rc);
    if (ts.size() == 1) return THPVariable_Wrap(*ts.begin());
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = nullptr;
        if (t.defined()) o = THPVariable_Wrap(t);
        else { o = Py_None; Py_INCREF(o); }
        if (!o) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// x, a, b, c of the calls whose b and c have x's layout.
struct Inputs {
    const at::Tensor &x, &a, &b, &c;
    explicit Inputs(Args& g) : x(g.tensor()), a(g.tensor()), b(g.tensor()), c(g.tensor()) {}
    bool check(const Args& g, int64_t block, int64_t flags, int64_t run_len, swr_problem_t* p) const {
        return g.ok && problem(x, a, block, flags, run_len, p) && same_layout(x, b) && same_layout(x, c);
    }
};

// forward(x, a, b, c, block, flags, run_len, y, carriers, want_carriers, stream) -> (y, carriers)
PyObject* forward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer();
    at::Tensor y = g.optional(), s = g.optional();
    const bool want = g.truth();
    swr_problem_t p;
    if (!in.check(g, block, flags, run_len, &p)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    const auto vs = carrier_shape(p);
    if (!g.ok || (y.defined() && !same_layout(in.x, y)) || (s.defined() && !float_state(s, in.x, vs))) return none();
    if (!y.defined()) y = like(in.x);
    if (want && !s.defined()) s = floats(in.x, vs);
    return results(call(abi.fn.forward, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(y), fptr(s), st), {y, s});
    END_HANDLE_TH_ERRORS
}

// backward(x, a, b, c, dy, carriers, block, flags, run_len, stream) -> (dx, da, db, dc)
PyObject* backward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const at::Tensor& dy = g.tensor();
    const at::Tensor s = g.optional();
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer();
    swr_problem_t p;
    if (!in.check(g, block, flags, run_len, &p) || !same_layout(in.x, dy)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    if (!g.ok || (s.defined() && !float_state(s, in.x, carrier_shape(p)))) return none();
    const at::Tensor dx = like(in.x), db = like(in.x), dc = like(in.x), da = decay_gradient(in.a);
    return results(call(abi.fn.backward, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(dy), fptr(s), ptr(dx),
                          fptr(da),
                                   ptr(db), ptr(dc), st), {dx, da, db, dc});
    END_HANDLE_TH_ERRORS
}

// exact_forward(x, a, b, c, block, flags, run_len, h0, want_carriers, want_h_last, stream)
//     -> (y, carriers, h_last)
PyObject* exact_forward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer();
    const at::Tensor h0 = g.optional();
    const bool want_v = g.truth(), want_h = g.truth();
    swr_problem_t p;
    if (!in.check(g, block, flags, run_len, &p)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    const std::array<int64_t, 3> hs{p.B, p.H, p.D};
    if (!g.ok || (h0.defined() && !float_state(h0, in.x, hs))) return none();
    const int64_t ws = abi.fn.exact_workspace_bytes(&p);
    if (ws < 0) return none();
    const at::Tensor y = like(in.x);
    at::Tensor s, hl;
    if (want_v) s = floats(in.x, carrier_shape(p));
    if (want_h) hl = floats(in.x, hs);
    const at::Tensor work = workspace(in.x, std::max<int64_t>(ws / 4, 1), *g.v, st);
    return results(call(abi.fn.exact_forward, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), fptr(h0), ptr(y), fptr(s),
                                        fptr(hl), ptr(work), st), {y, s, hl});
    END_HANDLE_TH_ERRORS
}

// exact_backward(x, a, b, c, dy, carriers, block, flags, run_len, h0, dh_last, want_dh0, stream)
//     -> (dx, da, db, dc, dh0)
PyObject* exact_backward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const at::Tensor &dy = g.tensor(), &s = g.tensor();
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer();
    const at::Tensor h0 = g.optional(), dhl = g.optional();
    const bool want = g.truth();
    swr_problem_t p;
    if (!in.check(g, block, flags, run_len, &p) || !same_layout(in.x, dy)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    const std::array<int64_t, 3> hs{p.B, p.H, p.D};
    if (!g.ok || !float_state(s, in.x, carrier_shape(p)) || (h0.defined() && !float_state(h0, in.x, hs)) ||
        (dhl.defined() && !float_state(dhl, in.x, hs)))
        return none();
    const int64_t ws = abi.fn.exact_workspace_bytes(&p);
    if (ws < 0) return none();
    const at::Tensor dx = like(in.x), db = like(in.x), dc = like(in.x), da = decay_gradient(in.a);
    at::Tensor dh0;
    if (want) dh0 = floats(in.x, hs);
    const at::Tensor work = workspace(in.x, std::max<int64_t>(ws / 4, 1), *g.v, st);
    return results(call(abi.fn.exact_backward, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(dy), fptr(h0),
                          fptr(s),
                                         fptr(dhl), ptr(dx), fptr(da), ptr(db), ptr(dc), fptr(dh0), ptr(work), st),
                   {dx, da, db, dc, dh0});
    END_HANDLE_TH_ERRORS
}

// step(x, a, b, c, block, flags, t0, state, y, stream) -> y; t0 < 0: the exact recurrence
PyObject* step(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const int64_t block = g.integer(), flags = g.integer(), t0 = g.integer();
    const at::Tensor& state = g.tensor();
    at::Tensor y = g.optional();
    swr_problem_t p;
    if (!in.check(g, block, flags, 0, &p)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    const std::array<int64_t, 4> js{p.B, p.H, 2, p.D};
    const std::array<int64_t, 3> hs{p.B, p.H, p.D};
    if (!g.ok || !float_state(state, in.x, t0 < 0 ? at::IntArrayRef(hs) : at::IntArrayRef(js)) ||
        (y.defined() && !same_layout(in.x, y)))
        return none();
    if (!y.defined()) y = like(in.x);
    const int rc = t0 < 0 ? call(abi.fn.exact_step, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(y),
          fptr(state), st)
                          : call(abi.fn.step, &p, t0, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(y), fptr(state),
                                st);
    return results(rc, {y});
    END_HANDLE_TH_ERRORS
}

// decode_state(x, a, carriers, block, flags, stream) -> state
PyObject* decode_state(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const at::Tensor &x = g.tensor(), &a = g.tensor(), &s = g.tensor();
    const int64_t block = g.integer(), flags = g.integer();
    swr_problem_t p;
    if (!g.ok || !problem(x, a, block, flags, 0, &p)) return none();
    void* st = stream_of(*g.v, x, &g.ok);
    if (!g.ok || !float_state(s, x, carrier_shape(p))) return none();
    const at::Tensor state = floats(x, {p.B, p.H, 2, p.D});
    return results(call(abi.fn.decode_state, &p, ptr(a), fptr(s), fptr(state), st), {state});
    END_HANDLE_TH_ERRORS
}

// uniform_forward(x, a, b, c, window, flags, run_len, stream) -> y
PyObject* uniform_forward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer();
    swr_problem_t p;
    if (!in.check(g, block, flags, run_len, &p)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    if (!g.ok) return none();
    const at::Tensor y = like(in.x);
    return results(call(abi.fn.uniform_forward, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(y), st), {y});
    END_HANDLE_TH_ERRORS
}

// uniform_backward(x, a, b, c, dy, window, flags, run_len, stream) -> (dx, da, db, dc)
PyObject* uniform_backward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const at::Tensor& dy = g.tensor();
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer();
    swr_problem_t p;
    if (!in.check(g, block, flags, run_len, &p) || !same_layout(in.x, dy)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    if (!g.ok) return none();
    const at::Tensor dx = like(in.x), db = like(in.x), dc = like(in.x), da = decay_gradient(in.a);
    return results(call(abi.fn.uniform_backward, &p, ptr(in.x), ptr(in.a), ptr(in.b), ptr(in.c), ptr(dy), ptr(dx),
                          fptr(da),
                                           ptr(db), ptr(dc), st), {dx, da, db, dc});
    END_HANDLE_TH_ERRORS
}

// The gates' checks: [B, T, H / group, D] with contiguous channels, b and c alike.
bool gates(const Args& g, const at::Tensor& x, const at::Tensor& a, const at::Tensor& b, const at::Tensor& c,
           int64_t group, int64_t block, int64_t flags, int64_t run_len, swr_problem_t* p) {
    if (!g.ok || !problem(x, a, block, flags, run_len, p) || group < 1 || p->H % group != 0) return false;
    const std::array<int64_t, 4> gs{p->B, p->T, p->H / group, p->D};
    return b.sizes() == at::IntArrayRef(gs) && b.scalar_type() == x.scalar_type() && b.device() == x.device() &&
           (b.stride(3) == 1 || p->D <= 1) && same_layout(b, c);
}

// forward_shared_gates(x, a, b, c, block, flags, run_len, group, want_carriers, stream) -> (y, carriers)
PyObject* forward_shared_gates(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer(), group = g.integer();
    const bool want = g.truth();
    swr_problem_t p;
    if (!gates(g, in.x, in.a, in.b, in.c, group, block, flags, run_len, &p)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    if (!g.ok) return none();
    const at::Tensor y = like(in.x);
    at::Tensor s;
    if (want) s = floats(in.x, carrier_shape(p));
    return results(call(abi.fn.forward_shared_gates, &p, group, in.b.strides().data(), ptr(in.x), ptr(in.a), ptr(in.b),
                                               ptr(in.c), ptr(y), fptr(s), st), {y, s});
    END_HANDLE_TH_ERRORS
}

// backward_shared_gates(x, a, b, c, dy, carriers, block, flags, run_len, group, stream) -> (dx, da, db, dc)
PyObject* backward_shared_gates(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const Inputs in(g);
    const at::Tensor &dy = g.tensor(), &s = g.tensor();
    const int64_t block = g.integer(), flags = g.integer(), run_len = g.integer(), group = g.integer();
    swr_problem_t p;
    if (!gates(g, in.x, in.a, in.b, in.c, group, block, flags, run_len, &p) || !same_layout(in.x, dy)) return none();
    void* st = stream_of(*g.v, in.x, &g.ok);
    if (!g.ok || !float_state(s, in.x, carrier_shape(p))) return none();
    const int64_t ws = abi.fn.shared_gates_workspace_bytes(&p, group);
    if (ws < 0) return none();
    const at::Tensor dx = like(in.x), db = like(in.b), dc = like(in.b), da = decay_gradient(in.a);
    at::Tensor work;
    if (ws > 0) work = workspace(in.x, ws / 4, *g.v, st);
    return results(call(abi.fn.backward_shared_gates, &p, group, in.b.strides().data(), ptr(in.x), ptr(in.a), ptr(in.b),
                                                ptr(in.c), ptr(dy), fptr(s), ptr(dx), fptr(da), ptr(db), ptr(dc),
                                                ptr(work), st), {dx, da, db, dc});
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// The hybrid model's operators
// ---------------------------------------------------------------------------

bool float_or_bf16(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat; }
int code_of(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? SWR_DTYPE_BF16 : SWR_DTYPE_F32; }
bool is(const at::Tensor& t, const at::Tensor& x, at::ScalarType type, at::IntArrayRef shape) {
    return t.scalar_type() == type && t.device() == x.device() && t.sizes() == shape;
}
bool dense(const at::Tensor& t, const at::Tensor& x, at::ScalarType type, at::IntArrayRef shape) {
    return is(t, x, type, shape) && t.is_contiguous();
}
at::Tensor made(const at::Tensor& x, at::IntArrayRef shape, at::ScalarType type) {
    return at::empty(shape, x.options().dtype(type).requires_grad(false));
}

// Rows of t: [width], [rows, width] or [outer, inner, width], channels contiguous
// (others go through Python).
bool rows(const at::Tensor& t, int64_t* outer, int64_t* inner, int64_t* so, int64_t* si) {
    const int64_t d = t.dim();
    if (d < 1 || d > 3 || (t.stride(d - 1) != 1 && t.size(d - 1) > 1)) return false;
    *outer = d == 3 ? t.size(0) : 1;
    *inner = d > 1 ? t.size(d - 2) : 1;
    *so = d == 3 ? t.stride(0) : 0;
    *si = d > 1 ? t.stride(d - 2) : 0;
    return true;
}

bool norm_problem(const at::Tensor& x, const at::Tensor& w, double eps, swr_norm_t* n) {
    *n = swr_norm_t{};
    if (!x.is_cuda() || !float_or_bf16(x) || !rows(x, &n->outer, &n->inner, &n->sx_o, &n->sx_i)) return false;
    if (w.device() != x.device() || !float_or_bf16(w) || w.dim() != 1 || w.size(0) != x.size(-1) || !w.is_contiguous())
        return false;
    n->abi_version = SWR_ABI_VERSION;
    n->dtype = n->out_dtype = code_of(x);
    n->weight_dtype = code_of(w);
    n->width = x.size(-1);
    n->eps = (float)eps;
    return true;
}
// Row strides of t, which has x's shape, type and device.
bool norm_rows(const at::Tensor& x, const at::Tensor& t, int64_t* so, int64_t* si) {
    int64_t outer, inner;
    return is(t, x, x.scalar_type(), x.sizes()) && rows(t, &outer, &inner, so, si);
}
// ... of a contiguous one
void dense_rows(const swr_norm_t& n, int64_t* so, int64_t* si) {
    *so = n.inner * n.width;
    *si = n.width;
}

// rms_norm(x, weight, residual, eps, fp8, stream) -> (y, scale, h)
PyObject* rms_norm(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const at::Tensor &x = g.tensor(), &w = g.tensor();
    const at::Tensor r = g.optional();
    const double eps = g.real();
    const bool fp8 = g.truth();
    swr_norm_t n;
    if (!g.ok || !norm_problem(x, w, eps, &n) || (r.defined() && !norm_rows(x, r, &n.sr_o, &n.sr_i))) return none();
    void* st = stream_of(*g.v, x, &g.ok);
    if (!g.ok) return none();
    if (fp8) n.out_dtype = SWR_DTYPE_FP8;
    dense_rows(n, &n.sy_o, &n.sy_i);
    if (r.defined()) dense_rows(n, &n.sh_o, &n.sh_i);
    at::Tensor y, s, h;
    int rc;
    {
        const Unlocked unlocked;
        y = made(x, x.sizes(), fp8 ? at::kFloat8_e4m3fn : x.scalar_type());
        if (fp8) s = made(x, x.sizes().slice(0, x.dim() - 1), at::kFloat);
        if (r.defined()) h = made(x, x.sizes(), x.scalar_type());
        rc = hybrid.fn.rms_norm(&n, ptr(x), ptr(r), ptr(w), ptr(y), fptr(s), ptr(h), st);
    }
    return results(rc, {y, s, h});
    END_HANDLE_TH_ERRORS
}

// rms_norm_backward(h, weight, dy, dh, eps, stream) -> (dx, dweight)
PyObject* rms_norm_backward(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const at::Tensor &h = g.tensor(), &w = g.tensor(), &dy = g.tensor();
    const at::Tensor dh = g.optional();
    const double eps = g.real();
    swr_norm_t n;
    if (!g.ok || !norm_problem(h, w, eps, &n) || !norm_rows(h, dy, &n.sy_o, &n.sy_i) ||
        (dh.defined() && !norm_rows(h, dh, &n.sr_o, &n.sr_i)))
        return none();
    void* st = stream_of(*g.v, h, &g.ok);
    if (!g.ok) return none();
    dense_rows(n, &n.sh_o, &n.sh_i);
    const int64_t ws = hybrid.fn.rms_norm_workspace_bytes(&n);
    if (ws < 0) return none();
    const at::Tensor work = workspace(h, std::max<int64_t>(ws / 4, 4), *g.v, st);
    at::Tensor dx, dw;
    int rc;
    {
        const Unlocked unlocked;
        dx = made(h, h.sizes(), h.scalar_type());
        dw = made(h, w.sizes(), at::kFloat);
        rc = hybrid.fn.rms_norm_backward(&n, ptr(h), ptr(w), ptr(dy), ptr(dh), ptr(dx), fptr(dw), ptr(work), st);
    }
    return results(rc, {dx, dw});
    END_HANDLE_TH_ERRORS
}

bool matrix(const at::Tensor& t) { return t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1); }

// fp4_linear(x, codes, powers, scale, stream) -> y, x a matrix
PyObject* fp4_linear(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const at::Tensor &x = g.tensor(), &c = g.tensor(), &e = g.tensor();
    const at::Tensor s = g.optional();
    const bool fp8 = x.defined() && x.scalar_type() == at::kFloat8_e4m3fn;
    if (!g.ok || !x.is_cuda() || !matrix(x) || !(fp8 || float_or_bf16(x)) || !matrix(c) || !matrix(e)) return none();
    void* st = stream_of(*g.v, x, &g.ok);
    swr_fp4_t p = {};
    p.abi_version = SWR_ABI_VERSION;
    p.M = x.size(0); p.K = x.size(1); p.N = c.size(0);
    const int64_t groups = (p.K + 31) / 32;
    if (!g.ok || !is(c, x, at::kByte, {p.N, 16 * groups}) || !is(e, x, at::kByte, {p.N, groups}) ||
        (s.defined() && !dense(s, x, at::kFloat, {p.M})))
        return none();
    p.dtype = fp8 ? SWR_DTYPE_FP8 : code_of(x);
    p.out_dtype = fp8 ? SWR_DTYPE_BF16 : p.dtype;
    p.sx = x.stride(0); p.sy = p.N; p.sc = c.stride(0); p.sp = e.stride(0);
    at::Tensor y;
    int rc;
    {
        const Unlocked unlocked;
        y = made(x, {p.M, p.N}, fp8 ? at::kBFloat16 : x.scalar_type());
        rc = hybrid.fn.fp4_linear(&p, ptr(x), fptr(s), ptr(c), ptr(e), ptr(y), st);
    }
    return results(rc, {y});
    END_HANDLE_TH_ERRORS
}

// block_tables(lengths, new_tokens, table, stack, count, page_size, tokens, stream)
//     -> (slots, starts, new_lengths, new_count)
PyObject* block_tables(PyObject*, PyObject* const* v, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{v};
    const at::Tensor &n = g.tensor(), &more = g.tensor(), &table = g.tensor(), &stack = g.tensor(), &count = g.tensor();
    swr_tables_t p = {};
    p.page_size = g.integer();
    p.tokens = g.integer();
    if (!g.ok || !n.is_cuda() || n.dim() != 1 || stack.dim() != 1 || !matrix(table) || p.tokens < 0) return none();
    void* st = stream_of(*g.v, n, &g.ok);
    p.abi_version = SWR_ABI_VERSION;
    p.batch = n.size(0); p.max_pages = table.size(1); p.st = table.stride(0); p.free_pages = stack.size(0);
    if (!g.ok || !dense(n, n, at::kInt, {p.batch}) || !dense(more, n, at::kInt, {p.batch}) ||
        !is(table, n, at::kInt, {p.batch, p.max_pages}) || !dense(stack, n, at::kInt, {p.free_pages}) ||
        !is(count, n, at::kInt, {1}))
        return none();
    at::Tensor slots, starts, lengths, left;
    int rc;
    {
        const Unlocked unlocked;
        slots = made(n, {p.tokens}, at::kLong);
        starts = made(n, {p.batch + 1}, at::kInt);
        lengths = made(n, {p.batch}, at::kInt);
        left = made(n, {1}, at::kInt);
        rc = hybrid.fn.block_tables(&p, (const int32_t*)ptr(n), (const int32_t*)ptr(more), (const int32_t*)ptr(stack),
                                    (const int32_t*)ptr(count), (int32_t*)ptr(table), (int64_t*)ptr(slots),
                                    (int32_t*)ptr(starts), (int32_t*)ptr(lengths), (int32_t*)ptr(left), st);
    }
    return results(rc, {slots, starts, lengths, left});
    END_HANDLE_TH_ERRORS
}

bool cache_problem(const at::Tensor& k, const at::Tensor& v, swr_cache_t* c) {
    if (!k.is_cuda() || k.dim() != 4 || !float_or_bf16(k) || !same_layout(k, v) || (k.stride(3) != 1 && k.size(3) > 1))
        return false;
    c->abi_version = SWR_ABI_VERSION;
    c->dtype = code_of(k);
    c->pages = k.size(0); c->page_size = k.size(1); c->heads = k.size(2); c->D = k.size(3);
    c->s_page = k.stride(0); c->s_token = k.stride(1); c->s_head = k.stride(2);
    return true;
}
bool head_rows(const at::Tensor& t, const at::Tensor& cache, at::IntArrayRef shape) {
    return is(t, cache, cache.scalar_type(), shape) && (t.stride(2) == 1 || t.size(2) <= 1);
}

// cache_append(k, v, k_cache, v_cache, slots, stream) -> True
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{a};
    const at::Tensor &k = g.tensor(), &v = g.tensor(), &kc = g.tensor(), &vc = g.tensor(), &slots = g.tensor();
    swr_cache_t c;
    if (!g.ok || !cache_problem(kc, vc, &c) || slots.dim() != 1) return none();
    void* st = stream_of(*g.v, kc, &g.ok);
    const int64_t tokens = slots.size(0);
    const std::array<int64_t, 3> shape{tokens, c.heads, c.D};
    if (!g.ok || !dense(slots, kc, at::kLong, {tokens}) || !head_rows(k, kc, shape) || !head_rows(v, kc, shape))
        return none();
    const int64_t sk[2] = {k.stride(0), k.stride(1)}, sv[2] = {v.stride(0), v.stride(1)};
    const int rc = call(hybrid.fn.cache_append, &c, tokens, sk, sv, ptr(k), ptr(v), (const int64_t*)ptr(slots), ptr(kc),
                        ptr(vc), st);
    if (rc != 0) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// paged_attention(q, k_cache, v_cache, table, lengths, scale, window, want_lse, stream) -> (y, lse)
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t) {
    HANDLE_TH_ERRORS
    Args g{a};
    const at::Tensor &q = g.tensor(), &kc = g.tensor(), &vc = g.tensor(), &table = g.tensor(), &n = g.tensor();
    const double scale = g.real();
    swr_paged_t p = {};
    p.window = g.integer();
    const bool want = g.truth();
    if (!g.ok || !cache_problem(kc, vc, &p.cache) || q.dim() != 3 || !matrix(table)) return none();
    void* st = stream_of(*g.v, kc, &g.ok);
    p.batch = q.size(0); p.q_heads = q.size(1); p.max_pages = table.size(1); p.st = table.stride(0);
    if (!g.ok || p.cache.heads < 1 || p.q_heads < 1 || p.q_heads % p.cache.heads != 0 ||
        !head_rows(q, kc, {p.batch, p.q_heads, p.cache.D}) || !is(table, kc, at::kInt, {p.batch, p.max_pages}) ||
        !dense(n, kc, at::kInt, {p.batch}))
        return none();
    p.sq_b = q.stride(0); p.sq_h = q.stride(1);
    p.sy_b = p.q_heads * p.cache.D; p.sy_h = p.cache.D;
    p.scale = (float)scale;
    const int64_t ws = hybrid.fn.paged_workspace_bytes(&p);
    if (ws < 0) return none();
    const at::Tensor work = workspace(q, std::max<int64_t>(ws / 4, 4), *g.v, st);
    at::Tensor y, lse;
    int rc;
    {
        const Unlocked unlocked;
        y = made(q, q.sizes(), q.scalar_type());
        if (want) lse = made(q, {p.batch, p.q_heads}, at::kFloat);
        rc = hybrid.fn.paged_attention(&p, ptr(q), ptr(kc), ptr(vc), (const int32_t*)ptr(table), (const int32_t*)ptr(n),
                                       ptr(y), fptr(lse), ptr(work), st);
    }
    return results(rc, {y, lse});
    END_HANDLE_TH_ERRORS
}

// bind(address, ...): the C ABI's entry points, in Abi's order
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != kEntries) {
        PyErr_SetString(PyExc_TypeError, "bind: wrong number of entry points");
        return nullptr;
    }
    for (int i = 0; i < kEntries; ++i) abi.address[i] = PyLong_AsVoidPtr(v[i]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// bind_hybrid(address, ...): those of the hybrid model's operators, in HybridAbi's order
PyObject* bind_hybrid(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n != kHybridEntries) {
        PyErr_SetString(PyExc_TypeError, "bind_hybrid: wrong number of entry points");
        return nullptr;
    }
    for (int i = 0; i < kHybridEntries; ++i) hybrid.address[i] = PyLong_AsVoidPtr(v[i]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

#define ENTRY(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind), ENTRY(forward), ENTRY(backward), ENTRY(exact_forward), ENTRY(exact_backward),
                         ENTRY(step), ENTRY(decode_state), ENTRY(uniform_forward), ENTRY(uniform_backward),
                         ENTRY(forward_shared_gates), ENTRY(backward_shared_gates), ENTRY(bind_hybrid),
                         ENTRY(rms_norm), ENTRY(rms_norm_backward), ENTRY(fp4_linear), ENTRY(block_tables),
                         ENTRY(cache_append), ENTRY(paged_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
