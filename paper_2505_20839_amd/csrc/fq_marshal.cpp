// The hot entry points of binding.py with their argument marshalling in native code: check the tensors, get the outputs
// and the scratch from torch's allocator, call the C ABI on the current stream.  A call of one decode layer takes 5 us on
// the GPU; the same steps in Python and ctypes took 11 us on the host, and every small layer waited for them.  The offline calls and
// the packing of a cache too: two caches packed 19.3 us of host time in Python against 17.8 on the GPU, 9.0 here; a 11008 x 4096
// weight, whose quantisation waits for the host to read the exponent, 102 -> 96 us.
//
// Every function returns its result, or an int (a non-zero status of the C ABI), or None for anything it does not take:
// a tensor of another type, dtype, device or layout, a wrong shape, an active torch-function mode, an
// exception of any kind.  binding.py then runs its own form of the call, which decides and raises.  No state is kept but the
// addresses of the C functions, handed over once by bind().
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/fireq.h"
#include "../../include/fireq_chunk.h"
#include "../../include/fireq_kv4_ws.h"
#include "../../include/fireq_norm.h"
#include "../../include/fireq_norm_block.h"
#include "../../include/fireq_paged.h"
#include "../../include/fireq_sample.h"
#include "../../include/fireq_wquant_ws.h"

namespace {

struct Api {
    decltype(&fq_quantize_act) quantize_act;
    decltype(&fq_quantize_act_ws) quantize_act_ws;
    decltype(&fq_packed_weight_bytes) packed_weight_bytes;
    decltype(&fq_w4a8_gemm_workspace_bytes) gemm_workspace_bytes;
    decltype(&fq_w4a8_gemm_ws) gemm_ws;
    decltype(&fq_w4a8_gemm_swiglu_ws) gemm_swiglu_ws;
    decltype(&fq_w4a8_gemm_add_ws) gemm_add_ws;
    decltype(&fq_w4a8_gemm_swiglu_quant_ws) gemm_swiglu_quant_ws;
    decltype(&fq_w4a8_linear_workspace_bytes) linear_workspace_bytes;
    decltype(&fq_w4a8_linear_ws) linear_ws;
    decltype(&fq_kv4_packed_bytes) kv4_packed_bytes;
    decltype(&fq_kv4_scores) kv4_scores;
    decltype(&fq_kv4_output_workspace_bytes) kv4_output_workspace_bytes;
    decltype(&fq_kv4_output_ws) kv4_output_ws;
    decltype(&fq_kv4_pack) kv4_pack;
    decltype(&fq_pack_weights) pack_weights;
    decltype(&fq_cas_scales_workspace_bytes) cas_scales_workspace_bytes;
    decltype(&fq_cas_scales_ws) cas_scales_ws;
    decltype(&fq_pts_exponent_workspace_bytes) pts_exponent_workspace_bytes;
    decltype(&fq_pts_exponent_ws) pts_exponent_ws;
    decltype(&fq_quantize_weights) quantize_weights;
    decltype(&fq_rmsnorm) rmsnorm;
    decltype(&fq_rmsnorm_quant_ws) rmsnorm_quant_ws;
    decltype(&fq_kv4_append) kv4_append;
    decltype(&fq_kv4_read) kv4_read;
    decltype(&fq_kv4_attention_workspace_bytes) attention_workspace_bytes;
    decltype(&fq_kv4_attention_ws) attention_ws;
    decltype(&fq_kv4_attention_prefix_ws) attention_prefix_ws;
    decltype(&fq_rmsnorm_block) rmsnorm_block;
    decltype(&fq_rmsnorm_block_quant_ws) rmsnorm_block_quant_ws;
    decltype(&fq_kv4_append_axes) kv4_append_axes;
    decltype(&fq_kv4_attention_chunk_workspace_bytes) chunk_workspace_bytes;
    decltype(&fq_kv4_attention_chunk_ws) attention_chunk_ws;
    decltype(&fq_sample_workspace_bytes) sample_workspace_bytes;
    decltype(&fq_sample_bf16_ws) sample_bf16_ws;
    decltype(&fq_sample_fp32_ws) sample_fp32_ws;
};
Api api = {};
bool bound = false;

constexpr int64_t GROUP = 128;
constexpr int64_t INT_LIMIT = 0x7FFFFFFF;

struct Decline {};                                        // "not for this path": None to the caller
void want(bool ok) { if (!ok) throw Decline(); }

const at::Tensor& tensor(PyObject* o) {
    want(THPVariable_CheckExact(o));
    return THPVariable_Unpack(o);
}

const at::Tensor& dev(PyObject* o, at::ScalarType t) {
    const at::Tensor& x = tensor(o);
    want(x.is_cuda() && x.scalar_type() == t && x.is_contiguous());
    return x;
}

int whole(PyObject* o) {
    want(PyLong_CheckExact(o));
    const long v = PyLong_AsLong(o);
    want(v >= 0 && v <= INT_LIMIT);                       // (an overflow answers -1 and leaves an exception, cleared below)
    return (int)v;
}

float number(PyObject* o) {
    if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
    return (float)whole(o);
}

bool truth(PyObject* o) {
    want(o == Py_True || o == Py_False);
    return o == Py_True;
}

// A tensor as torch.empty gives it, through the dispatcher: modes, transforms, profilers, the filling of fresh memory and kernels that a
// program has registered for it see every output (straight from the allocator 0.25 us less per tensor, and the last of these would not)
at::Tensor fresh(at::IntArrayRef size, at::ScalarType t, const at::Tensor& like) {
    return at::empty(size, at::TensorOptions().dtype(t).device(like.device()));
}

// the caller's scratch, or one of `need` bytes from the (stream-ordered) allocator, or none
struct Scratch {
    at::Tensor own;
    void* p = nullptr;
    size_t bytes = 0;
    Scratch(PyObject* o, size_t need, const at::Tensor& like) {
        if (o != Py_None) {
            const at::Tensor& t = tensor(o);
            p = t.data_ptr();
            bytes = (size_t)t.numel() * t.element_size();
        } else if (need > 0) {
            own = fresh({(int64_t)need}, at::kByte, like);
            p = own.data_ptr();
            bytes = need;
        }
    }
};

at::Tensor output(PyObject* o, at::IntArrayRef size, const at::Tensor& like) {
    if (o == Py_None) return fresh(size, at::kBFloat16, like);
    const at::Tensor& t = dev(o, at::kBFloat16);
    want(t.sizes() == size);
    return t;
}

void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }

template <class F>
int call(F f) {                                           // other threads run meanwhile, as they do under ctypes
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

template <class F>
PyObject* guarded(F f) {
    try {
        want(bound && at::impl::PythonTorchFunctionTLS::stack_len() == 0);
        return f();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* wrap(int rc, const at::Tensor& t) { return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(t); }

PyObject* wrap(int rc, std::initializer_list<at::Tensor> ts) {
    if (rc) return PyLong_FromLong(rc);
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));
    return r;
}

struct Gemm {                                             // operands shared by the GEMM calls
    const at::Tensor &A, &a_scale, &W, &gs;
    float ts;
    int M, N, K;
    Gemm(PyObject* const* a) : A(dev(a[0], at::kByte)), a_scale(dev(a[1], at::kFloat)), W(dev(a[2], at::kByte)), gs(dev(a[3], at::kByte)),
                               ts(number(a[4])), N(whole(a[5])) {
        want(A.dim() == 2 && A.size(0) <= INT_LIMIT && A.size(1) <= INT_LIMIT);
        M = (int)A.size(0);
        K = (int)A.size(1);
        want(M > 0 && N > 0 && K > 0 && K % GROUP == 0 && a_scale.numel() == M && gs.numel() == (int64_t)N * (K / GROUP) &&
             (size_t)W.numel() >= api.packed_weight_bytes(N, K));
    }
    const uint8_t* a() const { return (const uint8_t*)A.data_ptr(); }
    const float* s() const { return (const float*)a_scale.data_ptr(); }
    const uint8_t* w() const { return (const uint8_t*)W.data_ptr(); }
    const uint8_t* g() const { return (const uint8_t*)gs.data_ptr(); }
};

// quantize_act(X, workspace)
PyObject* quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 2);
        const at::Tensor& X = dev(a[0], at::kBFloat16);
        want(X.dim() == 2 && X.size(0) > 0 && X.size(1) > 0 && X.size(0) <= INT_LIMIT && X.size(1) <= INT_LIMIT);
        const int M = (int)X.size(0), K = (int)X.size(1);
        at::Tensor A = fresh({M, K}, at::kByte, X), s = fresh({M}, at::kFloat, X);
        const Scratch ws(a[1], 0, X);
        const uint16_t* x = (const uint16_t*)X.data_ptr();
        uint8_t* pa = (uint8_t*)A.data_ptr();
        float* ps = (float*)s.data_ptr();
        void* st = stream();
        const bool with = a[1] != Py_None;
        const int rc = call([&] { return with ? api.quantize_act_ws(x, pa, ps, M, K, ws.p, ws.bytes, st) : api.quantize_act(x, pa, ps, M, K, st); });
        return wrap(rc, {A, s});
    });
}

// gemm(A, a_scale, W, gs, ts, N, out, workspace, prepared), swiglu(the same), add(the same with the residual at the end)
enum class Mode { Plain, Swiglu, Add };
template <Mode MODE>
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == (MODE == Mode::Add ? 10 : 9));
        const Gemm o(a);
        want(MODE != Mode::Swiglu || o.N % 2 == 0);
        const at::Tensor Y = output(a[6], {o.M, MODE == Mode::Swiglu ? o.N / 2 : o.N}, o.A);
        const uint16_t* r = nullptr;
        if (MODE == Mode::Add) {
            const at::Tensor& R = dev(a[9], at::kBFloat16);
            want(R.dim() == 2 && R.size(0) == o.M && R.size(1) == o.N);
            r = (const uint16_t*)R.data_ptr();
        }
        const Scratch ws(a[7], api.gemm_workspace_bytes(o.M, o.N, o.K), o.A);
        const int prepared = truth(a[8]) && a[7] != Py_None ? 1 : 0;
        uint16_t* y = (uint16_t*)Y.data_ptr();
        const uint8_t *pa = o.a(), *pw = o.w(), *pg = o.g();
        const float* ps = o.s();
        void* st = stream();
        const int rc = call([&] {
            return MODE == Mode::Plain ? api.gemm_ws(pa, ps, pw, pg, o.ts, y, o.M, o.N, o.K, ws.p, ws.bytes, prepared, st)
                 : MODE == Mode::Swiglu ? api.gemm_swiglu_ws(pa, ps, pw, pg, o.ts, y, o.M, o.N, o.K, ws.p, ws.bytes, prepared, st)
                                        : api.gemm_add_ws(pa, ps, pw, pg, o.ts, r, y, o.M, o.N, o.K, ws.p, ws.bytes, prepared, st);
        });
        return wrap(rc, Y);
    });
}

// swiglu_quant(A, a_scale, W, gs, ts, N, out, workspace, prepared, next_workspace)
PyObject* swiglu_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 10);
        const Gemm o(a);
        want(o.N % 2 == 0);
        const int NH = o.N / 2;
        const at::Tensor H = output(a[6], {o.M, NH}, o.A);
        at::Tensor codes = fresh({o.M, NH}, at::kByte, o.A), scales = fresh({o.M}, at::kFloat, o.A);
        const Scratch ws(a[7], api.gemm_workspace_bytes(o.M, o.N, o.K), o.A), next(a[9], 0, o.A);
        const int prepared = truth(a[8]) && a[7] != Py_None ? 1 : 0;
        uint16_t* h = (uint16_t*)H.data_ptr();
        uint8_t* pc = (uint8_t*)codes.data_ptr();
        float* psc = (float*)scales.data_ptr();
        const uint8_t *pa = o.a(), *pw = o.w(), *pg = o.g();
        const float* ps = o.s();
        void* st = stream();
        const int rc = call([&] {
            return api.gemm_swiglu_quant_ws(pa, ps, pw, pg, o.ts, h, pc, psc, o.M, o.N, o.K, ws.p, ws.bytes, prepared, next.p, next.bytes, st);
        });
        return wrap(rc, {H, codes, scales});
    });
}

// linear(X, W, gs, ts, N, out, workspace)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 7);
        const at::Tensor &X = dev(a[0], at::kBFloat16), &W = dev(a[1], at::kByte), &G = dev(a[2], at::kByte);
        const float ts = number(a[3]);
        const int N = whole(a[4]);
        want(X.dim() == 2 && X.size(0) <= INT_LIMIT && X.size(1) <= INT_LIMIT);
        const int M = (int)X.size(0), K = (int)X.size(1);
        want(M > 0 && N > 0 && K > 0 && K % GROUP == 0 && G.numel() == (int64_t)N * (K / GROUP) &&
             (size_t)W.numel() >= api.packed_weight_bytes(N, K));
        const at::Tensor Y = output(a[5], {M, N}, X);
        const Scratch ws(a[6], a[6] == Py_None ? api.linear_workspace_bytes(M, N, K) : 0, X);
        const uint16_t* x = (const uint16_t*)X.data_ptr();
        const uint8_t *w = (const uint8_t*)W.data_ptr(), *g = (const uint8_t*)G.data_ptr();
        uint16_t* y = (uint16_t*)Y.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.linear_ws(x, w, g, ts, y, M, N, K, ws.p, ws.bytes, st); });
        return wrap(rc, Y);
    });
}

// kv4_scores(Q, q_scale, K_packed, k_scale, out_scale)
PyObject* kv4_scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 5);
        const at::Tensor &Q = dev(a[0], at::kByte), &qs = dev(a[1], at::kFloat), &kp = dev(a[2], at::kByte), &ks = dev(a[3], at::kByte);
        const float scale = number(a[4]);
        want(Q.dim() == 3 && qs.dim() == 2 && ks.dim() == 2);
        const int64_t h = Q.size(0), r = Q.size(1), t = ks.size(1);
        want(h > 0 && r > 0 && t > 0 && h <= INT_LIMIT && r <= INT_LIMIT && t <= INT_LIMIT && Q.size(2) == GROUP && qs.size(0) == h &&
             qs.size(1) == r && ks.size(0) == h);
        const int H = (int)h, R = (int)r, T = (int)t;
        want((size_t)kp.numel() >= api.kv4_packed_bytes(H, T, 0));
        at::Tensor S = fresh({h, r, t}, at::kBFloat16, Q);
        const uint8_t *q = (const uint8_t*)Q.data_ptr(), *k = (const uint8_t*)kp.data_ptr(), *s = (const uint8_t*)ks.data_ptr();
        const float* f = (const float*)qs.data_ptr();
        uint16_t* o = (uint16_t*)S.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.kv4_scores(q, f, k, s, scale, o, H, R, T, st); });
        return wrap(rc, S);
    });
}

// kv4_output(P, p_scale, V_packed, v_scale)
PyObject* kv4_output(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 4);
        const at::Tensor &P = dev(a[0], at::kByte), &ps = dev(a[1], at::kFloat), &vp = dev(a[2], at::kByte), &vs = dev(a[3], at::kByte);
        want(P.dim() == 3 && ps.dim() == 2 && vs.dim() == 2);
        const int64_t h = P.size(0), r = P.size(1), l = P.size(2), t = vs.size(1);
        want(h > 0 && r > 0 && t > 0 && h <= INT_LIMIT && r <= INT_LIMIT && l <= INT_LIMIT && l >= t && ps.size(0) == h && ps.size(1) == r &&
             vs.size(0) == h);
        const int H = (int)h, R = (int)r, T = (int)t, ldp = (int)l;
        want((size_t)vp.numel() >= api.kv4_packed_bytes(H, T, 1));
        at::Tensor O = fresh({h, r, GROUP}, at::kBFloat16, P);
        const Scratch ws(Py_None, api.kv4_output_workspace_bytes(H, R, T), P);
        const uint8_t *p = (const uint8_t*)P.data_ptr(), *v = (const uint8_t*)vp.data_ptr(), *s = (const uint8_t*)vs.data_ptr();
        const float* f = (const float*)ps.data_ptr();
        uint16_t* o = (uint16_t*)O.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.kv4_output_ws(p, f, v, s, o, H, R, T, ldp, ws.p, ws.bytes, st); });
        return wrap(rc, O);
    });
}

// kv4_pack(codes, values)
PyObject* kv4_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 2);
        const at::Tensor& C = dev(a[0], at::kChar);
        const int values = truth(a[1]) ? 1 : 0;
        want(C.dim() == 3 && C.size(0) > 0 && C.size(1) > 0 && C.size(0) <= INT_LIMIT && C.size(1) <= INT_LIMIT && C.size(2) == GROUP);
        const int H = (int)C.size(0), T = (int)C.size(1);
        at::Tensor out = fresh({(int64_t)api.kv4_packed_bytes(H, T, values)}, at::kByte, C);
        const int8_t* c = (const int8_t*)C.data_ptr();
        uint8_t* o = (uint8_t*)out.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.kv4_pack(c, o, H, T, values, st); });
        return wrap(rc, out);
    });
}

struct Matrix {                                           // a weight matrix [N,K] of the offline calls
    const at::Tensor& W;
    int N, K;
    Matrix(PyObject* o, at::ScalarType t) : W(dev(o, t)) {
        want(W.dim() == 2 && W.size(0) > 0 && W.size(1) > 0 && W.size(0) <= INT_LIMIT && W.size(1) <= INT_LIMIT);
        N = (int)W.size(0);
        K = (int)W.size(1);
    }
    const uint16_t* w() const { return (const uint16_t*)W.data_ptr(); }
    const float* lambda(PyObject* o) const {              // the channels' scales, or none
        if (o == Py_None) return nullptr;
        const at::Tensor& l = dev(o, at::kFloat);
        want(l.numel() == K);
        return (const float*)l.data_ptr();
    }
};

// pack_weights(q)
PyObject* pack_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 1);
        const Matrix m(a[0], at::kChar);
        const size_t bytes = api.packed_weight_bytes(m.N, m.K);
        want(bytes > 0);
        at::Tensor out = fresh({(int64_t)bytes}, at::kByte, m.W);
        const int8_t* q = (const int8_t*)m.W.data_ptr();
        uint8_t* o = (uint8_t*)out.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.pack_weights(q, o, m.N, m.K, st); });
        return wrap(rc, out);
    });
}

// cas_scales(W, target)
PyObject* cas_scales(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 2);
        const Matrix m(a[0], at::kBFloat16);
        const float target = number(a[1]);
        at::Tensor out = fresh({m.K}, at::kFloat, m.W);
        const Scratch ws(Py_None, api.cas_scales_workspace_bytes(m.N, m.K), m.W);
        const uint16_t* w = m.w();
        float* o = (float*)out.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.cas_scales_ws(w, target, o, m.N, m.K, ws.p, ws.bytes, st); });
        return wrap(rc, out);
    });
}

// pts_exponent(W, lam)
PyObject* pts_exponent(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 2);
        const Matrix m(a[0], at::kBFloat16);
        const float* lam = m.lambda(a[1]);
        at::Tensor out = fresh({16}, at::kInt, m.W);
        const Scratch ws(Py_None, api.pts_exponent_workspace_bytes(m.N, m.K), m.W);
        const uint16_t* w = m.w();
        int* o = (int*)out.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.pts_exponent_ws(w, lam, o, m.N, m.K, ws.p, ws.bytes, st); });
        return wrap(rc, out);
    });
}

// quantize_weights(W, lam, n_pts, sigma_nearest)
PyObject* quantize_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 4);
        const Matrix m(a[0], at::kBFloat16);
        const float* lam = m.lambda(a[1]);
        const int n_pts = whole(a[2]), nearest = truth(a[3]) ? 1 : 0;
        want(m.K % GROUP == 0);
        at::Tensor q = fresh({m.N, m.K}, at::kChar, m.W), gs = fresh({m.N, m.K / GROUP}, at::kByte, m.W);
        const uint16_t* w = m.w();
        int8_t* pq = (int8_t*)q.data_ptr();
        uint8_t* pg = (uint8_t*)gs.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.quantize_weights(w, lam, n_pts, nearest, pq, pg, m.N, m.K, st); });
        return wrap(rc, {q, gs});
    });
}

// a workspace that the Python form does not refuse
void scratch_or_none(PyObject* o) {
    if (o != Py_None) {
        const at::Tensor& t = tensor(o);
        want(t.is_cuda() && t.is_contiguous());
    }
}

// rmsnorm(X, weight, eps, residual, out), rmsnorm_quant(X, weight, eps, residual, out, workspace)
template <bool QUANT>
PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == (QUANT ? 6 : 5));
        const at::Tensor &X = dev(a[0], at::kBFloat16), &w = dev(a[1], at::kBFloat16);
        want(X.dim() == 2 && X.size(0) > 0 && X.size(0) <= INT_LIMIT && X.size(1) > 0 && X.size(1) <= INT_LIMIT && w.numel() == X.size(1));
        const float eps = number(a[2]);
        const int M = (int)X.size(0), K = (int)X.size(1);
        at::Tensor H;
        const uint16_t* r = nullptr;
        if (a[3] != Py_None) {
            const at::Tensor& R = dev(a[3], at::kBFloat16);
            want(R.sizes() == X.sizes());
            r = (const uint16_t*)R.data_ptr();
            H = output(a[4], X.sizes(), X);
        } else {
            want(a[4] == Py_None);
        }
        const uint16_t *x = (const uint16_t*)X.data_ptr(), *pw = (const uint16_t*)w.data_ptr();
        uint16_t* h = r ? (uint16_t*)H.data_ptr() : nullptr;
        void* st = stream();
        if (!QUANT) {
            at::Tensor Y = fresh({M, K}, at::kBFloat16, X);
            uint16_t* y = (uint16_t*)Y.data_ptr();
            const int rc = call([&] { return api.rmsnorm(x, r, pw, eps, h, y, M, K, st); });
            return r ? wrap(rc, {Y, H}) : wrap(rc, Y);
        }
        at::Tensor A = fresh({M, K}, at::kByte, X), s = fresh({M}, at::kFloat, X);
        scratch_or_none(a[QUANT ? 5 : 0]);
        const Scratch ws(a[QUANT ? 5 : 0], 0, X);
        uint8_t* pa = (uint8_t*)A.data_ptr();
        float* ps = (float*)s.data_ptr();
        const bool with = a[QUANT ? 5 : 0] != Py_None;
        const int rc = call([&] { return api.rmsnorm_quant_ws(x, r, pw, eps, h, pa, ps, M, K, with ? ws.p : nullptr, with ? ws.bytes : 0, st); });
        return r ? wrap(rc, {A, s, H}) : wrap(rc, {A, s});
    });
}

struct Paged {                                            // a paged cache [pages, heads, page / 16, 2080], its pages contiguous
    const at::Tensor& c;
    int pages, heads, page;
    int64_t page_stride, head_stride;
    explicit Paged(PyObject* o) : c(tensor(o)) {
        want(c.is_cuda() && c.scalar_type() == at::kByte && c.dim() == 4 && c.size(3) == FQ_KV4_TILE_BYTES && c.stride(3) == 1 && c.size(2) > 0 &&
             (c.size(2) == 1 || c.stride(2) == FQ_KV4_TILE_BYTES));
        want(c.size(0) > 0 && c.size(0) <= INT_LIMIT && c.size(1) > 0 && c.size(1) <= INT_LIMIT && c.size(2) <= INT_LIMIT / FQ_KV4_TILE_TOKENS);
        pages = (int)c.size(0);
        heads = (int)c.size(1);
        page = (int)c.size(2) * FQ_KV4_TILE_TOKENS;
        head_stride = heads > 1 ? c.stride(1) : c.size(2) * FQ_KV4_TILE_BYTES;
        page_stride = pages > 1 ? c.stride(0) : heads * head_stride;
    }
    uint8_t* p() const { return (uint8_t*)c.data_ptr(); }
};

// kv4_append(QKV, cos_sin, positions, slots, cache, interleaved)
PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 6);
        const at::Tensor &X = tensor(a[0]), &rot = dev(a[1], at::kFloat), &pos = dev(a[2], at::kInt), &slots = dev(a[3], at::kLong);
        want(X.is_cuda() && X.scalar_type() == at::kBFloat16 && X.dim() == 2 && X.stride(1) == 1);
        const Paged c(a[4]);
        const int interleaved = truth(a[5]) ? 1 : 0;
        const int64_t T = X.size(0), width = X.size(1), Hq = width / 128 - 2 * (int64_t)c.heads, ld = T > 1 ? X.stride(0) : width;
        want(T > 0 && T <= INT_LIMIT && width % 128 == 0 && Hq > 0 && Hq <= INT_LIMIT && ld >= width && pos.numel() == T && slots.numel() == T &&
             rot.dim() == 3 && rot.size(0) <= INT_LIMIT && rot.size(1) == 64 && rot.size(2) == 2);
        at::Tensor Q = fresh({T, Hq, 128}, at::kByte, X), s = fresh({T, Hq}, at::kFloat, X);
        const uint16_t* x = (const uint16_t*)X.data_ptr();
        const float* cs = (const float*)rot.data_ptr();
        const int32_t* pp = (const int32_t*)pos.data_ptr();
        const int64_t* sl = (const int64_t*)slots.data_ptr();
        uint8_t* q = (uint8_t*)Q.data_ptr();
        float* qs = (float*)s.data_ptr();
        const int positions = (int)rot.size(0);
        void* st = stream();
        const int rc = call([&] {
            return api.kv4_append(x, ld, cs, positions, pp, sl, interleaved, q, qs, c.p(), c.page_stride, c.head_stride, c.pages, c.page, (int)T, (int)Hq, c.heads, st);
        });
        return wrap(rc, {Q, s});
    });
}

// kv4_read(cache, slots)
PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 2);
        const Paged c(a[0]);
        const at::Tensor& slots = dev(a[1], at::kLong);
        const int64_t count = slots.numel();
        want(count > 0 && count <= INT_LIMIT);
        at::Tensor K = fresh({count, c.heads, 128}, at::kBFloat16, c.c), V = fresh({count, c.heads, 128}, at::kBFloat16, c.c);
        const int64_t* sl = (const int64_t*)slots.data_ptr();
        uint16_t *k = (uint16_t*)K.data_ptr(), *v = (uint16_t*)V.data_ptr();
        void* st = stream();
        const int rc = call([&] { return api.kv4_read(c.p(), c.page_stride, c.head_stride, c.pages, c.page, sl, k, v, (int)count, c.heads, st); });
        return wrap(rc, {K, V});
    });
}

// kv4_attention(Q, q_scale, cache, prefix_pages, prefix_len, block_table, seq_lens, out_scale, max_len, out, workspace)
PyObject* kv4_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 11);
        const at::Tensor &Q = dev(a[0], at::kByte), &qs = dev(a[1], at::kFloat);
        const Paged c(a[2]);
        const at::Tensor &table = dev(a[5], at::kInt), &lens = dev(a[6], at::kInt);
        want(Q.dim() == 3 && Q.size(2) == 128 && table.dim() == 2);
        const int64_t B = Q.size(0), Hq = Q.size(1), width = table.size(1);
        want(B > 0 && B <= INT_LIMIT && Hq > 0 && Hq <= INT_LIMIT && Hq % c.heads == 0 && width <= INT_LIMIT && qs.numel() == B * Hq && table.size(0) == B &&
             lens.numel() == B);
        const float out_scale = number(a[7]);
        const int64_t most = std::min<int64_t>(width * c.page, 1 << 30);
        const int max_len = a[8] == Py_None ? (int)most : whole(a[8]);
        const int32_t* shared = nullptr;
        int prefix = 0;
        const bool with = a[3] != Py_None;
        if (with) {
            const at::Tensor& p = dev(a[3], at::kInt);
            prefix = whole(a[4]);
            want(p.numel() * c.page >= prefix);
            shared = (const int32_t*)p.data_ptr();
        }
        at::Tensor O;
        if (a[9] == Py_None) {
            O = fresh({B, Hq, 128}, at::kBFloat16, Q);
        } else {
            O = dev(a[9], at::kBFloat16);
            want(O.sizes() == at::IntArrayRef({B, Hq, 128}) || O.sizes() == at::IntArrayRef({B, Hq * 128}));
        }
        scratch_or_none(a[10]);
        const Scratch ws(a[10], a[10] == Py_None ? api.attention_workspace_bytes((int)B, (int)Hq, c.heads, max_len, prefix) : 0, Q);
        const uint8_t* q = (const uint8_t*)Q.data_ptr();
        const float* s = (const float*)qs.data_ptr();
        const int32_t *tb = (const int32_t*)table.data_ptr(), *ln = (const int32_t*)lens.data_ptr();
        uint16_t* o = (uint16_t*)O.data_ptr();
        void* st = stream();
        const int rc = call([&] {
            return with ? api.attention_prefix_ws(q, s, c.p(), c.page_stride, c.head_stride, c.pages, c.page, shared, prefix, tb, (int)width, ln, out_scale, o,
                                                  (int)B, (int)Hq, c.heads, max_len, ws.p, ws.bytes, st)
                        : api.attention_ws(q, s, c.p(), c.page_stride, c.head_stride, c.pages, c.page, tb, (int)width, ln, out_scale, o, (int)B, (int)Hq,
                                           c.heads, max_len, ws.p, ws.bytes, st);
        });
        return wrap(rc, O);
    });
}

// A tensor on the device whose stream the call takes, of a type and `n` numbers (below 0: any number); none where None is given.
const at::Tensor& here(PyObject* o, at::ScalarType t, int64_t n) {
    const at::Tensor& x = dev(o, t);
    want(x.device().index() == c10::hip::current_device() && (n < 0 || x.numel() == n));
    return x;
}
template <class T>
const T* maybe(PyObject* o, at::ScalarType t, int64_t n) { return o == Py_None ? nullptr : (const T*)here(o, t, n).data_ptr(); }

void scratch_here(PyObject* o) {
    scratch_or_none(o);
    if (o != Py_None) want(tensor(o).device().index() == c10::hip::current_device());
}

// rmsnorm_block(X, weight, eps, residual, post, gate, gate_rows, scale, out), rmsnorm_block_quant(.., workspace)
template <bool QUANT>
PyObject* rmsnorm_block(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == (QUANT ? 10 : 9));
        const at::Tensor& X = here(a[0], at::kBFloat16, -1);
        want(X.dim() == 2 && X.size(0) > 0 && X.size(0) <= INT_LIMIT && X.size(1) > 0 && X.size(1) <= INT_LIMIT);
        const int M = (int)X.size(0), K = (int)X.size(1);
        const uint16_t* w = (const uint16_t*)here(a[1], at::kBFloat16, K).data_ptr();
        const float eps = number(a[2]), scale = number(a[7]);
        const at::Tensor& R = here(a[3], at::kBFloat16, -1);
        want(R.sizes() == X.sizes());
        const uint16_t *post = maybe<uint16_t>(a[4], at::kBFloat16, K), *gate = maybe<uint16_t>(a[5], at::kBFloat16, -1);
        int gates = 1;
        if (a[5] != Py_None) {                                // (the data of an empty tensor are NULL)
            const at::Tensor& g = tensor(a[5]);
            want(g.dim() == 2 ? g.size(1) == K && g.size(0) >= 1 && g.size(0) <= INT_LIMIT : g.numel() == K);
            gates = g.dim() == 2 ? (int)g.size(0) : 1;
        }
        want(gate || a[6] == Py_None);
        const int32_t* rows = maybe<int32_t>(a[6], at::kInt, M);
        if (a[8] != Py_None) here(a[8], at::kBFloat16, -1);
        at::Tensor H = output(a[8], X.sizes(), X);
        const uint16_t *x = (const uint16_t*)X.data_ptr(), *r = (const uint16_t*)R.data_ptr();
        uint16_t* h = (uint16_t*)H.data_ptr();
        void* st = stream();
        if (!QUANT) {
            at::Tensor Y = fresh({M, K}, at::kBFloat16, X);
            uint16_t* y = (uint16_t*)Y.data_ptr();
            const int rc = call([&] { return api.rmsnorm_block(x, post, gate, rows, gates, scale, r, w, eps, h, y, M, K, st); });
            return wrap(rc, {Y, H});
        }
        at::Tensor A = fresh({M, K}, at::kByte, X), s = fresh({M}, at::kFloat, X);
        PyObject* const o = a[QUANT ? 9 : 0];
        scratch_here(o);
        const Scratch ws(o, 0, X);
        uint8_t* pa = (uint8_t*)A.data_ptr();
        float* ps = (float*)s.data_ptr();
        const int rc = call([&] { return api.rmsnorm_block_quant_ws(x, post, gate, rows, gates, scale, r, w, eps, h, pa, ps, M, K, ws.p, ws.bytes, st); });
        return wrap(rc, {A, s, H});
    });
}

// kv4_append_axes(QKV, cos_sin, positions, axis_of_pair, slots, cache, interleaved)
PyObject* kv4_append_axes(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 7);
        const at::Tensor &X = tensor(a[0]), &rot = here(a[1], at::kFloat, -1), &pos = here(a[2], at::kInt, -1), &slots = here(a[4], at::kLong, -1);
        want(X.is_cuda() && X.device() == rot.device() && X.scalar_type() == at::kBFloat16 && X.dim() == 2 && X.stride(1) == 1);
        int8_t axis[64];
        const bool list = PyList_CheckExact(a[3]);
        want((list || PyTuple_CheckExact(a[3])) && (list ? PyList_GET_SIZE(a[3]) : PyTuple_GET_SIZE(a[3])) == 64 && pos.dim() == 2 && pos.size(0) >= 1 &&
             pos.size(0) <= 127);
        for (int j = 0; j < 64; ++j) {
            PyObject* const v = list ? PyList_GET_ITEM(a[3], j) : PyTuple_GET_ITEM(a[3], j);
            want(PyLong_CheckExact(v));
            const long x = PyLong_AsLong(v);              // (an overflow answers -1 and leaves an exception)
            want(x >= -1 && x < pos.size(0) && !(x == -1 && PyErr_Occurred()));
            axis[j] = (int8_t)x;
        }
        const Paged c(a[5]);
        want(c.c.device() == rot.device());
        const int interleaved = truth(a[6]) ? 1 : 0;
        const int64_t T = X.size(0), width = X.size(1), Hq = width / 128 - 2 * (int64_t)c.heads, ld = T > 1 ? X.stride(0) : width;
        want(T > 0 && T <= INT_LIMIT && width % 128 == 0 && Hq > 0 && Hq <= INT_LIMIT && ld >= width && pos.size(1) == T && slots.numel() == T &&
             rot.dim() == 3 && rot.size(0) <= INT_LIMIT && rot.size(1) == 64 && rot.size(2) == 2);
        at::Tensor Q = fresh({T, Hq, 128}, at::kByte, X), s = fresh({T, Hq}, at::kFloat, X);
        const uint16_t* x = (const uint16_t*)X.data_ptr();
        const float* cs = (const float*)rot.data_ptr();
        const int32_t* pp = (const int32_t*)pos.data_ptr();
        const int64_t* sl = (const int64_t*)slots.data_ptr();
        uint8_t* q = (uint8_t*)Q.data_ptr();
        float* qs = (float*)s.data_ptr();
        const int positions = (int)rot.size(0), axes = (int)pos.size(0);
        void* st = stream();
        const int rc = call([&] {
            return api.kv4_append_axes(x, ld, cs, positions, pp, axes, axis, sl, interleaved, q, qs, c.p(), c.page_stride, c.head_stride, c.pages, c.page,
                                       (int)T, (int)Hq, c.heads, st);
        });
        return wrap(rc, {Q, s});
    });
}

// kv4_attention_chunk(Q, q_scale, cache, block_table, starts, seq_lens, out_scale, max_new, max_len, first, end, window, cap, slopes, out, workspace)
PyObject* kv4_attention_chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 16);
        const at::Tensor& Q = here(a[0], at::kByte, -1);
        const Paged c(a[2]);
        const at::Tensor& table = here(a[3], at::kInt, -1);
        want(c.c.device() == Q.device() && Q.dim() == 3 && Q.size(2) == 128 && table.dim() == 2);
        const int64_t T = Q.size(0), Hq = Q.size(1), B = table.size(0), width = table.size(1);
        want(T > 0 && T <= INT_LIMIT && B > 0 && B < INT_LIMIT && Hq > 0 && Hq <= INT_LIMIT && Hq % c.heads == 0 && width <= INT_LIMIT);
        const float* s = (const float*)here(a[1], at::kFloat, T * Hq).data_ptr();
        const int32_t *starts = (const int32_t*)here(a[4], at::kInt, B + 1).data_ptr(), *lens = (const int32_t*)here(a[5], at::kInt, B).data_ptr();
        const float out_scale = number(a[6]), cap = number(a[12]);
        const int max_new = a[7] == Py_None ? (T <= B ? 1 : (int)T) : whole(a[7]), max_len = a[8] == Py_None ? (int)std::min<int64_t>(width * c.page, 1 << 30) : whole(a[8]);
        const int window = whole(a[11]);
        const int32_t *first = maybe<int32_t>(a[9], at::kInt, T), *end = maybe<int32_t>(a[10], at::kInt, T);
        const float* slopes = maybe<float>(a[13], at::kFloat, Hq);
        at::Tensor O;
        if (a[14] == Py_None) {
            O = fresh({T, Hq, 128}, at::kBFloat16, Q);
        } else {
            O = here(a[14], at::kBFloat16, -1);
            want(O.sizes() == at::IntArrayRef({T, Hq, 128}) || O.sizes() == at::IntArrayRef({T, Hq * 128}));
        }
        scratch_here(a[15]);
        const Scratch ws(a[15], a[15] == Py_None ? api.chunk_workspace_bytes((int)T, (int)B, (int)Hq, c.heads, max_new, max_len) : 0, Q);
        const uint8_t* q = (const uint8_t*)Q.data_ptr();
        const int32_t* tb = (const int32_t*)table.data_ptr();
        uint16_t* o = (uint16_t*)O.data_ptr();
        void* st = stream();
        const int rc = call([&] {
            return api.attention_chunk_ws(q, s, c.p(), c.page_stride, c.head_stride, c.pages, c.page, tb, (int)width, starts, lens, first, end, window, cap, slopes,
                                          out_scale, o, (int)T, (int)B, (int)Hq, c.heads, max_new, max_len, ws.p, ws.bytes, st);
        });
        return wrap(rc, O);
    });
}

// sample(logits, u, temperature, top_k, top_p, min_p, workspace)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 7);
        const at::Tensor& X = tensor(a[0]);
        want(X.is_cuda() && X.device().index() == c10::hip::current_device() && X.dim() == 2 && (X.scalar_type() == at::kBFloat16 || X.scalar_type() == at::kFloat));
        const int64_t B = X.size(0), V = X.size(1), ld = B > 1 ? X.stride(0) : V;
        want(B > 0 && B <= INT_LIMIT && V > 0 && V <= INT_LIMIT && (V == 1 || X.stride(1) == 1) && ld >= V);
        const float *u = (const float*)here(a[1], at::kFloat, B).data_ptr(), *T = maybe<float>(a[2], at::kFloat, B), *p = maybe<float>(a[4], at::kFloat, B),
                    *m = maybe<float>(a[5], at::kFloat, B);
        const int32_t* k = maybe<int32_t>(a[3], at::kInt, B);
        scratch_here(a[6]);
        const Scratch ws(a[6], a[6] == Py_None ? api.sample_workspace_bytes((int)B, (int)V) : 0, X);
        at::Tensor token = fresh({B}, at::kInt, X), logprob = fresh({B}, at::kFloat, X);
        int32_t* pt = (int32_t*)token.data_ptr();
        float* pl = (float*)logprob.data_ptr();
        const void* x = X.data_ptr();
        const bool wide = X.scalar_type() == at::kFloat;
        void* st = stream();
        const int rc = call([&] {
            return wide ? api.sample_fp32_ws((const float*)x, ld, u, T, k, p, m, pt, pl, (int)B, (int)V, ws.p, ws.bytes, st)
                        : api.sample_bf16_ws((const uint16_t*)x, ld, u, T, k, p, m, pt, pl, (int)B, (int)V, ws.p, ws.bytes, st);
        });
        return wrap(rc, {token, logprob});
    });
}

// gemm_workspace_bytes(M, N, K)
PyObject* gemm_workspace_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&] {
        want(n == 3);
        return PyLong_FromSize_t(api.gemm_workspace_bytes(whole(a[0]), whole(a[1]), whole(a[2])));
    });
}

// bind(addresses of the C functions, in the order of Api)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr Py_ssize_t COUNT = sizeof(Api) / sizeof(void*);
    if (n != COUNT) {
        PyErr_SetString(PyExc_TypeError, "bind() takes the address of every C function");
        return nullptr;
    }
    void* p[COUNT];
    for (Py_ssize_t i = 0; i < COUNT; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind(): a NULL address");
            return nullptr;
        }
    }
    __builtin_memcpy(&api, p, sizeof(api));
    bound = true;
    Py_RETURN_NONE;
}

#define FQ_METHOD(name, fn) {name, (PyCFunction)(void (*)(void))(fn), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FQ_METHOD("bind", bind),
    FQ_METHOD("quantize_act", quantize_act),
    FQ_METHOD("gemm", gemm<Mode::Plain>),
    FQ_METHOD("gemm_swiglu", gemm<Mode::Swiglu>),
    FQ_METHOD("gemm_add", gemm<Mode::Add>),
    FQ_METHOD("gemm_swiglu_quant", swiglu_quant),
    FQ_METHOD("linear", linear),
    FQ_METHOD("kv4_scores", kv4_scores),
    FQ_METHOD("kv4_output", kv4_output),
    FQ_METHOD("kv4_pack", kv4_pack),
    FQ_METHOD("pack_weights", pack_weights),
    FQ_METHOD("cas_scales", cas_scales),
    FQ_METHOD("pts_exponent", pts_exponent),
    FQ_METHOD("quantize_weights", quantize_weights),
    FQ_METHOD("rmsnorm", rmsnorm<false>),
    FQ_METHOD("rmsnorm_quant", rmsnorm<true>),
    FQ_METHOD("kv4_append", kv4_append),
    FQ_METHOD("kv4_read", kv4_read),
    FQ_METHOD("kv4_attention", kv4_attention),
    FQ_METHOD("rmsnorm_block", rmsnorm_block<false>),
    FQ_METHOD("rmsnorm_block_quant", rmsnorm_block<true>),
    FQ_METHOD("kv4_append_axes", kv4_append_axes),
    FQ_METHOD("kv4_attention_chunk", kv4_attention_chunk),
    FQ_METHOD("sample", sample),
    FQ_METHOD("gemm_workspace_bytes", gemm_workspace_bytes),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fq_marshal", "argument marshalling of the fireq binding", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fq_marshal(void) { return PyModule_Create(&module); }
