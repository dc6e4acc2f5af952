// The calls of lemo.py that a layer makes over and over, marshalled in native code: 0.4 us beside the launch where ctypes and the
// checks in Python take 3 to 4 (three calls of a small binary32 layer: 22 us enqueued from Python, 9.6 so).
//
// Every function takes the arguments of the call of the same name in order and answers None when anything about them is not
// the plain case -- another type, layout, device or size than the checks in lemo.py let through, an output still to be allocated,
// a value that the C ABI refuses -- and has then done nothing: the caller goes the long way, which raises what it always
// raised.  Otherwise the call's return code.  The GIL is released around the call, as ctypes does.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "lemo.h"

namespace {

PyObject *current_device = nullptr, *raw_stream = nullptr;  // Python callables: () -> device, (device) -> stream address

struct NotPlain {};  // go the long way

void need(bool ok) {
    if (!ok) throw NotPlain{};
}

// a tensor of exactly torch's own class, on the GPU, with storage and elements
const at::Tensor& tensor(PyObject* o, int64_t dim) {
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && t.dim() == dim && t.numel() > 0);
    return t;
}
lemo_dtype_t dtype(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return LEMO_F32;
    need(t.scalar_type() == at::kBFloat16);
    return LEMO_BF16;
}
int64_t whole(PyObject* o) {
    need(PyLong_CheckExact(o));
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &over);
    need(!over);
    return v;
}
int32_t whole32(PyObject* o) {
    const int64_t v = whole(o);
    need(v >= INT32_MIN && v <= INT32_MAX);
    return (int32_t)v;
}
int32_t size32(int64_t v) {
    need(v <= INT32_MAX);
    return (int32_t)v;
}
float real(PyObject* o) {
    need(PyFloat_CheckExact(o));
    return (float)PyFloat_AS_DOUBLE(o);
}
// a list of rows, or none
const at::Tensor* index(PyObject* o) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, 1);
    need(t.scalar_type() == at::kInt && t.is_contiguous());
    return &t;
}
const int32_t* rows(const at::Tensor* t) { return t ? static_cast<const int32_t*>(t->data_ptr()) : nullptr; }
const at::Tensor& matrix(PyObject* o) {  // rows contiguous
    const at::Tensor& t = tensor(o, 2);
    need(t.stride(1) == 1);
    return t;
}
const at::Tensor& heads(PyObject* o) {  // [S,H,d], d contiguous
    const at::Tensor& t = tensor(o, 3);
    need(t.stride(2) == 1);
    return t;
}
const void* bias_of(PyObject* o, const at::Tensor& like, int64_t n) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, 1);
    need(t.scalar_type() == like.scalar_type() && t.size(0) == n && t.is_contiguous());
    return t.data_ptr();
}
float* plane(PyObject* o, int64_t h, int64_t s) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, 2);
    need(t.scalar_type() == at::kFloat && t.size(0) == h && t.size(1) == s && t.is_contiguous());
    return static_cast<float*>(t.data_ptr());
}
struct Bytes { void* p; size_t n; };
Bytes workspace(PyObject* o) {
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage());
    return {t.data_ptr(), (size_t)t.numel() * t.element_size()};
}
void* stream() {
    PyObject* dev = PyObject_CallNoArgs(current_device);
    if (!dev) { PyErr_Clear(); throw NotPlain{}; }
    PyObject* s = PyObject_CallOneArg(raw_stream, dev);
    Py_DECREF(dev);
    if (!s) { PyErr_Clear(); throw NotPlain{}; }
    void* p = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) { PyErr_Clear(); throw NotPlain{}; }
    return p;
}
// what the C ABI refuses has had no effect and is left to the long way; a launch that failed is reported
template <typename F> PyObject* call(F f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f();
    Py_END_ALLOW_THREADS;
    if (rc != LEMO_OK && rc != LEMO_ERR_HIP) Py_RETURN_NONE;
    return PyLong_FromLong(rc);
}
// no C++ exception leaves this file: tensors that refuse to tell their address (inside vmap, for instance) throw c10::Error
template <Py_ssize_t N, PyObject* (*F)(PyObject* const*)> PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != N || !raw_stream) Py_RETURN_NONE;
    try {
        return F(a);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* score_segments(PyObject* const* a) {  // Q K L flags scale scores colsum diag workspace
    const at::Tensor &Q = heads(a[0]), &K = heads(a[1]);
    const int64_t S = Q.size(0), H = Q.size(1), d = Q.size(2);
    const lemo_dtype_t dt = dtype(Q);
    need(K.size(0) == S && K.size(2) == d && K.scalar_type() == Q.scalar_type());
    const at::Tensor& scores = tensor(a[5], 1);
    need(scores.scalar_type() == at::kFloat && scores.size(0) == S && scores.is_contiguous());
    float *col = plane(a[6], H, S), *dg = plane(a[7], H, S);
    const Bytes ws = workspace(a[8]);
    const int32_t L = whole32(a[2]), flags = whole32(a[3]), h = size32(H), hkv = size32(K.size(1)), dd = size32(d);
    const float scale = real(a[4]);
    void *q = Q.data_ptr(), *k = K.data_ptr(), *sc = scores.data_ptr(), *st = stream();
    const int64_t q0 = Q.stride(0), q1 = Q.stride(1), k0 = K.stride(0), k1 = K.stride(1);
    return call([=] {
        return lemo_score_segments(q, k, S, h, hkv, dd, dt, q0, q1, k0, k1, scale, L, (uint32_t)flags, (float*)sc, col, dg, ws.p, ws.n, st);
    });
}

PyObject* select_topk(PyObject* const* a) {  // scores L k kept_idx
    const at::Tensor& scores = tensor(a[0], 1);
    const at::Tensor* kept = index(a[3]);
    need(scores.scalar_type() == at::kFloat && scores.is_contiguous() && kept);
    const int64_t S = scores.size(0);
    const int32_t L = whole32(a[1]), k = whole32(a[2]);
    need(kept->numel() == lemo_kept_count(S, L, k));
    void *sc = scores.data_ptr(), *ki = kept->data_ptr(), *st = stream();
    return call([=] { return lemo_select_topk((const float*)sc, S, L, k, (int32_t*)ki, st); });
}

PyObject* kept_attention(PyObject* const* a) {  // Q K V kept_idx flags scale O workspace M
    const at::Tensor &Q = heads(a[0]), &K = heads(a[1]), &V = heads(a[2]), &O = heads(a[6]);
    const at::Tensor* kept = index(a[3]);
    const int64_t S = Q.size(0), H = Q.size(1), d = Q.size(2);
    const lemo_dtype_t dt = dtype(Q);
    need(K.size(0) == S && K.size(2) == d && K.scalar_type() == Q.scalar_type() && V.sizes() == K.sizes() && V.scalar_type() == K.scalar_type());
    const int64_t M = a[8] != Py_None ? whole(a[8]) : kept ? kept->numel() : S;
    need(M > 0 && (!kept || kept->numel() >= M) && O.scalar_type() == Q.scalar_type() && O.size(0) >= M && O.size(1) == H && O.size(2) == d);
    const Bytes ws = workspace(a[7]);
    const int32_t flags = whole32(a[4]), h = size32(H), hkv = size32(K.size(1)), dd = size32(d);
    const float scale = real(a[5]);
    const int32_t* ki = rows(kept);
    void *q = Q.data_ptr(), *k = K.data_ptr(), *v = V.data_ptr(), *o = O.data_ptr(), *st = stream();
    const int64_t q0 = Q.stride(0), q1 = Q.stride(1), k0 = K.stride(0), k1 = K.stride(1), v0 = V.stride(0), v1 = V.stride(1), o0 = O.stride(0), o1 = O.stride(1);
    return call([=] {
        return lemo_kept_attention(q, k, v, S, h, hkv, dd, dt, q0, q1, k0, k1, v0, v1, ki, M, scale, (uint32_t)flags, o, o0, o1, ws.p, ws.n, st);
    });
}

PyObject* gather_gemm(PyObject* const* a) {  // X kept_idx W bias Y M
    const at::Tensor &X = matrix(a[0]), &W = matrix(a[2]), &Y = matrix(a[4]);
    const at::Tensor* kept = index(a[1]);
    const lemo_dtype_t dt = dtype(X);
    const int64_t S = X.size(0), C = X.size(1), N = W.size(0);
    need(W.size(1) == C && W.scalar_type() == X.scalar_type());
    const int64_t M = a[5] != Py_None ? whole(a[5]) : kept ? kept->numel() : S;
    need(M > 0 && (!kept || kept->numel() >= M) && Y.scalar_type() == X.scalar_type() && Y.size(0) >= M && Y.size(1) == N);
    const void* b = bias_of(a[3], X, N);
    const int32_t* ki = rows(kept);
    const int32_t c = size32(C), n = size32(N);
    void *x = X.data_ptr(), *w = W.data_ptr(), *y = Y.data_ptr(), *st = stream();
    const int64_t x0 = X.stride(0), w0 = W.stride(0), y0 = Y.stride(0);
    return call([=] { return lemo_gather_gemm(x, S, x0, ki, M, w, w0, b, y, y0, c, n, dt, st); });
}

PyObject* gather_gemm_add(PyObject* const* a) {  // X kept_idx W R out_idx bias M
    const at::Tensor &X = matrix(a[0]), &W = matrix(a[2]), &R = matrix(a[3]);
    const at::Tensor *kept = index(a[1]), *out = index(a[4]);
    const lemo_dtype_t dt = dtype(X);
    const int64_t S = X.size(0), C = X.size(1), N = W.size(0);
    need(W.size(1) == C && W.scalar_type() == X.scalar_type() && R.scalar_type() == X.scalar_type() && R.size(1) == N);
    const int64_t M = a[6] != Py_None ? whole(a[6]) : kept ? kept->numel() : out ? out->numel() : S;
    need(M > 0 && (!kept || kept->numel() >= M) && (!out || out->numel() >= M));
    const void* b = bias_of(a[5], X, N);
    const int32_t *ki = rows(kept), *oi = rows(out);
    const int32_t c = size32(C), n = size32(N);
    void *x = X.data_ptr(), *w = W.data_ptr(), *r = R.data_ptr(), *st = stream();
    const int64_t x0 = X.stride(0), w0 = W.stride(0), r0 = R.stride(0), rs = R.size(0);
    return call([=] { return lemo_gather_gemm_add(x, S, x0, ki, M, w, w0, b, r, r0, rs, oi, c, n, dt, st); });
}

PyObject* gather_gemm_dx(PyObject* const* a) {  // dY W dX out_idx
    const at::Tensor &dY = matrix(a[0]), &W = matrix(a[1]), &dX = matrix(a[2]);
    const at::Tensor* out = index(a[3]);
    const lemo_dtype_t dt = dtype(W);
    const int64_t M = dY.size(0), N = dY.size(1), C = W.size(1);
    need(dY.scalar_type() == W.scalar_type() && dX.scalar_type() == W.scalar_type() && W.size(0) == N && dX.size(1) == C && (!out || out->numel() == M));
    const int32_t* oi = rows(out);
    const int32_t c = size32(C), n = size32(N);
    void *y = dY.data_ptr(), *w = W.data_ptr(), *x = dX.data_ptr(), *st = stream();
    const int64_t y0 = dY.stride(0), w0 = W.stride(0), x0 = dX.stride(0), xs = dX.size(0);
    return call([=] { return lemo_gather_gemm_dx(y, y0, M, w, w0, x, x0, xs, oi, c, n, dt, st); });
}

PyObject* gather_gemm_dw(PyObject* const* a) {  // dY X kept_idx dW workspace
    const at::Tensor &dY = matrix(a[0]), &X = matrix(a[1]), &dW = matrix(a[3]);
    const at::Tensor* kept = index(a[2]);
    const lemo_dtype_t dt = dtype(X);
    const int64_t M = dY.size(0), N = dY.size(1), S = X.size(0), C = X.size(1);
    need(dY.scalar_type() == X.scalar_type() && dW.scalar_type() == X.scalar_type() && dW.size(0) == N && dW.size(1) == C && (!kept || kept->numel() == M));
    Bytes ws{nullptr, 0};
    if (a[4] != Py_None) ws = workspace(a[4]);
    else need(dt == LEMO_BF16);  // binary32 needs one, which lemo.py allocates
    const int32_t* ki = rows(kept);
    const int32_t c = size32(C), n = size32(N);
    void *y = dY.data_ptr(), *x = X.data_ptr(), *w = dW.data_ptr(), *st = stream();
    const int64_t y0 = dY.stride(0), x0 = X.stride(0), w0 = dW.stride(0);
    return call([=] { return lemo_gather_gemm_dw(y, y0, x, S, x0, ki, M, w, w0, c, n, dt, ws.p, ws.n, st); });
}

PyObject* scatter_grad(PyObject* const* a) {  // G kept_idx dX mode
    const at::Tensor &G = matrix(a[0]), &dX = matrix(a[2]);
    const at::Tensor* kept = index(a[1]);
    const lemo_dtype_t gt = dtype(G), xt = dtype(dX);
    const int64_t M = G.size(0), C = G.size(1);
    need(kept && dX.size(1) == C && kept->numel() == M);
    const int32_t mode = whole32(a[3]), c = size32(C);
    const int32_t* ki = rows(kept);
    void *g = G.data_ptr(), *x = dX.data_ptr(), *st = stream();
    const int64_t g0 = G.stride(0), x0 = dX.stride(0), xs = dX.size(0);
    return call([=] { return lemo_scatter_grad(g, g0, ki, M, x, x0, xs, c, gt, xt, mode, st); });
}

// ---- the calls around chosen key blocks and the norms: results that are not given are allocated here, and come back in a tuple
// behind the return code.  Their tensors have to live on the current device, as lemo.py asks.

struct Place {
    int64_t device;
    void* stream;
    at::TensorOptions options;
    Place() {
        PyObject* dev = PyObject_CallNoArgs(current_device);
        if (!dev) { PyErr_Clear(); throw NotPlain{}; }
        device = PyLong_AsLongLong(dev);
        PyObject* s = PyObject_CallOneArg(raw_stream, dev);
        Py_DECREF(dev);
        if (!s) { PyErr_Clear(); throw NotPlain{}; }
        stream = PyLong_AsVoidPtr(s);
        Py_DECREF(s);
        if (PyErr_Occurred()) { PyErr_Clear(); throw NotPlain{}; }
        options = at::TensorOptions().device(at::kCUDA, (c10::DeviceIndex)device);
    }
    const at::Tensor& at(const at::Tensor& t) const {
        need(t.device().index() == device);
        return t;
    }
    // a contiguous result of the caller's, or a new one
    at::Tensor result(PyObject* o, at::IntArrayRef shape, at::ScalarType type) const {
        if (o == Py_None) return at::empty(shape, options.dtype(type));
        const at::Tensor& t = at(tensor(o, (int64_t)shape.size()));
        need(t.scalar_type() == type && t.sizes() == shape && t.is_contiguous());
        return t;
    }
    at::Tensor fresh(bool wanted, at::IntArrayRef shape, at::ScalarType type) const { return wanted ? at::empty(shape, options.dtype(type)) : at::Tensor(); }
    Bytes scratch(PyObject* o, size_t bytes, at::Tensor& keep) const {
        if (o != Py_None) {
            const Bytes b = workspace(o);
            need(THPVariable_Unpack(o).device().index() == device);
            return b;
        }
        if (bytes == 0) return {nullptr, 0};
        keep = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
        return {keep.data_ptr(), bytes};
    }
};
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// (return code, results...), or None where the C ABI refused
template <typename F> PyObject* call_for(F f, std::initializer_list<at::Tensor> results) {
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f();
    Py_END_ALLOW_THREADS;
    if (rc != LEMO_OK && rc != LEMO_ERR_HIP) Py_RETURN_NONE;
    PyObject* out = PyTuple_New(1 + (Py_ssize_t)results.size());
    if (!out) throw NotPlain{};
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(rc));
    Py_ssize_t i = 1;
    for (const at::Tensor& t : results) PyTuple_SET_ITEM(out, i++, t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None));
    return out;
}

const at::Tensor* maybe_matrix(PyObject* o, const Place& here, int64_t M, int64_t C, at::ScalarType type) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = here.at(matrix(o));
    need(t.size(0) == M && t.size(1) == C && t.scalar_type() == type);
    return &t;
}
const void* channels(PyObject* o, const Place& here, int64_t C, at::ScalarType type) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = here.at(tensor(o, 1));
    need(t.size(0) == C && t.scalar_type() == type && t.is_contiguous());
    return t.data_ptr();
}
struct NormSizes { int64_t M, S, C; const at::Tensor *Y, *gate, *kept; bool shared; const void* gate_at; int64_t ldg; };
NormSizes norm_sizes(PyObject* y, const at::Tensor& R, PyObject* k, PyObject* g, const Place& here) {
    NormSizes n{};
    n.S = R.size(0);
    n.C = R.size(1);
    n.kept = index(k);
    if (n.kept) here.at(*n.kept);
    n.M = y != Py_None ? matrix(y).size(0) : n.kept ? n.kept->numel() : n.S;
    need(!n.kept || n.kept->numel() == n.M);
    n.Y = maybe_matrix(y, here, n.M, n.C, R.scalar_type());
    if (g != Py_None) {
        need(THPVariable_CheckExact(g));
        n.shared = THPVariable_Unpack(g).dim() == 1;
        if (n.shared) n.gate_at = channels(g, here, n.C, R.scalar_type());
        else {
            n.gate = maybe_matrix(g, here, n.M, n.C, R.scalar_type());
            n.gate_at = n.gate->data_ptr();
            n.ldg = n.gate->stride(0);
        }
    }
    return n;
}

PyObject* norm_residual(PyObject* const* a) {  // Y R kept gate post next w_post b_post w_next b_next eps residual_scale block_scale flags N stats
    const Place here;
    const at::Tensor& R = here.at(matrix(a[1]));
    const lemo_dtype_t dt = dtype(R);
    const at::ScalarType type = R.scalar_type();
    const NormSizes n = norm_sizes(a[0], R, a[2], a[3], here);
    const int32_t post = whole32(a[4]), next = whole32(a[5]), flags = whole32(a[13]), C = size32(n.C);
    const void *wp = channels(a[6], here, n.C, type), *bp = channels(a[7], here, n.C, type), *wn = channels(a[8], here, n.C, type), *bn = channels(a[9], here, n.C, type);
    const float eps = real(a[10]), rs = real(a[11]), bs = real(a[12]);
    at::Tensor N;
    if (a[14] != Py_None) N = *maybe_matrix(a[14], here, n.M, n.C, type);
    else if (next != LEMO_NORM_NONE) N = at::empty({n.M, n.C}, here.options.dtype(type));
    const at::Tensor stats = here.result(a[15], {n.M, 4}, at::kFloat);
    const void* y = n.Y ? n.Y->data_ptr() : nullptr;
    void *r = R.data_ptr(), *out = address(N), *st = stats.data_ptr();
    const int64_t ldy = n.Y ? n.Y->stride(0) : n.C, ldn = N.defined() ? N.stride(0) : n.C, ldr = R.stride(0);
    const int32_t* ki = rows(n.kept);
    return call_for([=] {
        return lemo_norm_residual(y, ldy, n.gate_at, n.ldg, r, ldr, n.S, ki, n.M, wp, bp, post, wn, bn, next, eps, rs, bs, out, ldn, (float*)st, C, dt, (uint32_t)flags, here.stream);
    }, {N, stats});
}

PyObject* norm_residual_grad(PyObject* const* a) {  // dN dR R Y kept stats gate post next w_post b_post w_next residual_scale block_scale flags workspace dY dgate weights
    const Place here;
    const at::Tensor &dR = here.at(matrix(a[1])), &R = here.at(matrix(a[2])), &stats = here.at(tensor(a[5], 2));
    const lemo_dtype_t dt = dtype(R);
    const at::ScalarType type = R.scalar_type();
    const NormSizes n = norm_sizes(a[3], R, a[4], a[6], here);
    need(dR.sizes() == R.sizes() && dR.scalar_type() == type && stats.scalar_type() == at::kFloat && stats.is_contiguous() && stats.size(0) == n.M && stats.size(1) == 4);
    const at::Tensor* dN = maybe_matrix(a[0], here, n.M, n.C, type);
    const int32_t post = whole32(a[7]), next = whole32(a[8]), flags = whole32(a[14]), C = size32(n.C);
    const void *wp = channels(a[9], here, n.C, type), *bp = channels(a[10], here, n.C, type), *wn = channels(a[11], here, n.C, type);
    const float rs = real(a[12]), bs = real(a[13]);
    need(PyBool_Check(a[18]) && (n.Y || a[16] == Py_None) && (n.gate || n.shared || a[17] == Py_None));
    const bool p = a[18] == Py_True && post != LEMO_NORM_NONE, q = a[18] == Py_True && next != LEMO_NORM_NONE;
    size_t bytes = 0;
    need(!(p || q || n.shared) || lemo_norm_residual_grad_workspace_bytes(n.M, C, &bytes) == LEMO_OK);
    at::Tensor keep;
    const Bytes ws = here.scratch(a[15], bytes, keep);
    const at::Tensor *dy_given = maybe_matrix(a[16], here, n.M, n.C, type), *dg_given = n.shared ? nullptr : maybe_matrix(a[17], here, n.M, n.C, type);
    const at::Tensor dY = dy_given ? *dy_given : here.fresh(n.Y, {n.M, n.C}, type), dgate = dg_given ? *dg_given : here.fresh(n.gate, {n.M, n.C}, type);
    const at::Tensor dgs = n.shared ? here.result(a[17], {n.C}, at::kFloat) : at::Tensor();
    const at::Tensor dwp = here.fresh(p, {n.C}, at::kFloat), dbp = here.fresh(p && (bp || post == LEMO_NORM_LAYER), {n.C}, at::kFloat);
    const at::Tensor dwn = here.fresh(q, {n.C}, at::kFloat), dbn = here.fresh(q, {n.C}, at::kFloat);
    const void *y = n.Y ? n.Y->data_ptr() : nullptr, *dn = dN ? dN->data_ptr() : nullptr, *r = R.data_ptr(), *stp = stats.data_ptr();
    void *dr = dR.data_ptr(), *dy = address(dY), *dg = address(dgate), *s0 = address(dwp), *s1 = address(dbp), *s2 = address(dwn), *s3 = address(dbn), *s4 = address(dgs);
    const int64_t ldy = n.Y ? n.Y->stride(0) : n.C, lddn = dN ? dN->stride(0) : n.C, ldr = R.stride(0), lddr = dR.stride(0);
    const int64_t lddy = dY.defined() ? dY.stride(0) : n.C, lddg = dgate.defined() ? dgate.stride(0) : n.C;
    const int32_t* ki = rows(n.kept);
    return call_for([=] {
        return lemo_norm_residual_grad(dn, lddn, dr, lddr, n.S, r, ldr, y, ldy, n.gate_at, n.ldg, ki, n.M, wp, bp, post, wn, next, rs, bs, (const float*)stp, dy, lddy, dg, lddg,
                                       (float*)s0, (float*)s1, (float*)s2, (float*)s3, (float*)s4, C, dt, (uint32_t)flags, ws.p, ws.n, here.stream);
    }, {dY, n.shared ? dgs : dgate, dwp, dbp, dwn, dbn});
}

int64_t blocks_of(int64_t n, int64_t b) {
    need(b > 0);
    return (n + b - 1) / b;
}

PyObject* block_means(PyObject* const* a) {  // K b means
    const Place here;
    const at::Tensor& K = here.at(heads(a[0]));
    const lemo_dtype_t dt = dtype(K);
    const int32_t b = whole32(a[1]), hkv = size32(K.size(1)), d = size32(K.size(2));
    const at::Tensor means = here.result(a[2], {blocks_of(K.size(0), b), K.size(1), K.size(2)}, at::kFloat);
    void *k = K.data_ptr(), *m = means.data_ptr();
    const int64_t S = K.size(0), k0 = K.stride(0), k1 = K.stride(1);
    return call_for([=] { return lemo_block_means(k, S, hkv, d, dt, k0, k1, b, (float*)m, here.stream); }, {means});
}

PyObject* select_blocks(PyObject* const* a) {  // Q means S_k b bq T flags q_start blocks
    const Place here;
    const at::Tensor &Q = here.at(heads(a[0])), &means = here.at(tensor(a[1], 3));
    const lemo_dtype_t dt = dtype(Q);
    const int64_t Sk = whole(a[2]), start = whole(a[7]), S = Q.size(0);
    const int32_t b = whole32(a[3]), bq = whole32(a[4]), T = whole32(a[5]), flags = whole32(a[6]), h = size32(Q.size(1)), hkv = size32(means.size(1)), d = size32(Q.size(2));
    need(Sk > 0 && T > 0 && means.scalar_type() == at::kFloat && means.is_contiguous() && means.size(0) == blocks_of(Sk, b) && means.size(2) == d);
    const at::Tensor blocks = here.result(a[8], {blocks_of(S, bq), means.size(1), T}, at::kInt);
    void *q = Q.data_ptr(), *m = means.data_ptr(), *o = blocks.data_ptr();
    const int64_t q0 = Q.stride(0), q1 = Q.stride(1);
    return call_for([=] { return lemo_select_blocks(q, S, h, hkv, d, dt, q0, q1, (const float*)m, Sk, start, b, bq, T, (uint32_t)flags, (int32_t*)o, here.stream); }, {blocks});
}

struct AttentionSizes { int64_t S, Sk; int32_t h, hkv, d, T; };
AttentionSizes attention_sizes(const at::Tensor& Q, const at::Tensor& K, const at::Tensor& V, const at::Tensor& blocks, int64_t bq) {
    need(K.size(2) == Q.size(2) && V.sizes() == K.sizes() && K.scalar_type() == Q.scalar_type() && V.scalar_type() == Q.scalar_type());
    need(blocks.scalar_type() == at::kInt && blocks.is_contiguous() && blocks.size(0) == blocks_of(Q.size(0), bq) && blocks.size(1) == K.size(1));
    return {Q.size(0), K.size(0), size32(Q.size(1)), size32(K.size(1)), size32(Q.size(2)), size32(blocks.size(2))};
}

PyObject* block_attention(PyObject* const* a) {  // Q K V blocks b bq flags scale q_start O lse2 workspace
    const Place here;
    const at::Tensor &Q = here.at(heads(a[0])), &K = here.at(heads(a[1])), &V = here.at(heads(a[2])), &blocks = here.at(tensor(a[3], 3));
    const lemo_dtype_t dt = dtype(Q);
    const int32_t b = whole32(a[4]), bq = whole32(a[5]), flags = whole32(a[6]);
    const float scale = real(a[7]);
    const int64_t start = whole(a[8]);
    const AttentionSizes n = attention_sizes(Q, K, V, blocks, bq);
    const at::Tensor O = a[9] == Py_None ? at::empty({n.S, n.h, n.d}, here.options.dtype(Q.scalar_type())) : here.at(heads(a[9]));
    need(O.scalar_type() == Q.scalar_type() && O.sizes() == Q.sizes());
    const at::Tensor lse2 = here.result(a[10], {n.h, n.S}, at::kFloat);
    size_t bytes = 0;
    need(lemo_block_attention_workspace_bytes(n.S, n.Sk, n.h, n.hkv, n.d, n.T, b, bq, &bytes) == LEMO_OK);
    at::Tensor keep;
    const Bytes ws = here.scratch(a[11], bytes, keep);
    void *q = Q.data_ptr(), *k = K.data_ptr(), *v = V.data_ptr(), *bl = blocks.data_ptr(), *o = O.data_ptr(), *l = lse2.data_ptr();
    const int64_t q0 = Q.stride(0), q1 = Q.stride(1), k0 = K.stride(0), k1 = K.stride(1), v0 = V.stride(0), v1 = V.stride(1), o0 = O.stride(0), o1 = O.stride(1);
    return call_for([=] {
        return lemo_block_attention(q, k, v, n.S, n.Sk, n.h, n.hkv, n.d, dt, q0, q1, k0, k1, v0, v1, (const int32_t*)bl, n.T, b, bq, start, scale, (uint32_t)flags, o, o0, o1,
                                    (float*)l, ws.p, ws.n, here.stream);
    }, {O, lse2});
}

PyObject* block_attention_grad(PyObject* const* a) {  // dO Q K V O lse2 blocks b bq flags scale q_start dQ dK dV workspace
    const Place here;
    const at::Tensor &dO = here.at(heads(a[0])), &Q = here.at(heads(a[1])), &K = here.at(heads(a[2])), &V = here.at(heads(a[3])), &O = here.at(heads(a[4]));
    const at::Tensor &lse2 = here.at(tensor(a[5], 2)), &blocks = here.at(tensor(a[6], 3));
    const lemo_dtype_t dt = dtype(Q);
    const at::ScalarType type = Q.scalar_type();
    const int32_t b = whole32(a[7]), bq = whole32(a[8]), flags = whole32(a[9]);
    const float scale = real(a[10]);
    const int64_t start = whole(a[11]);
    const AttentionSizes n = attention_sizes(Q, K, V, blocks, bq);
    need(dO.sizes() == Q.sizes() && O.sizes() == Q.sizes() && dO.scalar_type() == type && O.scalar_type() == type);
    need(lse2.scalar_type() == at::kFloat && lse2.is_contiguous() && lse2.size(0) == n.h && lse2.size(1) == n.S);
    const at::Tensor dQ = here.result(a[12], {n.S, n.h, n.d}, type), dK = here.result(a[13], {n.Sk, n.hkv, n.d}, type), dV = here.result(a[14], {n.Sk, n.hkv, n.d}, type);
    size_t bytes = 0;
    need(lemo_block_attention_grad_workspace_bytes(n.S, n.Sk, n.h, n.hkv, n.d, n.T, b, bq, &bytes) == LEMO_OK);
    at::Tensor keep;
    const Bytes ws = here.scratch(a[15], bytes, keep);
    void *g = dO.data_ptr(), *q = Q.data_ptr(), *k = K.data_ptr(), *v = V.data_ptr(), *o = O.data_ptr(), *l = lse2.data_ptr(), *bl = blocks.data_ptr();
    void *gq = dQ.data_ptr(), *gk = dK.data_ptr(), *gv = dV.data_ptr();
    const int64_t g0 = dO.stride(0), g1 = dO.stride(1), q0 = Q.stride(0), q1 = Q.stride(1), k0 = K.stride(0), k1 = K.stride(1), v0 = V.stride(0), v1 = V.stride(1),
                  o0 = O.stride(0), o1 = O.stride(1);
    return call_for([=] {
        return lemo_block_attention_grad(g, q, k, v, o, (const float*)l, n.S, n.Sk, n.h, n.hkv, n.d, dt, g0, g1, q0, q1, k0, k1, v0, v1, o0, o1, (const int32_t*)bl, n.T, b, bq,
                                         start, scale, (uint32_t)flags, gq, gk, gv, ws.p, ws.n, here.stream);
    }, {dQ, dK, dV});
}

const at::Tensor& cache(PyObject* o, const Place& here) {  // [B,S,H_kv,d], d contiguous
    const at::Tensor& t = here.at(tensor(o, 4));
    need(t.stride(3) == 1);
    return t;
}
const int32_t* sequence_lengths(PyObject* o, const Place& here, int64_t B) {
    const at::Tensor* t = index(o);
    need(t && t->numel() == B);
    here.at(*t);
    return rows(t);
}

PyObject* select_blocks_step(PyObject* const* a) {  // Q means lengths b T blocks S_max
    const Place here;
    const at::Tensor &Q = here.at(heads(a[0])), &means = here.at(tensor(a[1], 4));
    const lemo_dtype_t dt = dtype(Q);
    const int32_t b = whole32(a[3]), T = whole32(a[4]), B = size32(Q.size(0)), h = size32(Q.size(1)), hkv = size32(means.size(2)), d = size32(Q.size(2));
    const int64_t S = a[6] == Py_None ? means.size(1) * b : whole(a[6]);
    need(S > 0 && T > 0 && means.scalar_type() == at::kFloat && means.is_contiguous() && means.size(0) == B && means.size(1) == blocks_of(S, b) && means.size(3) == d);
    const int32_t* len = sequence_lengths(a[2], here, B);
    const at::Tensor blocks = here.result(a[5], {B, means.size(2), T}, at::kInt);
    void *q = Q.data_ptr(), *m = means.data_ptr(), *o = blocks.data_ptr();
    const int64_t q0 = Q.stride(0), q1 = Q.stride(1);
    return call_for([=] { return lemo_select_blocks_step(q, B, h, hkv, d, dt, q0, q1, (const float*)m, S, len, b, T, (int32_t*)o, here.stream); }, {blocks});
}

PyObject* block_attention_step(PyObject* const* a) {  // Q K V lengths blocks b scale O workspace
    const Place here;
    const at::Tensor &Q = here.at(heads(a[0])), &K = cache(a[1], here), &V = cache(a[2], here), &blocks = here.at(tensor(a[4], 3));
    const lemo_dtype_t dt = dtype(Q);
    const int32_t b = whole32(a[5]), B = size32(Q.size(0)), h = size32(Q.size(1)), hkv = size32(K.size(2)), d = size32(Q.size(2)), T = size32(blocks.size(2));
    const float scale = real(a[6]);
    need(K.size(0) == B && K.size(3) == d && V.sizes() == K.sizes() && K.scalar_type() == Q.scalar_type() && V.scalar_type() == Q.scalar_type());
    need(blocks.scalar_type() == at::kInt && blocks.is_contiguous() && blocks.size(0) == B && blocks.size(1) == hkv);
    const int32_t* len = sequence_lengths(a[3], here, B);
    const at::Tensor O = a[7] == Py_None ? at::empty({B, h, d}, here.options.dtype(Q.scalar_type())) : here.at(heads(a[7]));
    need(O.scalar_type() == Q.scalar_type() && O.sizes() == Q.sizes());
    size_t bytes = 0;
    need(lemo_block_attention_step_workspace_bytes(B, h, hkv, d, T, b, &bytes) == LEMO_OK);
    at::Tensor keep;
    const Bytes ws = here.scratch(a[8], bytes, keep);
    void *q = Q.data_ptr(), *k = K.data_ptr(), *v = V.data_ptr(), *bl = blocks.data_ptr(), *o = O.data_ptr();
    const int64_t S = K.size(1), q0 = Q.stride(0), q1 = Q.stride(1), k0 = K.stride(0), k1 = K.stride(1), k2 = K.stride(2), v0 = V.stride(0), v1 = V.stride(1), v2 = V.stride(2),
                  o0 = O.stride(0), o1 = O.stride(1);
    return call_for([=] {
        return lemo_block_attention_step(q, k, v, B, S, h, hkv, d, dt, q0, q1, k0, k1, k2, v0, v1, v2, len, (const int32_t*)bl, T, b, scale, o, o0, o1, ws.p, ws.n, here.stream);
    }, {O});
}

// queries or keys of the calls on heads, or none
struct Side { const at::Tensor* t; void* p; int64_t ts, hs; int32_t heads; };
Side side(PyObject* o, const Place& here) {
    if (o == Py_None) return {nullptr, nullptr, 0, 0, 0};
    const at::Tensor& t = here.at(heads(o));
    return {&t, t.data_ptr(), t.stride(0), t.stride(1), size32(t.size(1))};
}
// a result like `s`: the caller's, or a new one in `keep`
Side like(const Side& s, PyObject* o, const Place& here, at::Tensor& keep) {
    if (!s.t) {
        need(o == Py_None);
        return s;
    }
    keep = o == Py_None ? at::empty(s.t->sizes(), here.options.dtype(s.t->scalar_type())) : here.at(heads(o));
    need(keep.sizes() == s.t->sizes() && keep.scalar_type() == s.t->scalar_type());
    return {&keep, keep.data_ptr(), keep.stride(0), keep.stride(1), s.heads};
}
struct Rotation { int64_t M; int32_t d, rot, flags; lemo_dtype_t dt; at::ScalarType type; const float* freq; const void *wq, *wk; const at::Tensor *tq, *tk; };
Rotation rotation(const Side& q, const Side& k, PyObject* freq, PyObject* wq, PyObject* wk, int32_t norm, int32_t flags, const Place& here) {
    need(q.t || k.t);
    const at::Tensor& one = q.t ? *q.t : *k.t;
    Rotation r{one.size(0), size32(one.size(2)), 0, flags, dtype(one), one.scalar_type(), nullptr, nullptr, nullptr, nullptr, nullptr};
    need(!q.t || !k.t || (k.t->size(0) == r.M && k.t->size(2) == r.d && k.t->scalar_type() == r.type));
    if (freq != Py_None) {
        const at::Tensor& t = here.at(tensor(freq, 1));
        need(t.scalar_type() == at::kFloat && t.is_contiguous() && t.size(0) < (1 << 20));
        r.freq = static_cast<const float*>(t.data_ptr());
        r.rot = 2 * (int32_t)t.size(0);
    }
    auto weight = [&](PyObject* o, const Side& of, const void*& p, const at::Tensor*& t) {
        if (o == Py_None) return;
        need(THPVariable_CheckExact(o) && of.t && norm != LEMO_NORM_NONE);
        const int64_t dims = THPVariable_Unpack(o).dim();
        t = &here.at(tensor(o, dims));
        need((dims == 1 || (dims == 2 && t->size(0) == of.heads)) && t->size(dims - 1) == r.d && t->scalar_type() == r.type && t->is_contiguous());
        p = t->data_ptr();
    };
    weight(wq, q, r.wq, r.tq);
    weight(wk, k, r.wk, r.tk);
    need(!r.tq || !r.tk || r.tq->dim() == r.tk->dim());
    if ((r.tq && r.tq->dim() == 2) || (r.tk && r.tk->dim() == 2)) r.flags |= LEMO_WEIGHTS_PER_HEAD;
    need(!(flags & LEMO_WEIGHTS_PER_HEAD) || ((!r.tq || r.tq->dim() == 2) && (!r.tk || r.tk->dim() == 2)));  // (shared ones are no [heads, d])
    return r;
}
const int32_t* positions_of(PyObject* o, const Place& here, int64_t M) {
    const at::Tensor* t = index(o);
    need(!t || (t->numel() == M && here.at(*t).defined()));
    return rows(t);
}

PyObject* qk_rotate(PyObject* const* a) {  // Q K inv_freq positions pos_start norm w_q w_k eps amplitude flags Q_out K_out
    const Place here;
    const Side q = side(a[0], here), k = side(a[1], here);
    const int64_t start = whole(a[4]);
    const int32_t norm = whole32(a[5]);
    const float eps = real(a[8]), amplitude = real(a[9]);
    const Rotation r = rotation(q, k, a[2], a[6], a[7], norm, whole32(a[10]), here);
    const int32_t* pos = positions_of(a[3], here, r.M);
    at::Tensor Q, K;
    const Side qo = like(q, a[11], here, Q), ko = like(k, a[12], here, K);
    return call_for([=] {
        return lemo_qk_rotate(q.p, q.ts, q.hs, k.p, k.ts, k.hs, r.M, q.heads, k.heads, r.d, r.dt, pos, start, r.freq, r.rot, amplitude, norm, r.wq, r.wk, eps, (uint32_t)r.flags,
                              qo.p, qo.ts, qo.hs, ko.p, ko.ts, ko.hs, here.stream);
    }, {Q, K});
}

PyObject* qk_rotate_grad(PyObject* const* a) {  // dQ_out dK_out Q K inv_freq positions pos_start norm w_q w_k eps amplitude flags dQ dK weights workspace
    const Place here;
    const Side gq = side(a[0], here), gk = side(a[1], here);
    const int64_t start = whole(a[6]);
    const int32_t norm = whole32(a[7]);
    const float eps = real(a[10]), amplitude = real(a[11]);
    const Rotation r = rotation(gq, gk, a[4], a[8], a[9], norm, whole32(a[12]), here);
    const int32_t* pos = positions_of(a[5], here, r.M);
    need(PyBool_Check(a[15]));
    const bool sums = a[15] == Py_True && (r.tq || r.tk);
    auto operand = [&](PyObject* o, const Side& g) {
        if (norm == LEMO_NORM_NONE) return Side{nullptr, nullptr, 0, 0, 0};
        const Side x = side(o, here);
        need((x.t != nullptr) == (g.t != nullptr) && (!x.t || (x.t->sizes() == g.t->sizes() && x.t->scalar_type() == g.t->scalar_type())));
        return x;
    };
    const Side q = operand(a[2], gq), k = operand(a[3], gk);
    at::Tensor Q, K, keep;
    const Side dq = like(gq, a[13], here, Q), dk = like(gk, a[14], here, K);
    const at::Tensor wq = here.fresh(sums && r.tq, r.tq ? r.tq->sizes() : at::IntArrayRef{}, at::kFloat), wk = here.fresh(sums && r.tk, r.tk ? r.tk->sizes() : at::IntArrayRef{}, at::kFloat);
    size_t bytes = 0;
    need(!sums || lemo_qk_rotate_grad_workspace_bytes(r.M, gq.heads, gk.heads, r.d, r.dt, (uint32_t)r.flags, &bytes) == LEMO_OK);
    const Bytes ws = here.scratch(a[16], bytes, keep);
    void *sq = address(wq), *sk = address(wk);
    return call_for([=] {
        return lemo_qk_rotate_grad(gq.p, gq.ts, gq.hs, gk.p, gk.ts, gk.hs, q.p, q.ts, q.hs, k.p, k.ts, k.hs, r.M, gq.heads, gk.heads, r.d, r.dt, pos, start, r.freq, r.rot, amplitude,
                                   norm, r.wq, r.wk, eps, (uint32_t)r.flags, dq.p, dq.ts, dq.hs, dk.p, dk.ts, dk.hs, (float*)sq, (float*)sk, ws.p, ws.n, here.stream);
    }, {Q, K, wq, wk});
}

PyObject* qk_rotate_step(PyObject* const* a) {  // Q K V K_cache V_cache lengths inv_freq norm w_q w_k eps amplitude flags Q_out
    const Place here;
    const Side q = side(a[0], here), k = side(a[1], here), v = side(a[2], here);
    const int32_t norm = whole32(a[7]);
    const float eps = real(a[10]), amplitude = real(a[11]);
    const Rotation r = rotation(q, k, a[6], a[8], a[9], norm, whole32(a[12]), here);
    need(q.t && k.t && (v.t != nullptr) == (a[4] != Py_None));
    const at::Tensor& kc = cache(a[3], here);
    const at::Tensor& vc = v.t ? cache(a[4], here) : kc;
    need(kc.size(0) == r.M && kc.size(2) == k.heads && kc.size(3) == r.d && kc.scalar_type() == r.type && vc.sizes() == kc.sizes() && vc.scalar_type() == r.type);
    need(!v.t || (v.t->sizes() == k.t->sizes() && v.t->scalar_type() == r.type));
    const int32_t* len = sequence_lengths(a[5], here, r.M);
    const int32_t B = size32(r.M);
    at::Tensor Q;
    const Side qo = like(q, a[13], here, Q);
    void *kp = kc.data_ptr(), *vp = v.t ? vc.data_ptr() : nullptr;
    const int64_t S = kc.size(1), k0 = kc.stride(0), k1 = kc.stride(1), k2 = kc.stride(2), v0 = vc.stride(0), v1 = vc.stride(1), v2 = vc.stride(2);
    return call_for([=] {
        return lemo_qk_rotate_step(q.p, q.ts, q.hs, k.p, k.ts, k.hs, v.p, v.ts, v.hs, B, S, q.heads, k.heads, r.d, r.dt, len, r.freq, r.rot, amplitude, norm, r.wq, r.wk, eps,
                                   (uint32_t)r.flags, qo.p, qo.ts, qo.hs, kp, k0, k1, k2, vp, v0, v1, v2, here.stream);
    }, {Q});
}

double real64(PyObject* o) {
    need(PyFloat_CheckExact(o));
    return PyFloat_AS_DOUBLE(o);
}
const uint64_t* generator(PyObject* o, const Place& here) {
    const at::Tensor& t = here.at(tensor(o, 1));
    need((t.scalar_type() == at::kLong || t.scalar_type() == at::kUInt64) && t.size(0) == 2 && t.is_contiguous());
    return static_cast<const uint64_t*>(t.data_ptr());
}

PyObject* dropout_add(PyObject* const* a) {  // Y R kept rng p site
    const Place here;
    const at::Tensor &Y = here.at(matrix(a[0])), &R = here.at(matrix(a[1]));
    const lemo_dtype_t dt = dtype(R);
    const int64_t M = Y.size(0), S = R.size(0), site = whole(a[5]), ldy = Y.stride(0), ldr = R.stride(0);
    const int32_t C = size32(R.size(1));
    need(Y.size(1) == C && Y.scalar_type() == R.scalar_type());
    const int32_t* ki = positions_of(a[2], here, M);
    const uint64_t* rng = generator(a[3], here);
    const double p = real64(a[4]);
    void *y = Y.data_ptr(), *r = R.data_ptr();
    return call([=] { return lemo_dropout_add(y, ldy, r, ldr, S, ki, M, p, rng, (uint64_t)site, C, dt, here.stream); });
}

PyObject* dropout_add_grad(PyObject* const* a) {  // dR kept rng p site dY
    const Place here;
    const at::Tensor& R = here.at(matrix(a[0]));
    const lemo_dtype_t dt = dtype(R);
    const at::Tensor* kept = index(a[1]);
    const int64_t S = R.size(0), site = whole(a[4]), ldr = R.stride(0), C = R.size(1);
    need(kept || a[5] == Py_None || THPVariable_CheckExact(a[5]));
    const int64_t M = kept ? here.at(*kept).numel() : a[5] == Py_None ? S : matrix(a[5]).size(0);
    const at::Tensor* given = maybe_matrix(a[5], here, M, C, R.scalar_type());
    const uint64_t* rng = generator(a[2], here);
    const double p = real64(a[3]);
    const at::Tensor Y = given ? *given : here.fresh(true, {M, C}, R.scalar_type());
    void *y = Y.data_ptr(), *r = R.data_ptr();
    const int64_t ldy = Y.stride(0);
    const int32_t c = size32(C), *ki = rows(kept);
    return call_for([=] { return lemo_dropout_add_grad(r, ldr, S, ki, M, p, rng, (uint64_t)site, y, ldy, c, dt, here.stream); }, {Y});
}

struct Head { int64_t S, M, ldx, ldw; int32_t C, V; lemo_dtype_t dt; at::ScalarType type; void *X, *W; const int32_t *kept, *labels; };
Head head(PyObject* x, PyObject* k, PyObject* w, PyObject* l, const Place& here) {
    const at::Tensor &X = here.at(matrix(x)), &W = here.at(matrix(w)), &labels = here.at(tensor(l, 1));
    need(X.size(1) == W.size(1) && X.scalar_type() == W.scalar_type() && labels.scalar_type() == at::kInt && labels.is_contiguous());
    const int64_t M = labels.numel();
    return {X.size(0), M, X.stride(0), W.stride(0), size32(X.size(1)), size32(W.size(0)), dtype(X), X.scalar_type(), X.data_ptr(), W.data_ptr(), positions_of(k, here, M),
            static_cast<const int32_t*>(labels.data_ptr())};
}

PyObject* vocab_loss(PyObject* const* a) {  // X kept W labels softcap smoothing z_weight loss lse total workspace
    const Place here;
    const Head h = head(a[0], a[1], a[2], a[3], here);
    const float cap = real(a[4]), s = real(a[5]), z = real(a[6]);
    const at::Tensor loss = here.result(a[7], {h.M}, at::kFloat), lse = here.result(a[8], {h.M}, at::kFloat), total = here.result(a[9], {4}, at::kFloat);
    size_t bytes = 0;
    need(lemo_vocab_loss_workspace_bytes(h.M, h.C, h.V, h.dt, &bytes) == LEMO_OK);
    at::Tensor keep;
    const Bytes ws = here.scratch(a[10], bytes, keep);
    void *l0 = loss.data_ptr(), *l1 = lse.data_ptr(), *l2 = total.data_ptr();
    return call_for([=] {
        return lemo_vocab_loss(h.X, h.S, h.ldx, h.kept, h.M, h.W, h.ldw, h.C, h.V, h.dt, h.labels, cap, s, z, (float*)l0, (float*)l1, (float*)l2, ws.p, ws.n, here.stream);
    }, {loss, lse, total});
}

PyObject* vocab_loss_grad(PyObject* const* a) {  // dloss X kept W labels lse softcap smoothing z_weight want_dX want_dW dX dW piece workspace
    const Place here;
    const Head h = head(a[1], a[2], a[3], a[4], here);
    const at::Tensor &dloss = here.at(tensor(a[0], 1)), &lse = here.at(tensor(a[5], 1));
    need(dloss.scalar_type() == at::kFloat && dloss.is_contiguous() && (dloss.numel() == 1 || dloss.numel() == h.M));
    need(lse.scalar_type() == at::kFloat && lse.is_contiguous() && lse.numel() == h.M && PyBool_Check(a[9]) && PyBool_Check(a[10]));
    const float cap = real(a[6]), s = real(a[7]), z = real(a[8]);
    const bool x = a[9] == Py_True, w = a[10] == Py_True;
    const int32_t piece = whole32(a[13]);
    const at::Tensor *gx = x ? maybe_matrix(a[11], here, h.M, h.C, h.type) : nullptr, *gw = w ? maybe_matrix(a[12], here, h.V, h.C, h.type) : nullptr;
    const at::Tensor dX = gx ? *gx : here.fresh(x, {h.M, h.C}, h.type), dW = gw ? *gw : here.fresh(w, {h.V, h.C}, h.type);
    size_t bytes = 0;
    need(lemo_vocab_loss_grad_workspace_bytes(h.M, h.C, h.V, h.ldw, h.dt, piece, &bytes) == LEMO_OK);
    at::Tensor keep;
    const Bytes ws = here.scratch(a[14], bytes, keep);
    void *g = dloss.data_ptr(), *l = lse.data_ptr(), *px = address(dX), *pw = address(dW);
    const int64_t gs = dloss.numel() == h.M, lddx = x ? dX.stride(0) : h.C, lddw = w ? dW.stride(0) : h.C;
    return call_for([=] {
        return lemo_vocab_loss_grad((const float*)g, gs, h.X, h.S, h.ldx, h.kept, h.M, h.W, h.ldw, h.C, h.V, h.dt, h.labels, (const float*)l, cap, s, z, px, lddx, pw, lddw, piece,
                                    ws.p, ws.n, here.stream);
    }, {dX, dW});
}

PyObject* set_stream_source(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "set_stream_source(current_device, raw_stream)");
        return nullptr;
    }
    Py_XSETREF(current_device, Py_NewRef(a[0]));
    Py_XSETREF(raw_stream, Py_NewRef(a[1]));
    Py_RETURN_NONE;
}

#define LEMO_FAST(name, n) {#name, (PyCFunction)(void*)(guarded<n, name>), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LEMO_FAST(score_segments, 9), LEMO_FAST(select_topk, 4), LEMO_FAST(kept_attention, 9), LEMO_FAST(gather_gemm, 6),
                         LEMO_FAST(gather_gemm_add, 7), LEMO_FAST(gather_gemm_dx, 4), LEMO_FAST(gather_gemm_dw, 5), LEMO_FAST(scatter_grad, 4),
                         LEMO_FAST(norm_residual, 16), LEMO_FAST(norm_residual_grad, 19), LEMO_FAST(block_means, 3), LEMO_FAST(select_blocks, 9),
                         LEMO_FAST(block_attention, 12), LEMO_FAST(block_attention_grad, 16), LEMO_FAST(select_blocks_step, 7), LEMO_FAST(block_attention_step, 9),
                         LEMO_FAST(qk_rotate, 13), LEMO_FAST(qk_rotate_grad, 17), LEMO_FAST(qk_rotate_step, 14), LEMO_FAST(dropout_add, 6), LEMO_FAST(dropout_add_grad, 6),
                         LEMO_FAST(vocab_loss, 11), LEMO_FAST(vocab_loss_grad, 15),
                         {"set_stream_source", (PyCFunction)(void*)set_stream_source, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "lemo_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_lemo_native() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", LEMO_TORCH_VERSION) != 0) Py_CLEAR(m);  // (build.py)
    return m;
}
