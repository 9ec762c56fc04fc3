// Argument marshalling between torch tensors and the C-ABI of libflare, as a Python extension module.
//
// A small problem takes the GPU a few microseconds per kernel, so what a call costs on the host is most of it: checking
// nine tensors and converting them to C pointers in Python took longer than the kernels ran.  Here a check is a few loads,
// and the convenience calls take their scratch (workspace, statistics) in one allocation.  Measured, host time of a call: float32
// forward of 1024 tokens 45 -> 17 us, training step of 16384 tokens 127 -> 61 us (its launches are most of that).
//
// The module does not link libflare: flare.py loads the library and hands over the addresses of its functions (bind).
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <map>
#include <string>
#include <vector>

#include "../../include/flare.h"

namespace {

struct Library {
    decltype(&flare_workspace_bytes) workspace_bytes;
    decltype(&flare_encode) encode;
    decltype(&flare_encode_static_scratch) encode_static_scratch;
    decltype(&flare_decode) decode;
    decltype(&flare_forward) forward;
    decltype(&flare_backward) backward;
    decltype(&flare_forward_host) forward_host;
    decltype(&flare_forward_variant) forward_variant;
    decltype(&flare_backward_variant) backward_variant;
    decltype(&flare_spectral_gram) spectral_gram;
    decltype(&flare_spectral_eig) spectral_eig;
    decltype(&flare_block_workspace_bytes) block_workspace_bytes;
    decltype(&flare_norm_forward) norm_forward;
    decltype(&flare_norm_backward) norm_backward;
    decltype(&flare_join_forward) join_forward;
    decltype(&flare_join_backward) join_backward;
    decltype(&flare_orthogonalize_workspace_bytes) orthogonalize_workspace_bytes;
    decltype(&flare_orthogonalize) orthogonalize;
    decltype(&flare_muon_update) muon_update;
} lib{};
PyObject *flare_error = nullptr;   // the exception class (status, where)

// Raised inside the marshalling code after a Python error has been set.
struct PythonError {};

[[noreturn]] void fail(PyObject *type, const std::string &text) {
    PyErr_SetString(type, text.c_str());
    throw PythonError{};
}
void check_status(int rc, const char *where) {
    if (rc == FLARE_OK) return;
    PyObject *e = PyObject_CallFunction(flare_error, "is", rc, where);
    if (e) {
        PyErr_SetObject(flare_error, e);
        Py_DECREF(e);
    }
    throw PythonError{};
}

std::string dtype_name(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return "torch.float32";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kHalf: return "torch.float16";
        case at::kByte: return "torch.uint8";
        default: return c10::toString(t);
    }
}
std::string shape_text(at::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += std::to_string(s[i]) + (s.size() == 1 ? "," : i + 1 < s.size() ? ", " : "");
    return r + ")";
}

const at::Tensor &tensor(PyObject *o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a torch tensor");
    return THPVariable_Unpack(o);
}
void check(const at::Tensor &t, at::ScalarType dtype, at::IntArrayRef shape, bool cuda = true) {
    if (cuda && !t.is_cuda()) fail(PyExc_ValueError, "expected a CUDA tensor");
    if (!t.is_contiguous()) fail(PyExc_ValueError, "expected a contiguous tensor");
    if (t.scalar_type() != dtype) fail(PyExc_TypeError, "expected " + dtype_name(dtype) + ", got " + dtype_name(t.scalar_type()));
    if (t.sizes() != shape) fail(PyExc_ValueError, "expected shape " + shape_text(shape) + ", got " + shape_text(t.sizes()));
}

// The tensors of one call: shapes follow from the descriptor, the call's element type from K.
struct Call {
    const flare_desc_t *d;
    at::ScalarType dt;
    void *ptr(PyObject *o, at::ScalarType dtype, at::IntArrayRef shape, bool cuda = true) const {
        if (o == Py_None) return nullptr;
        const at::Tensor &t = tensor(o);
        check(t, dtype, shape, cuda);
        return t.data_ptr();
    }
    void *q(PyObject *o, bool shared = false, bool cuda = true) const {
        return shared ? ptr(o, dt, {d->M, d->D}, cuda) : ptr(o, dt, {d->H, d->M, d->D}, cuda);
    }
    void *tok(PyObject *o, bool cuda = true) const { return ptr(o, dt, {d->B, d->N, d->H, d->D}, cuda); }
    uint8_t *mask(PyObject *o, bool cuda = true) const { return (uint8_t *)ptr(o, at::kByte, {d->B, d->N}, cuda); }
    float *z(PyObject *o) const { return (float *)ptr(o, at::kFloat, {d->B, d->H, d->M, d->D}); }
    float *le(PyObject *o) const { return (float *)ptr(o, at::kFloat, {d->B, d->H, d->M}); }
    float *ld(PyObject *o) const { return (float *)ptr(o, at::kFloat, {d->B, d->N, d->H}); }
    float *dq(PyObject *o, bool shared = false) const {
        return (float *)(shared ? ptr(o, at::kFloat, {d->M, d->D}) : ptr(o, at::kFloat, {d->H, d->M, d->D}));
    }
};
struct Workspace {
    void *p = nullptr;
    size_t n = 0;
    explicit Workspace(PyObject *o) {
        if (o == Py_None) return;
        const at::Tensor &t = tensor(o);
        check(t, at::kByte, t.sizes());
        p = t.data_ptr();
        n = (size_t)t.numel();
    }
};

// A FlareDesc (a ctypes structure: its memory through the buffer protocol).
struct Desc {
    Py_buffer view;
    explicit Desc(PyObject *o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw PythonError{};
        if (view.len != (Py_ssize_t)sizeof(flare_desc_t)) {
            PyBuffer_Release(&view);
            fail(PyExc_TypeError, "expected a FlareDesc");
        }
    }
    ~Desc() { PyBuffer_Release(&view); }
    Desc(const Desc &) = delete;
    const flare_desc_t *get() const { return (const flare_desc_t *)view.buf; }
};

flare_stream_t stream_of(PyObject *o) {
    if (o == Py_None) return (flare_stream_t)c10::cuda::getCurrentCUDAStream().stream();
    PyObject *h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) throw PythonError{};
    void *p = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (PyErr_Occurred()) throw PythonError{};
    return (flare_stream_t)p;
}

// Every function below takes positional arguments only; the defaults and keyword names are those of the wrappers in flare.py.
template <typename F>
PyObject *guarded(Py_ssize_t got, Py_ssize_t want, F body) {
    if (got != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
        return nullptr;
    }
    try {
        return body();
    } catch (const PythonError &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
// Call into the library without the interpreter's lock.
template <typename F>
int unlocked(F call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

#define BINDING(name, count) PyObject *py_##name(PyObject *, PyObject *const *a, Py_ssize_t n) { return guarded(n, count, [&]() -> PyObject * {
#define BINDING_END Py_RETURN_NONE; }); }

// desc, Q, K, V, key_mask, Z, lse_enc, workspace, stream
BINDING(encode, 9)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *q = c.q(a[1]), *k = c.tok(a[2]), *v = c.tok(a[3]);
    uint8_t *m = c.mask(a[4]);
    float *z = c.z(a[5]), *le = c.le(a[6]);
    const Workspace w(a[7]);
    flare_stream_t st = stream_of(a[8]);
    check_status(unlocked([&] { return lib.encode(c.d, q, k, v, m, z, le, w.p, w.n, st); }), "flare_encode");
BINDING_END

// desc, Q, K, V, key_mask, Z, lse_enc, stream
BINDING(encode_static_scratch, 8)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *q = c.q(a[1]), *k = c.tok(a[2]), *v = c.tok(a[3]);
    uint8_t *m = c.mask(a[4]);
    float *z = c.z(a[5]), *le = c.le(a[6]);
    flare_stream_t st = stream_of(a[7]);
    check_status(unlocked([&] { return lib.encode_static_scratch(c.d, q, k, v, m, z, le, st); }), "flare_encode_static_scratch");
BINDING_END

// desc, Q, K, Z, Y, lse_dec, workspace, stream
BINDING(decode, 8)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *q = c.q(a[1]), *k = c.tok(a[2]);
    float *z = c.z(a[3]);
    void *y = c.tok(a[4]);
    float *ld = c.ld(a[5]);
    const Workspace w(a[6]);
    flare_stream_t st = stream_of(a[7]);
    check_status(unlocked([&] { return lib.decode(c.d, q, k, z, y, ld, w.p, w.n, st); }), "flare_decode");
BINDING_END

// desc, Q, K, V, key_mask, Y, Z, lse_enc, lse_dec, workspace, stream
BINDING(forward, 11)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *q = c.q(a[1]), *k = c.tok(a[2]), *v = c.tok(a[3]);
    uint8_t *m = c.mask(a[4]);
    void *y = c.tok(a[5]);
    float *z = c.z(a[6]), *le = c.le(a[7]), *ld = c.ld(a[8]);
    const Workspace w(a[9]);
    flare_stream_t st = stream_of(a[10]);
    check_status(unlocked([&] { return lib.forward(c.d, q, k, v, m, y, z, le, ld, w.p, w.n, st); }), "flare_forward");
BINDING_END

// desc, Q, K, V, key_mask, Y, dY, Z, lse_enc, lse_dec, dQ, dK, dV, workspace, stream
BINDING(backward, 15)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *q = c.q(a[1]), *k = c.tok(a[2]), *v = c.tok(a[3]);
    uint8_t *m = c.mask(a[4]);
    void *y = c.tok(a[5]), *dy = c.tok(a[6]);
    float *z = c.z(a[7]), *le = c.le(a[8]), *ld = c.ld(a[9]), *dq = c.dq(a[10]);
    void *dk = c.tok(a[11]), *dv = c.tok(a[12]);
    const Workspace w(a[13]);
    flare_stream_t st = stream_of(a[14]);
    check_status(unlocked([&] { return lib.backward(c.d, q, k, v, m, y, dy, z, le, ld, dq, dk, dv, w.p, w.n, st); }), "flare_backward");
BINDING_END

// desc, hQ, hK, hV, hmask, hY, dQ, dK, dV, dmask, dY, workspace, stream
BINDING(forward_host, 13)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *hq = c.q(a[1], false, false), *hk = c.tok(a[2], false), *hv = c.tok(a[3], false);
    uint8_t *hm = c.mask(a[4], false);
    void *hy = c.tok(a[5], false), *q = c.q(a[6]), *k = c.tok(a[7]), *v = c.tok(a[8]);
    uint8_t *m = c.mask(a[9]);
    void *y = c.tok(a[10]);
    const Workspace w(a[11]);
    flare_stream_t st = stream_of(a[12]);
    check_status(unlocked([&] { return lib.forward_host(c.d, hq, hk, hv, hm, hy, q, k, v, m, y, w.p, w.n, st); }), "flare_forward_host");
BINDING_END

// desc, shared, Q_enc, Q_dec, K, V, key_mask, Y, Z, lse_enc, lse_dec, workspace, stream
BINDING(forward_variant, 13)
    Desc desc(a[0]);
    const int shared = PyObject_IsTrue(a[1]);
    const Call c{desc.get(), tensor(a[4]).scalar_type()};
    void *qe = c.q(a[2], shared), *qd = c.q(a[3], shared), *k = c.tok(a[4]), *v = c.tok(a[5]);
    uint8_t *m = c.mask(a[6]);
    void *y = c.tok(a[7]);
    float *z = c.z(a[8]), *le = c.le(a[9]), *ld = c.ld(a[10]);
    const Workspace w(a[11]);
    flare_stream_t st = stream_of(a[12]);
    check_status(unlocked([&] { return lib.forward_variant(c.d, shared, qe, qd, k, v, m, y, z, le, ld, w.p, w.n, st); }), "flare_forward_variant");
BINDING_END

// desc, shared, Q_enc, Q_dec, K, V, key_mask, Y, dY, Z, lse_enc, lse_dec, dQ_enc, dQ_dec, dK, dV, workspace, stream
BINDING(backward_variant, 18)
    Desc desc(a[0]);
    const int shared = PyObject_IsTrue(a[1]);
    const Call c{desc.get(), tensor(a[4]).scalar_type()};
    void *qe = c.q(a[2], shared), *qd = c.q(a[3], shared), *k = c.tok(a[4]), *v = c.tok(a[5]);
    uint8_t *m = c.mask(a[6]);
    void *y = c.tok(a[7]), *dy = c.tok(a[8]);
    float *z = c.z(a[9]), *le = c.le(a[10]), *ld = c.ld(a[11]), *dqe = c.dq(a[12], shared), *dqd = c.dq(a[13], shared);
    void *dk = c.tok(a[14]), *dv = c.tok(a[15]);
    const Workspace w(a[16]);
    flare_stream_t st = stream_of(a[17]);
    check_status(unlocked([&] { return lib.backward_variant(c.d, shared, qe, qd, k, v, m, y, dy, z, le, ld, dqe, dqd, dk, dv, w.p, w.n, st); }),
                 "flare_backward_variant");
BINDING_END

// desc, Q, K, lse_enc, lse_dec, G, workspace, stream
BINDING(spectral_gram, 8)
    Desc desc(a[0]);
    const Call c{desc.get(), tensor(a[2]).scalar_type()};
    void *q = c.q(a[1]), *k = c.tok(a[2]);
    float *le = c.le(a[3]), *ld = c.ld(a[4]);
    float *g = (float *)c.ptr(a[5], at::kFloat, {c.d->B, c.d->H, c.d->M, c.d->M});
    const Workspace w(a[6]);
    flare_stream_t st = stream_of(a[7]);
    check_status(unlocked([&] { return lib.spectral_gram(c.d, q, k, le, ld, g, w.p, w.n, st); }), "flare_spectral_gram");
BINDING_END

// A Python float, or any number that converts to one.
double number(PyObject *o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw PythonError{};
    return x;
}

// ---- the convenience calls: descriptor from the tensors, outputs and scratch allocated here

flare_desc_t make_desc(const at::Tensor &Q, const at::Tensor &K, double scale) {
    if (Q.dim() != 3 || K.dim() != 4) fail(PyExc_ValueError, "expected Q_lat [H,M,D] and K [B,N,H,D]");
    if (K.size(2) != Q.size(0) || K.size(3) != Q.size(2)) fail(PyExc_ValueError, "Q_lat [H,M,D] and K [B,N,H,D] disagree");
    int dtype;
    switch (K.scalar_type()) {
        case at::kFloat: dtype = FLARE_DTYPE_F32; break;
        case at::kBFloat16: dtype = FLARE_DTYPE_BF16; break;
        case at::kHalf: dtype = FLARE_DTYPE_F16; break;
        default: fail(PyExc_TypeError, "unsupported dtype " + dtype_name(K.scalar_type()));
    }
    return flare_desc_t{(int32_t)K.size(0), (int32_t)K.size(2), (int32_t)K.size(1), (int32_t)Q.size(1), (int32_t)K.size(3), dtype, (float)scale};
}
size_t workspace_bytes(const flare_desc_t &d, int op) {
    const size_t n = lib.workspace_bytes(&d, op);
    if (n == 0) check_status(FLARE_ERR_UNSUPPORTED, "flare_workspace_bytes");
    return n;
}
size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Scratch that is dropped when the call returns, with its kernels still queued: allocated on the stream it is used on (none given: the
// current one), so that nothing of another stream takes its place before they have run, or is still at work on it when they start.
at::Tensor scratch(size_t bytes, const at::Tensor &like, PyObject *stream, flare_stream_t st) {
    c10::cuda::OptionalCUDAStreamGuard guard;
    if (stream != Py_None) guard.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)st, like.device().index()));
    return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}

// What a call returns comes from its stream's memory as well: of the current stream's, what has just been given back may still be in use by work that is
// queued there, and what the caller drops would be handed on with the call's kernels still writing.  The current stream is known to use it too: where a
// result is dropped, its memory is not handed on before what that has queued by then is done.
at::Tensor result(at::IntArrayRef shape, const at::TensorOptions &options, PyObject *stream, flare_stream_t st) {
    if (stream == Py_None) return at::empty(shape, options);
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(options.device().index());
    if ((cudaStream_t)st == current.stream()) return at::empty(shape, options);
    const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal((cudaStream_t)st, options.device().index()));
    at::Tensor t = at::empty(shape, options);
    t.record_stream(current);
    return t;
}

// Q, K, V, key_mask, scale, want_stats, stream -> Y, or (Y, Z, lse_enc, lse_dec)
BINDING(call_forward, 7)
    const at::Tensor &Q = tensor(a[0]), &K = tensor(a[1]);
    const flare_desc_t d = make_desc(Q, K, number(a[4]));
    const Call c{&d, K.scalar_type()};
    void *q = c.q(a[0]), *k = c.tok(a[1]), *v = c.tok(a[2]);
    uint8_t *m = c.mask(a[3]);
    const bool stats = PyObject_IsTrue(a[5]) == 1;
    flare_stream_t st = stream_of(a[6]);
    const size_t ws = workspace_bytes(d, FLARE_OP_FORWARD);
    const at::Tensor Y = result({d.B, d.N, d.H, d.D}, K.options(), a[6], st);
    const auto f32 = K.options().dtype(at::kFloat);
    if (stats) {
        const at::Tensor Z = result({d.B, d.H, d.M, d.D}, f32, a[6], st), le = result({d.B, d.H, d.M}, f32, a[6], st), ld = result({d.B, d.N, d.H}, f32, a[6], st);
        const at::Tensor w = scratch(ws, K, a[6], st);
        check_status(unlocked([&] { return lib.forward(&d, q, k, v, m, Y.data_ptr(), (float *)Z.data_ptr(), (float *)le.data_ptr(),
                                                       (float *)ld.data_ptr(), w.data_ptr(), ws, st); }), "flare_forward");
        return Py_BuildValue("(NNNN)", THPVariable_Wrap(Y), THPVariable_Wrap(Z), THPVariable_Wrap(le), THPVariable_Wrap(ld));
    }
    // Z lives in the workspace, the statistics (asked for: the encode weights are then as accurate as in training) behind it
    const size_t le_at = round256(ws), ld_at = round256(le_at + 4 * (size_t)d.B * d.H * d.M), total = ld_at + 4 * (size_t)d.B * d.N * d.H;
    const at::Tensor w = scratch(total, K, a[6], st);
    char *base = (char *)w.data_ptr();
    check_status(unlocked([&] { return lib.forward(&d, q, k, v, m, Y.data_ptr(), nullptr, (float *)(base + le_at), (float *)(base + ld_at), base, ws, st); }),
                 "flare_forward");
    return THPVariable_Wrap(Y);
BINDING_END

// Q, K, V, dY, key_mask, scale, stream -> (Y, dQ, dK, dV, workspace: the forward's, and from byte 256 on the backward's)
BINDING(call_forward_backward, 7)
    const at::Tensor &Q = tensor(a[0]), &K = tensor(a[1]);
    const flare_desc_t d = make_desc(Q, K, number(a[5]));
    const Call c{&d, K.scalar_type()};
    void *q = c.q(a[0]), *k = c.tok(a[1]), *v = c.tok(a[2]), *dy = c.tok(a[3]);
    uint8_t *m = c.mask(a[4]);
    flare_stream_t st = stream_of(a[6]);
    // one workspace: the backward starts when the forward is done with it.  But for the header, which keeps what the forward reports: the
    // backward has its own behind it.
    const size_t fwd_bytes = workspace_bytes(d, FLARE_OP_FORWARD), bwd_bytes = workspace_bytes(d, FLARE_OP_BACKWARD), bwd_at = 256;
    const size_t ws = std::max(fwd_bytes, bwd_at + bwd_bytes);
    const at::Tensor Y = result({d.B, d.N, d.H, d.D}, K.options(), a[6], st), dK = result({d.B, d.N, d.H, d.D}, K.options(), a[6], st);
    const at::Tensor dV = result({d.B, d.N, d.H, d.D}, K.options(), a[6], st), dQ = result({d.H, d.M, d.D}, K.options().dtype(at::kFloat), a[6], st);
    const size_t z_at = round256(ws), le_at = round256(z_at + 4 * (size_t)d.B * d.H * d.M * d.D), ld_at = round256(le_at + 4 * (size_t)d.B * d.H * d.M);
    const at::Tensor w = scratch(ld_at + 4 * (size_t)d.B * d.N * d.H, K, a[6], st);
    char *base = (char *)w.data_ptr();
    float *z = (float *)(base + z_at), *le = (float *)(base + le_at), *ld = (float *)(base + ld_at);
    check_status(unlocked([&] { return lib.forward(&d, q, k, v, m, Y.data_ptr(), z, le, ld, base, fwd_bytes, st); }), "flare_forward");
    check_status(unlocked([&] { return lib.backward(&d, q, k, v, m, Y.data_ptr(), dy, z, le, ld, (float *)dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(),
                                                    base + bwd_at, bwd_bytes, st); }), "flare_backward");
    return Py_BuildValue("(NNNNN)", THPVariable_Wrap(Y), THPVariable_Wrap(dQ), THPVariable_Wrap(dK), THPVariable_Wrap(dV), THPVariable_Wrap(w));
BINDING_END

// G, eigenvalues, U, sweeps, stream
BINDING(spectral_eig, 5)
    const at::Tensor &G = tensor(a[0]);
    const int64_t M = G.dim() > 0 ? G.size(-1) : 0;
    if (M < 1) fail(PyExc_ValueError, "expected matrices [..., M, M], got shape " + shape_text(G.sizes()));
    // (rows longer than the library takes are left to it to refuse: their square might not even be a number of elements)
    const int64_t matrices = M <= 1024 ? G.numel() / (M * M) : 0;
    const long sweeps = PyLong_AsLong(a[3]);
    if (sweeps == -1 && PyErr_Occurred()) throw PythonError{};
    // (the library is told sizes of G alone: what it writes must have room)
    auto ptr = [](PyObject *o, int64_t least) -> float * {
        if (o == Py_None) return nullptr;
        const at::Tensor &t = tensor(o);
        check(t, at::kFloat, t.sizes());
        if (t.numel() < least) fail(PyExc_ValueError, "expected at least " + std::to_string(least) + " elements, got shape " + shape_text(t.sizes()));
        return (float *)t.data_ptr();
    };
    float *g = ptr(a[0], 0), *ev = ptr(a[1], matrices * M), *u = ptr(a[2], matrices * M * M);
    flare_stream_t st = stream_of(a[4]);
    check_status(unlocked([&] { return lib.spectral_eig((int32_t)matrices, (int32_t)M, g, ev, u, (int32_t)sweeps, st); }), "flare_spectral_eig");
BINDING_END

// ---- around a block: tensors [..., width] whose leading dimensions are rows at one distance

int dtype_code(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return FLARE_DTYPE_F32;
        case at::kBFloat16: return FLARE_DTYPE_BF16;
        case at::kHalf: return FLARE_DTYPE_F16;
        default: fail(PyExc_TypeError, "unsupported dtype " + dtype_name(t));
    }
}
struct Rows {
    void *p = nullptr;
    int64_t stride = 0;
};
Rows rows_of(const at::Tensor &t, at::ScalarType dtype, at::IntArrayRef shape, const char *name) {
    if (!t.is_cuda()) fail(PyExc_ValueError, std::string(name) + ": expected a CUDA tensor");
    if (t.scalar_type() != dtype) fail(PyExc_TypeError, std::string(name) + ": expected " + dtype_name(dtype) + ", got " + dtype_name(t.scalar_type()));
    if (t.sizes() != shape) fail(PyExc_ValueError, std::string(name) + ": expected shape " + shape_text(shape) + ", got " + shape_text(t.sizes()));
    const int64_t n = t.dim(), C = t.size(n - 1);
    if (t.numel() == 0) return Rows{t.data_ptr(), C};
    int64_t stride = 0, rows = 1;                            // of the innermost leading dimension that has more than one entry
    bool ok = C == 1 || t.stride(n - 1) == 1;
    for (int64_t i = n - 2; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (stride == 0) stride = t.stride(i);
        else ok = ok && t.stride(i) == stride * rows;
        rows *= t.size(i);
    }
    if (stride == 0) stride = C;
    if (!ok || stride < C) fail(PyExc_ValueError, std::string(name) + ": expected rows of adjacent columns at one distance from each other");
    return Rows{t.data_ptr(), stride};
}
float *row_param(PyObject *o, int64_t C, const char *name) {
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || !t.is_contiguous()) fail(PyExc_ValueError, std::string(name) + ": expected a contiguous CUDA tensor");
    if (t.scalar_type() != at::kFloat) fail(PyExc_TypeError, std::string(name) + ": expected torch.float32, got " + dtype_name(t.scalar_type()));
    if (t.dim() != 1 || t.size(0) != C) fail(PyExc_ValueError, std::string(name) + ": expected shape (" + std::to_string(C) + ",), got " + shape_text(t.sizes()));
    return (float *)t.data_ptr();
}
// A Norm (kind, weight, bias, eps), or None: taken apart here, a call of Python's less.
struct NormArg {
    int kind = FLARE_NORM_NONE;
    float *weight = nullptr, *bias = nullptr;
    float eps = 0.f;
    NormArg(PyObject *o, int64_t C, const char *weight_name, const char *bias_name) {
        if (o == Py_None) return;
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) fail(PyExc_TypeError, "expected a Norm (kind, weight, bias, eps) or None");
        kind = kind_of(PyTuple_GET_ITEM(o, 0), {{"layer", FLARE_NORM_LAYER}, {"rms", FLARE_NORM_RMS}}, "norm");
        weight = row_param(PyTuple_GET_ITEM(o, 1), C, weight_name);
        bias = row_param(PyTuple_GET_ITEM(o, 2), C, bias_name);
        eps = (float)number(PyTuple_GET_ITEM(o, 3));
    }
    static int kind_of(PyObject *name, std::initializer_list<std::pair<const char *, int>> table, const char *what) {
        if (PyUnicode_Check(name))
            for (const auto &entry : table)
                if (PyUnicode_CompareWithASCIIString(name, entry.first) == 0) return entry.second;
        std::string text = std::string(what) + ": expected one of";
        for (const auto &entry : table) text += std::string(&entry == table.begin() ? " " : ", ") + entry.first;
        PyObject *repr = PyObject_Repr(name);
        if (repr) text += std::string(", got ") + PyUnicode_AsUTF8(repr);
        Py_XDECREF(repr);
        fail(PyExc_ValueError, text);
    }
};
int gate_kind_of(PyObject *gate, PyObject *kind) {
    if (gate == Py_None) return FLARE_GATE_NONE;
    return NormArg::kind_of(kind, {{"sigmoid", FLARE_GATE_SIGMOID}, {"linear", FLARE_GATE_LINEAR}}, "gate_kind");
}
// The tuple of results as an instance of a NamedTuple class.
PyObject *named(PyObject *cls, PyObject *values) {
    if (!values) throw PythonError{};
    PyObject *args = PyTuple_Pack(1, values);
    Py_DECREF(values);
    PyObject *r = args ? PyTuple_Type.tp_new((PyTypeObject *)cls, args, nullptr) : nullptr;
    Py_XDECREF(args);
    if (!r) throw PythonError{};
    return r;
}
int number_of(PyObject *o) {
    const long x = PyLong_AsLong(o);
    if (x == -1 && PyErr_Occurred()) throw PythonError{};
    return (int)std::max<long>(INT32_MIN, std::min<long>(x, INT32_MAX));      // (what is out of range stays so)
}
PyObject *wrap(const at::Tensor &t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject *wrap_all(std::initializer_list<at::Tensor> ts) {
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) throw PythonError{};
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) PyTuple_SET_ITEM(r, i++, wrap(t));
    return r;
}

// A tensor of the caller's that has been written: as after an operation in place, autograd tells a graph that still wants what it held.
void mark_written(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// The tensors to write to: a tuple with one, or None, for every result (or None), and where the others are allocated.
struct Outputs {
    PyObject *out, *stream;
    flare_stream_t st;
    at::Tensor given(Py_ssize_t i) const {
        if (out == Py_None) return at::Tensor();
        if (!PyTuple_Check(out) || i >= PyTuple_GET_SIZE(out)) fail(PyExc_ValueError, "out: expected a tuple with a tensor, or None, for every result");
        PyObject *o = PyTuple_GET_ITEM(out, i);
        return o != Py_None ? tensor(o) : at::Tensor();
    }
    at::Tensor operator()(Py_ssize_t i, at::IntArrayRef shape, const at::TensorOptions &options) const {
        const at::Tensor t = given(i);
        return t.defined() ? t : result(shape, options, stream, st);
    }
    // The call's results in the order of the tuple, once it has been made: those of them that were given have been written.
    PyObject *wrapped(std::initializer_list<at::Tensor> results) const {
        Py_ssize_t i = 0;
        for (const at::Tensor &t : results) {
            if (t.defined() && given(i).defined()) mark_written(t);
            ++i;
        }
        return wrap_all(results);
    }
    at::Tensor sums(const float *present, Py_ssize_t i, int64_t C, const at::TensorOptions &f32) const { return present ? (*this)(i, {C}, f32) : at::Tensor(); }
    // statistics of the rows, where they are wanted
    at::Tensor stats(PyObject *want, Py_ssize_t i, int64_t rows, const at::TensorOptions &f32) const {
        const int yes = PyObject_IsTrue(want);
        if (yes < 0) throw PythonError{};
        if (yes) return (*this)(i, {rows, 4}, f32);
        if (given(i).defined()) fail(PyExc_ValueError, "stats: a tensor to write to, but want_stats is false");
        return at::Tensor();
    }
};

// What a call says about its rows: shape, types and norms.
struct Around {
    flare_block_desc_t d{};
    std::vector<int64_t> shape;
    int64_t C = 0;
    at::ScalarType dt, res;
    at::TensorOptions options;
    Around(const at::Tensor &stream_like, const at::Tensor &branch_like) : dt(branch_like.scalar_type()), res(stream_like.scalar_type()), options(stream_like.options()) {
        init(stream_like.sizes());
    }
    Around(const at::Tensor &x, at::ScalarType h) : dt(h), res(x.scalar_type()), options(x.options()) { init(x.sizes()); }
    void init(at::IntArrayRef s) {
        if (s.size() < 1) fail(PyExc_ValueError, "expected tensors [..., width]");
        shape = s.vec();
        C = shape.back();
        if (C < 1 || C > INT32_MAX) fail(PyExc_ValueError, "expected tensors [..., width], got shape " + shape_text(s));
        d.rows = 1;
        for (size_t i = 0; i + 1 < shape.size(); ++i) d.rows *= shape[i];
        d.width = (int32_t)C;
        d.dtype = dtype_code(dt);
        d.residual_dtype = dtype_code(res);
        d.residual_scale = 1.f;
    }
    Rows rows(PyObject *o, at::ScalarType t, int64_t &stride, const char *name) const {
        if (o == Py_None) return Rows{};
        const Rows r = rows_of(tensor(o), t, shape, name);
        stride = r.stride;
        return r;
    }
    Rows rows(const at::Tensor &o, int64_t &stride, const char *name, at::ScalarType t) const {
        const Rows r = rows_of(o, t, shape, name);
        stride = r.stride;
        return r;
    }
    // the gate: one row per row, or, with fewer leading entries, per group of consecutive rows
    std::vector<int64_t> gate_shape;
    Rows gate(PyObject *o, int kind) {
        d.gate = kind;
        d.gate_rows = 1;
        if ((o == Py_None) != (kind == FLARE_GATE_NONE)) fail(PyExc_ValueError, "gate: a tensor and its kind go together");
        if (o == Py_None) return Rows{};
        const at::Tensor &g = tensor(o);
        gate_shape = g.sizes().vec();
        int64_t n = 1;
        for (size_t i = 0; i + 1 < gate_shape.size(); ++i) n *= gate_shape[i];
        const bool leads = !gate_shape.empty() && gate_shape.back() == C && gate_shape.size() <= shape.size() &&
                           std::equal(gate_shape.begin(), gate_shape.end() - 1, shape.begin());
        if (!leads) fail(PyExc_ValueError, "gate: expected [..., width] with the leading dimensions of the branch, or the first of them, got shape " + shape_text(gate_shape));
        if (d.rows > 0) d.gate_rows = d.rows / n;            // (no rows: there may be gate rows all the same, of items without any)
        const Rows r = rows_of(g, dt, gate_shape, "gate");
        d.stride_gate = r.stride;
        return r;
    }
    float *stats(const at::Tensor &t) const {
        if (!t.defined()) return nullptr;
        check(t, at::kFloat, {d.rows, 4});
        return (float *)t.data_ptr();
    }
    at::TensorOptions as(at::ScalarType t) const { return options.dtype(t); }
};

float *sums_ptr(const at::Tensor &t, int64_t C) {
    if (!t.defined()) return nullptr;
    check(t, at::kFloat, {C});
    return (float *)t.data_ptr();
}

// x, norm, dtype or None, whether statistics are wanted, out (h, stats) or None, stream -> (h, stats)
BINDING(block_norm, 6)
    const at::Tensor &x = tensor(a[0]);
    if (a[2] != Py_None && !THPDtype_Check(a[2])) fail(PyExc_TypeError, "dtype: expected a torch dtype");
    Around c(x, a[2] == Py_None ? x.scalar_type() : ((THPDtype *)a[2])->scalar_type);
    const NormArg n(a[1], c.C, "weight", "bias");
    c.d.pre_norm = n.kind;
    c.d.pre_eps = n.eps;
    const Rows rx = c.rows(x, c.d.stride_x, "x", c.res);
    flare_stream_t st = stream_of(a[5]);
    const Outputs output{a[4], a[5], st};
    const at::Tensor h = output(0, c.shape, c.as(c.dt)), stats = output.stats(a[3], 1, c.d.rows, c.as(at::kFloat));
    const Rows rh = c.rows(h, c.d.stride_h, "h", c.dt);
    float *ps = c.stats(stats);
    check_status(unlocked([&] { return lib.norm_forward(&c.d, rx.p, n.weight, n.bias, rh.p, ps, st); }), "flare_norm_forward");
    return output.wrapped({h, stats});
BINDING_END

// x, stats, dh, dy, norm, out (dx, dweight, dbias) or None, stream, class of the result -> (dx, dweight, dbias)
BINDING(block_norm_backward, 8)
    const at::Tensor &x = tensor(a[0]), &dh = tensor(a[2]);
    Around c(x, dh);
    const NormArg n(a[4], c.C, "weight", "bias");
    c.d.pre_norm = n.kind;
    c.d.pre_eps = n.eps;
    const Rows rx = c.rows(x, c.d.stride_x, "x", c.res), rdh = c.rows(dh, c.d.stride_dh, "dh", c.dt), rdy = c.rows(a[3], c.res, c.d.stride_dy, "dy");
    const float *ps = c.stats(tensor(a[1]));
    const auto f32 = c.as(at::kFloat);
    flare_stream_t st = stream_of(a[6]);
    const Outputs output{a[5], a[6], st};
    const at::Tensor dx = output(0, c.shape, c.as(c.res)), dw = output.sums(n.weight, 1, c.C, f32), db = output.sums(n.bias, 2, c.C, f32);
    const Rows rdx = c.rows(dx, c.d.stride_dx, "dx", c.res);
    float *pw = sums_ptr(dw, c.C), *pb = sums_ptr(db, c.C);
    const size_t need = lib.block_workspace_bytes(&c.d);
    if (need == 0) check_status(FLARE_ERR_UNSUPPORTED, "flare_norm_backward");
    const at::Tensor ws = scratch(need, x, a[6], st);
    check_status(unlocked([&] { return lib.norm_backward(&c.d, rx.p, n.weight, ps, rdy.p, rdh.p, rdx.p, pw, pb, ws.data_ptr(), need, st); }), "flare_norm_backward");
    return named(a[7], output.wrapped({dx, dw, db}));
BINDING_END

// x, branch, post, pre, gate, gate kind, scale, residual scale, whether statistics are wanted, out (y, h, stats) or None, stream -> (y, h, stats)
BINDING(block_join, 11)
    const at::Tensor &x = tensor(a[0]), &o = tensor(a[1]);
    Around c(x, o);
    const NormArg post(a[2], c.C, "post weight", "post bias"), pre(a[3], c.C, "pre weight", "pre bias");
    c.d.post_norm = post.kind; c.d.post_eps = post.eps;
    c.d.pre_norm = pre.kind; c.d.pre_eps = pre.eps;
    c.d.residual_scale = (float)number(a[7]);
    const float *s = row_param(a[6], c.C, "scale");
    const Rows rx = c.rows(x, c.d.stride_x, "x", c.res), ro = c.rows(o, c.d.stride_branch, "branch", c.dt), rg = c.gate(a[4], gate_kind_of(a[4], a[5]));
    const bool next = pre.kind != FLARE_NORM_NONE;
    flare_stream_t st = stream_of(a[10]);
    const Outputs output{a[9], a[10], st};
    const at::Tensor y = output(0, c.shape, c.as(c.res)), h = next ? output(1, c.shape, c.as(c.dt)) : at::Tensor(),
                     stats = output.stats(a[8], 2, c.d.rows, c.as(at::kFloat));
    const Rows ry = c.rows(y, c.d.stride_y, "y", c.res), rh = next ? c.rows(h, c.d.stride_h, "h", c.dt) : Rows{};
    float *ps = c.stats(stats);
    check_status(unlocked([&] { return lib.join_forward(&c.d, rx.p, ro.p, rg.p, s, post.weight, post.bias, pre.weight, pre.bias, ry.p, rh.p, ps, st); }),
                 "flare_join_forward");
    return output.wrapped({y, h, stats});
BINDING_END

// branch, y, stats, dy, dh, post, pre, gate, gate kind, scale, residual scale, out or None, stream, class of the result
// -> (dx, dbranch, dgate, dscale, dpost_weight, dpost_bias, dpre_weight, dpre_bias)
BINDING(block_join_backward, 14)
    const at::Tensor &o = tensor(a[0]), &y = tensor(a[1]);
    Around c(y, o);
    const NormArg post(a[5], c.C, "post weight", "post bias"), pre(a[6], c.C, "pre weight", "pre bias");
    c.d.post_norm = post.kind; c.d.post_eps = post.eps;
    c.d.pre_norm = pre.kind; c.d.pre_eps = pre.eps;
    c.d.residual_scale = (float)number(a[10]);
    const float *s = row_param(a[9], c.C, "scale");
    const Rows ro = c.rows(o, c.d.stride_branch, "branch", c.dt), ry = c.rows(y, c.d.stride_x, "y", c.res), rdy = c.rows(a[3], c.res, c.d.stride_dy, "dy"),
               rdh = c.rows(a[4], c.dt, c.d.stride_dh, "dh"), rg = c.gate(a[7], gate_kind_of(a[7], a[8]));
    const float *ps = c.stats(tensor(a[2]));
    const auto f32 = c.as(at::kFloat);
    flare_stream_t st = stream_of(a[12]);
    const Outputs output{a[11], a[12], st};
    const at::Tensor dx = output(0, c.shape, c.as(c.res)), d_o = output(1, c.shape, c.as(c.dt));
    const at::Tensor dg = a[7] != Py_None ? output(2, c.gate_shape, c.as(c.dt)) : at::Tensor();
    const at::Tensor ds = output.sums(s, 3, c.C, f32), dwo = output.sums(post.weight, 4, c.C, f32), dbo = output.sums(post.bias, 5, c.C, f32),
                     dwy = output.sums(pre.weight, 6, c.C, f32), dby = output.sums(pre.bias, 7, c.C, f32);
    const Rows rdx = c.rows(dx, c.d.stride_dx, "dx", c.res), rdo = c.rows(d_o, c.d.stride_dbranch, "dbranch", c.dt);
    Rows rdg;
    if (dg.defined()) {
        rdg = rows_of(dg, c.dt, c.gate_shape, "dgate");
        c.d.stride_dgate = rdg.stride;
        if (c.d.rows == 0 && dg.numel() > 0) {               // gate rows without rows: the library knows of none, and theirs are sums of nothing
            c10::cuda::OptionalCUDAStreamGuard guard;
            if (a[12] != Py_None) guard.reset_stream(c10::cuda::getStreamFromExternal((cudaStream_t)st, y.device().index()));
            dg.zero_();
        }
    }
    float *p3 = sums_ptr(ds, c.C), *p4 = sums_ptr(dwo, c.C), *p5 = sums_ptr(dbo, c.C), *p6 = sums_ptr(dwy, c.C), *p7 = sums_ptr(dby, c.C);
    const size_t need = lib.block_workspace_bytes(&c.d);
    if (need == 0) check_status(FLARE_ERR_UNSUPPORTED, "flare_join_backward");
    const at::Tensor ws = scratch(need, y, a[12], st);
    check_status(unlocked([&] { return lib.join_backward(&c.d, ro.p, rg.p, s, post.weight, post.bias, ry.p, pre.weight, ps, rdy.p, rdh.p, rdx.p, rdo.p, rdg.p, p3,
                                                         p4, p5, p6, p7, ws.data_ptr(), need, st); }), "flare_join_backward");
    return named(a[13], output.wrapped({dx, d_o, dg, ds, dwo, dbo, dwy, dby}));
BINDING_END

// ---- orthogonalised updates

// Matrices [..., rows, cols]: the columns next to each other, rows at one distance, matrices at one distance.
struct Matrices {
    flare_orth_desc_t d{};
    std::vector<int64_t> shape;
    Matrices(const at::Tensor &g, PyObject *steps, PyObject *ca, PyObject *cb, PyObject *cc, PyObject *eps) {
        shape = g.sizes().vec();
        if (shape.size() < 2) fail(PyExc_ValueError, "expected matrices [..., rows, cols], got shape " + shape_text(shape));
        const int64_t rows = shape[shape.size() - 2], cols = shape.back();
        int64_t count = 1;
        for (size_t i = 0; i + 2 < shape.size(); ++i) count *= shape[i];
        if (rows > INT32_MAX || cols > INT32_MAX || count > INT32_MAX) fail(PyExc_ValueError, "matrices out of range: shape " + shape_text(shape));
        d.count = (int32_t)count; d.rows = (int32_t)rows; d.cols = (int32_t)cols;
        d.dtype = d.weight_dtype = dtype_code(g.scalar_type());
        d.steps = number_of(steps);
        d.coefficients[0] = (float)number(ca); d.coefficients[1] = (float)number(cb); d.coefficients[2] = (float)number(cc);
        d.eps = (float)number(eps);
    }
    // pointer, and the strides into row, matrix
    void *strided(const at::Tensor &t, at::ScalarType dtype, const char *name, int64_t &row, int64_t &matrix) const {
        if (!t.is_cuda()) fail(PyExc_ValueError, std::string(name) + ": expected a CUDA tensor");
        if (t.scalar_type() != dtype) fail(PyExc_TypeError, std::string(name) + ": expected " + dtype_name(dtype) + ", got " + dtype_name(t.scalar_type()));
        if (t.sizes() != at::IntArrayRef(shape)) fail(PyExc_ValueError, std::string(name) + ": expected shape " + shape_text(shape) + ", got " + shape_text(t.sizes()));
        const int64_t n = t.dim();
        bool ok = t.size(n - 1) <= 1 || t.stride(n - 1) == 1;
        row = t.size(n - 2) > 1 ? t.stride(n - 2) : t.size(n - 1);
        int64_t at = 0, many = 1;
        for (int64_t i = n - 3; i >= 0; --i) {
            if (t.size(i) == 1) continue;
            if (at == 0) at = t.stride(i);
            else ok = ok && t.stride(i) == at * many;
            many *= t.size(i);
        }
        matrix = at;
        if (t.numel() > 0 && (!ok || row < t.size(n - 1) || (many > 1 && at < 1)))
            fail(PyExc_ValueError, std::string(name) + ": expected matrices of adjacent columns, rows and matrices each at one distance");
        if (t.numel() == 0) row = matrix = 0;
        return t.data_ptr();
    }
    size_t need(const char *where) const {
        const size_t n = lib.orthogonalize_workspace_bytes(&d);
        if (n == 0) check_status(d.count < 0 || d.rows < 1 || d.cols < 1 || d.steps < 1 ? FLARE_ERR_INVALID_ARG : FLARE_ERR_UNSUPPORTED, where);
        return n;
    }
};

// G, steps, a, b, c, eps, out or None, stream -> (O, workspace)
BINDING(orthogonalize, 8)
    const at::Tensor &G = tensor(a[0]);
    Matrices c(G, a[1], a[2], a[3], a[4], a[5]);
    void *g = c.strided(G, G.scalar_type(), "G", c.d.stride_row, c.d.stride_matrix);
    flare_stream_t st = stream_of(a[7]);
    const at::Tensor O = a[6] == Py_None ? result(c.shape, G.options(), a[7], st) : tensor(a[6]);
    void *o = c.strided(O, G.scalar_type(), "out", c.d.out_stride_row, c.d.out_stride_matrix);
    const size_t need = c.need("flare_orthogonalize");
    const at::Tensor ws = scratch(need, G, a[7], st);
    check_status(unlocked([&] { return lib.orthogonalize(&c.d, g, o, ws.data_ptr(), need, st); }), "flare_orthogonalize");
    if (a[6] != Py_None) mark_written(O);
    return wrap_all({O, ws});
BINDING_END

// w, m, g, lr, momentum, weight decay, update scale, nesterov, steps, a, b, c, eps, w_out, m_out (or None: in place), stream -> (w_out, m_out, workspace)
BINDING(muon_update, 16)
    const at::Tensor &w = tensor(a[0]), &m = tensor(a[1]), &g = tensor(a[2]);
    Matrices c(g, a[8], a[9], a[10], a[11], a[12]);
    void *pg = c.strided(g, g.scalar_type(), "g", c.d.stride_row, c.d.stride_matrix);
    const at::Tensor &w_out = a[13] == Py_None ? w : tensor(a[13]), &m_out = a[14] == Py_None ? m : tensor(a[14]);
    c.d.weight_dtype = dtype_code(w.scalar_type());
    check(w, w.scalar_type(), c.shape); check(w_out, w.scalar_type(), c.shape); check(m, at::kFloat, c.shape); check(m_out, at::kFloat, c.shape);
    const flare_muon_t rule{(float)number(a[3]), (float)number(a[4]), (float)number(a[5]), (float)number(a[6]), PyObject_IsTrue(a[7]) == 1};
    flare_stream_t st = stream_of(a[15]);
    const size_t need = c.need("flare_muon_update");
    const at::Tensor ws = scratch(need, w, a[15], st);
    check_status(unlocked([&] { return lib.muon_update(&c.d, &rule, w.data_ptr(), (const float *)m.data_ptr(), pg, w_out.data_ptr(), (float *)m_out.data_ptr(),
                                                       ws.data_ptr(), need, st); }), "flare_muon_update");
    mark_written(w_out);
    mark_written(m_out);
    return wrap_all({w_out, m_out, ws});
BINDING_END

// bind(addresses: dict name -> int, FlareError)
BINDING(bind, 2)
    auto get = [&](const char *name, auto &slot) {
        PyObject *o = PyDict_GetItemString(a[0], name);
        if (!o) fail(PyExc_KeyError, name);
        slot = (std::remove_reference_t<decltype(slot)>)PyLong_AsVoidPtr(o);
    };
    get("flare_workspace_bytes", lib.workspace_bytes);
    get("flare_encode", lib.encode);
    get("flare_encode_static_scratch", lib.encode_static_scratch);
    get("flare_decode", lib.decode);
    get("flare_forward", lib.forward);
    get("flare_backward", lib.backward);
    get("flare_forward_host", lib.forward_host);
    get("flare_forward_variant", lib.forward_variant);
    get("flare_backward_variant", lib.backward_variant);
    get("flare_spectral_gram", lib.spectral_gram);
    get("flare_spectral_eig", lib.spectral_eig);
    get("flare_block_workspace_bytes", lib.block_workspace_bytes);
    get("flare_norm_forward", lib.norm_forward);
    get("flare_norm_backward", lib.norm_backward);
    get("flare_join_forward", lib.join_forward);
    get("flare_join_backward", lib.join_backward);
    get("flare_orthogonalize_workspace_bytes", lib.orthogonalize_workspace_bytes);
    get("flare_orthogonalize", lib.orthogonalize);
    get("flare_muon_update", lib.muon_update);
    Py_INCREF(a[1]);
    flare_error = a[1];
BINDING_END

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(encode), METHOD(encode_static_scratch), METHOD(decode), METHOD(forward), METHOD(backward),
                         METHOD(forward_host), METHOD(forward_variant), METHOD(backward_variant), METHOD(spectral_gram), METHOD(spectral_eig),
                         METHOD(call_forward), METHOD(call_forward_backward), METHOD(block_norm), METHOD(block_norm_backward), METHOD(block_join),
                         METHOD(block_join_backward), METHOD(orthogonalize), METHOD(muon_update), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_binding", "Argument marshalling for libflare.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module_def); }
