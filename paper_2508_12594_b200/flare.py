"""Python binding of libflare: the same entry points as ``include/flare.h``, argument marshalling only.

Every step of the mixer runs in the library's CUDA kernels.  PyTorch is used for device memory and streams:
the functions take torch tensors, check layout and dtype, and pass raw pointers (in ``csrc/flare_binding.cpp``, an extension
module, for the calls that enqueue work; through ctypes for the rest).  There is no CPU fallback: if ``libflare.so`` or
the extension is missing or cannot be loaded the first call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflare.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_ARCH, ERR_CUDA, ERR_TIMEOUT = range(7)
DTYPE_F32, DTYPE_BF16, DTYPE_F16 = 0, 1, 2
OP_ENCODE, OP_DECODE, OP_FORWARD, OP_BACKWARD, OP_SPECTRAL = range(5)


class FlareDesc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("N", ctypes.c_int32), ("M", ctypes.c_int32),
                ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class FlareBlockDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int32), ("dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32),
                ("pre_norm", ctypes.c_int32), ("post_norm", ctypes.c_int32), ("gate", ctypes.c_int32), ("gate_rows", ctypes.c_int64),
                ("pre_eps", ctypes.c_float), ("post_eps", ctypes.c_float), ("residual_scale", ctypes.c_float)] + [
                    (f"stride_{n}", ctypes.c_int64) for n in ("x", "branch", "gate", "y", "h", "dy", "dh", "dx", "dbranch", "dgate")]


class FlareOrthDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("count", "rows", "cols", "dtype", "weight_dtype", "steps")] + [
        ("coefficients", ctypes.c_float * 3), ("eps", ctypes.c_float)] + [
            (n, ctypes.c_int64) for n in ("stride_row", "stride_matrix", "out_stride_row", "out_stride_matrix")]


class FlareMuon(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("lr", "momentum", "weight_decay", "update_scale")] + [("nesterov", ctypes.c_int32)]


class FlareDrop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_float), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("step", ctypes.c_void_p)]


class FlareDropoutDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("width", "dtype", "residual_dtype")] + [
        (n, ctypes.c_int64) for n in ("stride_x", "stride_residual", "stride_y")]


class FlareEmbedDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "positions")] + [(n, ctypes.c_int32) for n in ("width", "vocab", "dtype", "out_dtype", "token_bits")] + [
        ("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in ("stride_table", "stride_out")]


class FlareLossDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("width", "vocab", "dtype", "label_bits")] + [
        (n, ctypes.c_float) for n in ("scale", "dloss_scale")] + [(n, ctypes.c_int64) for n in ("stride_x", "stride_w", "stride_dx", "stride_dw")]


class FlareError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = _lib_or_none()
        text = lib.flare_status_string(status).decode() if lib else str(status)
        detail = lib.flare_last_cuda_error().decode() if lib and status == ERR_CUDA else ""
        super().__init__(f"{where}: {text}" + (f" ({detail})" if detail else ""))
        self.status = status


_lib = None

_vp, _sz = ctypes.c_void_p, ctypes.c_size_t
_dp = ctypes.POINTER(FlareDesc)
_bp = ctypes.POINTER(FlareBlockDesc)
_op = ctypes.POINTER(FlareOrthDesc)
_SIGNATURES = {
    "flare_version": (ctypes.c_int, []),
    "flare_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "flare_last_cuda_error": (ctypes.c_char_p, []),
    "flare_workspace_bytes": (_sz, [_dp, ctypes.c_int]),
    "flare_encode_partials": (ctypes.c_int, [_dp]),
    "flare_encode": (ctypes.c_int, [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "flare_encode_static_scratch": (ctypes.c_int, [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "flare_decode": (ctypes.c_int, [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "flare_set_path": (ctypes.c_int, [ctypes.c_int]),
    "flare_forward": (ctypes.c_int, [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "flare_backward": (ctypes.c_int, [_dp] + [_vp] * 13 + [_sz, _vp]),
    "flare_forward_host": (ctypes.c_int, [_dp] + [_vp] * 11 + [_sz, _vp]),
    "flare_check": (ctypes.c_int, [_vp, _vp]),
    "flare_microbench": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, _vp, _sz, ctypes.POINTER(ctypes.c_double), _vp]),
    "flare_variant_workspace_bytes": (_sz, [_dp, ctypes.c_int, ctypes.c_int, ctypes.c_int]),
    "flare_forward_variant": (ctypes.c_int, [_dp, ctypes.c_int] + [_vp] * 10 + [_sz, _vp]),
    "flare_backward_variant": (ctypes.c_int, [_dp, ctypes.c_int] + [_vp] * 15 + [_sz, _vp]),
    "flare_spectral_gram": (ctypes.c_int, [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "flare_spectral_eig": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, _vp, _vp, _vp, ctypes.c_int32, _vp]),
    "flare_launch_count": (ctypes.c_int, [_dp, ctypes.c_int]),
    "flare_block_workspace_bytes": (_sz, [_bp]),
    "flare_norm_forward": (ctypes.c_int, [_bp] + [_vp] * 6),
    "flare_norm_backward": (ctypes.c_int, [_bp] + [_vp] * 9 + [_sz, _vp]),
    "flare_join_forward": (ctypes.c_int, [_bp] + [_vp] * 12),
    "flare_join_backward": (ctypes.c_int, [_bp] + [_vp] * 19 + [_sz, _vp]),
    "flare_orthogonalize_workspace_bytes": (_sz, [_op]),
    "flare_orthogonalize_plan": (ctypes.c_int, [_op, ctypes.POINTER(ctypes.c_int32)]),
    "flare_orthogonalize": (ctypes.c_int, [_op, _vp, _vp, _vp, _sz, _vp]),
    "flare_muon_update": (ctypes.c_int, [_op, ctypes.POINTER(FlareMuon)] + [_vp] * 6 + [_sz, _vp]),
    "flare_dropout_forward": (ctypes.c_int, [ctypes.POINTER(FlareDropoutDesc), ctypes.POINTER(FlareDrop)] + [_vp] * 4),
    "flare_dropout_backward": (ctypes.c_int, [ctypes.POINTER(FlareDropoutDesc), ctypes.POINTER(FlareDrop)] + [_vp] * 3),
    "flare_embed_forward": (ctypes.c_int, [ctypes.POINTER(FlareEmbedDesc), ctypes.POINTER(FlareDrop)] + [_vp] * 5),
    "flare_embed_workspace_bytes": (_sz, [ctypes.POINTER(FlareEmbedDesc)]),
    "flare_embed_backward": (ctypes.c_int, [ctypes.POINTER(FlareEmbedDesc), ctypes.POINTER(FlareDrop)] + [_vp] * 4 + [ctypes.c_int32, _vp, _sz, _vp]),
    "flare_loss_workspace_bytes": (_sz, [ctypes.POINTER(FlareLossDesc), ctypes.c_int32]),
    "flare_loss_forward": (ctypes.c_int, [ctypes.POINTER(FlareLossDesc)] + [_vp] * 6 + [_sz, _vp]),
    "flare_loss_backward": (ctypes.c_int, [ctypes.POINTER(FlareLossDesc)] + [_vp] * 8 + [_sz, _vp]),
    "flare_selftest_wait": (ctypes.c_int, [_vp, ctypes.c_uint64, _vp]),
    "flare_selftest_team": (ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_uint64, _vp]),
}


def _lib_or_none():
    return _lib


def load():
    """Load libflare.so (once).  Raises if the CUDA extension has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: build it with `python -m paper_2508_12594_b200.build`")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


_native = None


def _bind():
    """The marshalling extension, with the library's functions handed to it (once)."""
    global _native
    if _native is None:
        lib = load()
        from . import _binding
        _binding.bind({name: ctypes.cast(getattr(lib, name), _vp).value for name in _SIGNATURES}, FlareError)
        _native = _binding
    return _native


def exported_symbols():
    return list(_SIGNATURES)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return DTYPE_F32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    if t.dtype == torch.float16:
        return DTYPE_F16
    raise TypeError(f"unsupported dtype {t.dtype}")


def make_desc(Q: torch.Tensor, K: torch.Tensor, scale: float = 1.0) -> FlareDesc:
    H, M, D = Q.shape
    B, N, H2, D2 = K.shape
    if (H2, D2) != (H, D):
        raise ValueError("Q_lat [H,M,D] and K [B,N,H,D] disagree")
    return FlareDesc(B, H, N, M, D, _dtype_code(K), float(scale))


def _ptr(t: Optional[torch.Tensor], dtype=None, shape=None, cuda=True):
    if t is None:
        return None
    if cuda and not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream: Optional[torch.cuda.Stream]):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _raise(rc: int, where: str):
    if rc != OK:
        raise FlareError(rc, where)


def flare_version() -> int:
    return load().flare_version()


def flare_workspace_bytes(desc: FlareDesc, op: int) -> int:
    return int(load().flare_workspace_bytes(ctypes.byref(desc), op))


def flare_encode_partials(desc: FlareDesc) -> int:
    return int(load().flare_encode_partials(ctypes.byref(desc)))


def alloc_workspace(desc: FlareDesc, op: int, device="cuda") -> torch.Tensor:
    n = flare_workspace_bytes(desc, op)
    if n == 0:
        raise FlareError(ERR_UNSUPPORTED, "flare_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def flare_encode(desc, Q, K, V, key_mask, Z, lse_enc, workspace, stream=None):
    (_native or _bind()).encode(desc, Q, K, V, key_mask, Z, lse_enc, workspace, stream)


STATIC_SCRATCH_BYTES = 8 << 20


def flare_encode_static_scratch(desc, Q, K, V, key_mask, Z, lse_enc, stream=None):
    """flare_encode for callers that cannot allocate device memory: the partial results go to the library's
    built-in scratch array (STATIC_SCRATCH_BYTES, shared by all calls on the device, so calls must not overlap
    on the GPU).  Larger problems raise FlareError(ERR_WORKSPACE_TOO_SMALL)."""
    (_native or _bind()).encode_static_scratch(desc, Q, K, V, key_mask, Z, lse_enc, stream)


def flare_decode(desc, Q, K, Z, Y, lse_dec, workspace=None, stream=None):
    (_native or _bind()).decode(desc, Q, K, Z, Y, lse_dec, workspace, stream)


PATH_AUTO, PATH_EXACT, PATH_FAST = 0, 1, 2


def flare_set_path(path: int):
    """Which form of the bfloat16 forward kernels runs: PATH_AUTO, PATH_EXACT (running maximum) or PATH_FAST."""
    _raise(load().flare_set_path(int(path)), "flare_set_path")


def flare_forward(desc, Q, K, V, key_mask, Y, Z, lse_enc, lse_dec, workspace, stream=None):
    (_native or _bind()).forward(desc, Q, K, V, key_mask, Y, Z, lse_enc, lse_dec, workspace, stream)


def flare_backward(desc, Q, K, V, key_mask, Y, dY, Z, lse_enc, lse_dec, dQ, dK, dV, workspace, stream=None):
    (_native or _bind()).backward(desc, Q, K, V, key_mask, Y, dY, Z, lse_enc, lse_dec, dQ, dK, dV, workspace, stream)


def flare_forward_host(desc, hQ, hK, hV, hmask, hY, dQ, dK, dV, dmask, dY, workspace, stream=None):
    """Host tensors in, host tensor out; the device tensors are the caller's staging buffers."""
    (_native or _bind()).forward_host(desc, hQ, hK, hV, hmask, hY, dQ, dK, dV, dmask, dY, workspace, stream)


def flare_check(workspace, stream=None):
    """workspace=None checks the built-in scratch array of flare_encode_static_scratch."""
    _raise(load().flare_check(_ptr(workspace, torch.uint8), _stream(stream)), "flare_check")


def flare_launch_count(desc: FlareDesc, op: int) -> int:
    return int(load().flare_launch_count(ctypes.byref(desc), op))


def flare_selftest_wait(workspace, budget_ns: int, stream=None):
    _raise(load().flare_selftest_wait(_ptr(workspace, torch.uint8), int(budget_ns), _stream(stream)), "flare_selftest_wait")


def flare_selftest_team(workspace, gone: int, budget_ns: int, stream=None):
    _raise(load().flare_selftest_team(_ptr(workspace, torch.uint8), int(gone), int(budget_ns), _stream(stream)), "flare_selftest_team")


def flare_variant_workspace_bytes(desc, op, shared_latents, separate) -> int:
    return int(load().flare_variant_workspace_bytes(ctypes.byref(desc), op, int(shared_latents), int(separate)))


def flare_forward_variant(desc, shared_latents, Q_enc, Q_dec, K, V, key_mask, Y, Z, lse_enc, lse_dec, workspace, stream=None):
    """The mixer with one latent sequence for all heads (Q [M, D]) and / or separate decode queries (Q_dec, else None)."""
    (_native or _bind()).forward_variant(desc, shared_latents, Q_enc, Q_dec, K, V, key_mask, Y, Z, lse_enc, lse_dec, workspace, stream)


def flare_backward_variant(desc, shared_latents, Q_enc, Q_dec, K, V, key_mask, Y, dY, Z, lse_enc, lse_dec, dQ_enc, dQ_dec, dK,
                           dV, workspace, stream=None):
    (_native or _bind()).backward_variant(desc, shared_latents, Q_enc, Q_dec, K, V, key_mask, Y, dY, Z, lse_enc, lse_dec, dQ_enc,
                                          dQ_dec, dK, dV, workspace, stream)


def flare_microbench(which: int, iters: int = 20000, stream=None) -> float:
    """One of the library's instruction-level measurements (see include/flare.h)."""
    scratch = torch.empty(4096, dtype=torch.uint8, device="cuda")
    out = ctypes.c_double(0.0)
    _raise(load().flare_microbench(int(which), int(iters), _ptr(scratch, torch.uint8), scratch.numel(), ctypes.byref(out),
                                   _stream(stream)), "flare_microbench")
    return float(out.value)


def flare_spectral_gram(desc, Q, K, lse_enc, lse_dec, G, workspace, stream=None):
    (_native or _bind()).spectral_gram(desc, Q, K, lse_enc, lse_dec, G, workspace, stream)


def flare_spectral_eig(G, eigenvalues, U=None, sweeps=0, stream=None):
    """G [..., M, M] float32 (destroyed) -> eigenvalues [..., M] descending, U [..., M, M] eigenvectors as columns."""
    (_native or _bind()).spectral_eig(G, eigenvalues, U, int(sweeps), stream)


def forward(Q, K, V, key_mask=None, scale=1.0, want_stats=False, stream=None):
    """Convenience: allocate outputs and workspace with torch, call flare_forward, return Y (and Z, lse's)."""
    return (_native or _bind()).call_forward(Q, K, V, key_mask, scale, want_stats, stream)


def forward_backward(Q, K, V, dY, key_mask=None, scale=1.0, stream=None, check=False):
    """Convenience: flare_forward (keeping Z and the log-sum-exp rows) then flare_backward.
    Returns (Y, dQ_lat [H,M,D] float32, dK, dV).  With check=True the stream is synchronised and a device-side
    wait that gave up raises."""
    Y, dQ, dK, dV, ws = (_native or _bind()).call_forward_backward(Q, K, V, dY, key_mask, scale, stream)
    if check:
        (stream or torch.cuda.current_stream()).synchronize()
        flare_check(ws, stream)
        flare_check(ws[256:], stream)
    return Y, dQ, dK, dV


# ---- around a block: the norms before and after it, its gate and residual scale

NORM_NONE, NORM_LAYER, NORM_RMS = range(3)
GATE_NONE, GATE_SIGMOID, GATE_LINEAR = range(3)


class Norm(NamedTuple):
    """A norm over the last dimension: kind "layer" or "rms"; weight and bias float32 [width] or None (ones, zeros)."""
    kind: str
    weight: Optional[torch.Tensor] = None
    bias: Optional[torch.Tensor] = None
    eps: float = 1e-5


class NormGrads(NamedTuple):
    dx: torch.Tensor
    dweight: Optional[torch.Tensor]
    dbias: Optional[torch.Tensor]


class JoinGrads(NamedTuple):
    dx: torch.Tensor
    dbranch: torch.Tensor
    dgate: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]
    dpost_weight: Optional[torch.Tensor]
    dpost_bias: Optional[torch.Tensor]
    dpre_weight: Optional[torch.Tensor]
    dpre_bias: Optional[torch.Tensor]


def block_norm(x, norm: Norm, dtype=None, out=None, stream=None, want_stats=True):
    """The norm before a block.  x [..., width] -> (h [..., width] of `dtype` (x's), stats [rows, 4] float32, None
    without want_stats).  out: (h, stats) to write to, either None.  Results that are allocated here, and in the calls below, come
    from the memory of `stream`."""
    return (_native or _bind()).block_norm(x, norm, dtype, want_stats, out, stream)


def block_norm_backward(x, stats, dh, norm: Norm, dy=None, out=None, stream=None) -> NormGrads:
    """Gradients of block_norm; dy: what reaches x beside the norm.  Those of weights that are None are None.
    out: (dx, dweight, dbias) to write to, any None."""
    return (_native or _bind()).block_norm_backward(x, stats, dh, dy, norm, out, stream, NormGrads)


def block_join(x, branch, post: Optional[Norm] = None, pre: Optional[Norm] = None, gate=None, gate_kind="sigmoid", scale=None,
               residual_scale=1.0, out=None, stream=None, want_stats=True):
    """What follows a block, and the norm before the next one:
    y = residual_scale * x + scale * act(gate) * post(branch);  h = pre(y).  Returns (y, h or None, stats [rows, 4], or None without want_stats).

    x, branch [..., width]; gate like the branch, or with fewer of its leading dimensions (one row per batch item, say);
    gate_kind "sigmoid" or "linear"; scale float32 [width].  out: (y, h, stats) to write to, any None."""
    return (_native or _bind()).block_join(x, branch, post, pre, gate, gate_kind, scale, residual_scale, want_stats, out, stream)


def block_join_backward(branch, y, stats, dy, dh, post: Optional[Norm] = None, pre: Optional[Norm] = None, gate=None, gate_kind="sigmoid",
                        scale=None, residual_scale=1.0, out=None, stream=None) -> JoinGrads:
    """Gradients of block_join from its inputs, its y and its stats; dy may be None where there is a dh, dh goes
    with pre.  Gradients of what is None are None.  out: a tuple in the order of JoinGrads to write to, any None."""
    return (_native or _bind()).block_join_backward(branch, y, stats, dy, dh, post, pre, gate, gate_kind, scale, residual_scale, out, stream, JoinGrads)


# ---- orthogonalised updates of matrices

NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def orthogonalize(G, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7, out=None, stream=None, check=False):
    """G [..., rows, cols] -> the same after `steps` Newton-Schulz steps of the odd quintic `coefficients` on G / (|G|_F + eps): singular
    values near 1, singular vectors kept.  out: a tensor to write to (G itself is allowed).  With check=True the stream is synchronised
    and a device-side wait that gave up raises."""
    O, ws = (_native or _bind()).orthogonalize(G, steps, *coefficients, eps, out, stream)
    if check:
        (stream or torch.cuda.current_stream()).synchronize()
        flare_check(ws, stream)
    return O


ORTH_BLOCK, ORTH_TEAM, ORTH_PAIRS, ORTH_CLUSTER = range(4)


def orthogonalize_plan(count, rows, cols, dtype=torch.float32, steps=5, coefficients=NEWTON_SCHULZ):
    """How that many matrices are run: (ORTH_BLOCK, ORTH_TEAM, ORTH_PAIRS or ORTH_CLUSTER, blocks to a matrix, matrices at a time; 0 where
    neither is fixed)."""
    code = _dtype_code(torch.empty(0, dtype=dtype))
    desc = FlareOrthDesc(count=count, rows=rows, cols=cols, dtype=code, weight_dtype=code, steps=steps, coefficients=(ctypes.c_float * 3)(*coefficients), eps=1e-7)
    plan = (ctypes.c_int32 * 3)()
    _raise(load().flare_orthogonalize_plan(ctypes.byref(desc), plan), "flare_orthogonalize_plan")
    return tuple(plan)


def muon_update(w, m, g, lr, momentum=0.95, weight_decay=0.0, nesterov=True, update_scale=None, steps=5, coefficients=NEWTON_SCHULZ, eps=1e-7,
                w_out=None, m_out=None, stream=None, check=False):
    """One step of the optimiser that orthogonalises its momentum, on matrices [..., rows, cols]: w of any of the three types, m float32, g
    a gradient of any type.  m' = momentum m + (1 - momentum) g; w' = (1 - lr weight_decay) w - lr update_scale O, O the orthogonalised
    momentum m' + (1 - momentum)(g - m') (nesterov) or m'.  update_scale: None means sqrt(max(1, rows / cols)).  In place unless
    w_out, m_out are given; returns (w', m')."""
    if update_scale is None:                                      # (what is no matrix is refused by the call)
        update_scale = max(1.0, g.shape[-2] / g.shape[-1]) ** 0.5 if g.dim() > 1 and g.shape[-1] > 0 else 1.0
    w1, m1, ws = (_native or _bind()).muon_update(w, m, g, lr, momentum, weight_decay, update_scale, nesterov, steps, *coefficients, eps, w_out, m_out, stream)
    if check:
        (stream or torch.cuda.current_stream()).synchronize()
        flare_check(ws, stream)
    return w1, m1


# ---- tokens: embedding, dropout, the loss over a vocabulary


def _check_waits(ws, stream):
    """Waits for the call that has used ws (on its tensors' device, which need not be the current one) and raises if a wait of it gave up."""
    (stream or torch.cuda.current_stream(ws.device)).synchronize()
    with torch.cuda.device(ws.device):
        flare_check(ws, stream)


class Drop(NamedTuple):
    """Dropout: the share p of elements (to 2^-17) that become 0, by a counter-based generator from seed and offset, 64 bits each.  step: an int64 tensor of one
    number on the GPU that the kernels add to offset when they run, so that a captured graph that counts it up drops other elements every time."""
    p: float
    seed: int
    offset: int = 0
    step: Optional[torch.Tensor] = None


class EmbedGrads(NamedTuple):
    dtable: Optional[torch.Tensor]
    dpositions: Optional[torch.Tensor]


class LossGrads(NamedTuple):
    dx: Optional[torch.Tensor]
    dw: Optional[torch.Tensor]


def dropout(x, drop: Drop, residual=None, out=None, stream=None):
    """residual + drop(x) for x [..., width]; of the residual's type (x's, or float32).  What is kept is multiplied by 1 / (1 - p).  out: a tensor to write to
    (x or residual themselves are allowed)."""
    return (_native or _bind()).dropout(x, drop, residual, out, stream)


def dropout_backward(dy, drop: Drop, dtype=None, out=None, stream=None):
    """The gradient of dropout's x, of `dtype` (dy's; any where dy is float32): the elements that the same Drop keeps.  The residual's is dy."""
    return (_native or _bind()).dropout_backward(dy, drop, dtype, out, stream)


def embed(tokens, table, positions=None, scale=1.0, drop: Optional[Drop] = None, dtype=None, out=None, stream=None):
    """drop(scale * table[tokens] + positions): tokens [..., L] int32 or int64, table [vocab, width], positions [L, width] or None -> [..., L, width] of
    `dtype` (the table's).  A token outside [0, vocab) has no row: zeros in its place."""
    return (_native or _bind()).embed(tokens, table, positions, scale, drop, dtype, out, stream)


def embed_backward(tokens, dy, vocab: int, positions: int = 0, scale=1.0, drop: Optional[Drop] = None, dtype=None, accumulate=False, out=None,
                   stream=None, want_dtable=True) -> EmbedGrads:
    """Gradients of embed's tables, of `dtype` (dy's): dtable [vocab, width] (None without want_dtable) and, with positions = L, dpositions [L, width].
    out: (dtable, dpositions) to write to, either None; accumulate: they are added to instead."""
    return (_native or _bind()).embed_backward(tokens, dy, vocab, positions, scale, drop, dtype, accumulate, out, stream, want_dtable, EmbedGrads)


def token_loss(x, w, labels, scale=1.0, out=None, stream=None, check=False):
    """Softmax cross entropy of the logits scale * x w^T over a vocabulary, which are never kept: x [..., width], w [vocab, width] of the same type, labels
    [...] int32 or int64 -> (loss [...], lse [...]) float32, lse the logarithm of a row's sum of exponentials.  A row whose label is outside [0, vocab) takes no
    part: 0 and 0.  out: (loss, lse) to write to, either None.  With check=True the stream is synchronised and a device-side wait that gave up raises."""
    r, ws = (_native or _bind()).token_loss(x, w, labels, scale, out, stream)
    if check:
        _check_waits(ws, stream)
    return r


def token_loss_backward(x, w, labels, lse, dloss=1.0, scale=1.0, out=None, stream=None, check=False, want_dx=True, want_dw=True) -> LossGrads:
    """Gradients of token_loss from its inputs and its lse.  dloss: what reaches every row's loss, a float32 tensor like lse or one number for all.
    out: (dx, dw) to write to, either None.  want_dx, want_dw: one that is not wanted is not computed, and None."""
    r, ws = (_native or _bind()).token_loss_backward(x, w, labels, lse, dloss, scale, out, stream, want_dx, want_dw, LossGrads)
    if check:
        _check_waits(ws, stream)
    return r
