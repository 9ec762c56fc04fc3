"""Orthogonalised updates against float64 (needs a B200).

Bounds, derived before the first run.  Factors of two float16 halves are off by up to 2^-23 of their size, some 1e-7; what is rounded away of X stands
beside its large singular directions and is lifted with the small ones, by up to 485, but spreads over all S directions: 5e-5 / sqrt(S)
of the result's 2-norm, and sums in float32 with truncation add a few 2^-24 sqrt(K).  So 3e-5 in 2-norm (S = 1, where nothing is lifted
against anything else, included), seven times that of the RMS for any one entry, and one rounding where it is stored in 16 bits.
"""
import ctypes
import math

import pytest
import torch

from paper_2508_12594_b200 import flare
from tests._util import STORE_ULP

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ULP = {DT[k]: v for k, v in STORE_ULP.items()}
NORM, ENTRY = 3e-5, 2.1e-4


def reference(G, steps=5, coefficients=flare.NEWTON_SCHULZ, eps=1e-7):
    a, b, c = coefficients
    X = G.double()
    X = X / (X.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    tall = X.shape[-2] > X.shape[-1]
    X = X.mT if tall else X
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * A @ A) @ X
    return X.mT if tall else X


def close(got, ref, what="O"):
    assert got.shape == ref.shape
    err = (got.double() - ref).abs()
    rms = ref.square().mean((-2, -1), keepdim=True).sqrt()
    stored = ULP[got.dtype] * ref.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0.0)
    excess = (err - stored).clamp(min=0.0)
    rel = (excess.square().mean((-2, -1), keepdim=True).sqrt() / rms.clamp(min=1e-300)).max()
    assert rel <= NORM, f"{what}: off by {float(rel):.3e} of its 2-norm"
    worst = (excess / rms.clamp(min=1e-300)).max()
    assert worst <= ENTRY, f"{what}: an entry off by {float(worst):.3e} of the RMS"


def gradient(count, rows, cols, dtype="f32", seed=0, strong=10.0, size=1e-3):
    """A few strong directions over noise."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = max(1, min(rows, cols) // 16)
    low = torch.randn(count, rows, r, device="cuda", generator=g) @ torch.randn(count, r, cols, device="cuda", generator=g)
    return (size * (torch.randn(count, rows, cols, device="cuda", generator=g) + strong * low / math.sqrt(r))).to(DT[dtype])


# one row, short sides around the steps of 16, 64 and 128, long sides up to what one block holds and just beyond; then matrices of many tiles
SHAPES = [(1, 1, 1), (1, 1, 70), (2, 3, 2), (1, 15, 40), (3, 16, 16), (2, 17, 33), (8, 256, 16), (2, 31, 512), (1, 64, 64), (2, 64, 832), (1, 64, 833), (1, 65, 130),
          (2, 100, 300), (5, 128, 128), (1, 128, 320), (1, 128, 321), (1, 321, 128), (1, 127, 129), (1, 129, 129), (2, 200, 129), (1, 256, 256), (3, 300, 1000),
          (1, 1000, 301), (2, 520, 70), (1, 640, 2048), (1, 1100, 1100), (1, 130, 5000), (1, 16, 3000), (1, 20, 9000)]


@pytest.mark.parametrize("i", range(len(SHAPES)), ids=lambda i: str(SHAPES[i]))
def test_against_float64(i):
    for dtype in (("f32", "bf16"), ("f32", "f16"))[i % 2]:
        G = gradient(*SHAPES[i], dtype=dtype, seed=i)
        close(flare.orthogonalize(G, check=True), reference(G))


@pytest.mark.parametrize("rows,cols", [(48, 48), (200, 300)])
@pytest.mark.parametrize("steps,coefficients", [(1, flare.NEWTON_SCHULZ), (2, flare.NEWTON_SCHULZ), (7, flare.NEWTON_SCHULZ), (12, (1.5, -0.5, 0.0)), (3, (1.875, -1.25, 0.375))])
def test_steps_and_coefficients(rows, cols, steps, coefficients):
    G = gradient(2, rows, cols, seed=steps, strong=1.0)
    close(flare.orthogonalize(G, steps=steps, coefficients=coefficients, check=True), reference(G, steps, coefficients))


@pytest.mark.parametrize("rows,cols", [(40, 64), (64, 40), (150, 260)])
def test_singular_vectors_are_kept_and_values_near_one(rows, cols):
    G = gradient(1, rows, cols, seed=5, strong=2.0)[0]
    U, s, Vh = torch.linalg.svd(G.double(), full_matrices=False)
    O = flare.orthogonalize(G).double()
    values = torch.linalg.svdvals(O)
    assert values.max() < 1.25
    D = U.mT @ O @ Vh.mT                                          # diagonal: the polynomial of the singular values
    x = s / s.square().sum().sqrt()
    a, b, c = flare.NEWTON_SCHULZ
    for _ in range(5):
        x = a * x + b * x ** 3 + c * x ** 5
    assert (D - torch.diag(x)).abs().max() < 2e-4


@pytest.mark.parametrize("rows,cols", [(32, 100), (160, 260)])
def test_size_of_the_gradient_does_not_matter(rows, cols):
    G = gradient(1, rows, cols, seed=8)
    want = flare.orthogonalize(G, eps=0.0)
    for size in (2.0 ** -80, 2.0 ** 60):                          # powers of two: the same bits
        assert torch.equal(flare.orthogonalize(G * size, eps=0.0), want)
    assert (flare.orthogonalize(torch.zeros_like(G)) == 0).all()


@pytest.mark.parametrize("rows,cols", [(32, 100), (160, 260)])
def test_one_matrix_of_a_batch_does_not_reach_another(rows, cols):
    G = gradient(4, rows, cols, seed=11)
    want = flare.orthogonalize(G)
    G[1, 3, 7] = float("nan")
    G[2, rows - 1, cols - 1] = float("inf")
    got = flare.orthogonalize(G, check=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])
    assert got[1].isnan().all() and got[2].isnan().all()


@pytest.mark.parametrize("rows,cols", [(24, 90), (90, 24), (150, 300), (300, 150)])
def test_strides_and_in_place(rows, cols):
    wide = torch.full((3, rows + 5, cols + 7), 3.0, device="cuda", dtype=torch.bfloat16)
    G = wide[:, 2:2 + rows, 3:3 + cols]
    G.copy_(gradient(3, rows, cols, "bf16", seed=4))
    want = flare.orthogonalize(G.contiguous())
    assert torch.equal(flare.orthogonalize(G), want)
    out = torch.full((3, rows, cols + 1), 5.0, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(flare.orthogonalize(G, out=out[..., :cols]), want) and (out[..., cols] == 5).all()
    flare.orthogonalize(G, out=G)
    assert torch.equal(G, want)
    wide[:, 2:2 + rows, 3:3 + cols] = 3.0
    assert (wide == 3).all()


@pytest.mark.parametrize("rows,cols", [(16, 256), (256, 16), (128, 128), (400, 150), (257, 300)])
@pytest.mark.parametrize("weights,grads", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon(rows, cols, weights, grads, nesterov):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.randn(2, rows, cols, device="cuda", generator=gen).to(DT[weights])
    m, g = gradient(2, rows, cols, seed=1), gradient(2, rows, cols, grads, seed=2)
    lr, mu, decay = 0.05, 0.9, 0.1
    m64 = mu * m.double() + (1 - mu) * g.double()
    u = mu * m64 + (1 - mu) * g.double() if nesterov else m64
    rho = math.sqrt(max(1.0, rows / cols))
    O = reference(u)
    w64 = (1 - lr * decay) * w.double() - lr * rho * O
    w_out, m_out = torch.empty_like(w), torch.empty_like(m)
    got_w, got_m = flare.muon_update(w, m, g, lr, momentum=mu, weight_decay=decay, nesterov=nesterov, w_out=w_out, m_out=m_out, check=True)
    assert got_w.data_ptr() == w_out.data_ptr() and got_m.data_ptr() == m_out.data_ptr()
    # momentum: the coefficients are float32, two operations; weights: one rounding, and lr rho times what O is off by
    assert ((got_m.double() - m64).abs() <= 4 * 2.0 ** -24 * (m.double().abs() + g.double().abs())).all()
    rms = O.square().mean().sqrt()
    bound = max(ULP[w.dtype], 4 * 2.0 ** -24) * w64.abs() + 4 * 2.0 ** -24 * w.double().abs() + lr * rho * ENTRY * rms + (2.0 ** -25 if weights == "f16" else 0.0)
    assert ((got_w.double() - w64).abs() <= bound).all()
    w2, m2 = w.clone(), m.clone()
    flare.muon_update(w2, m2, g, lr, momentum=mu, weight_decay=decay, nesterov=nesterov)
    assert torch.equal(w2, got_w) and torch.equal(m2, got_m)


def test_no_matrices():
    assert flare.orthogonalize(torch.empty(0, 5, 7, device="cuda")).shape == (0, 5, 7)
    w, m = torch.empty(0, 300, 200, device="cuda"), torch.empty(0, 300, 200, device="cuda")
    flare.muon_update(w, m, m, lr=0.1)


@pytest.mark.parametrize("rows,cols", [(64, 100), (260, 520)])
def test_on_another_stream_captured_and_repeated(rows, cols):
    src = gradient(3, rows, cols, seed=21)
    want = flare.orthogonalize(src)
    for _ in range(3):
        assert torch.equal(flare.orthogonalize(src), want)
    G = torch.zeros_like(src)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = torch.randn(4096, 4096, device="cuda")
        for _ in range(4):
            a = a @ a * 1e-2
        G.copy_(src)
    O = flare.orthogonalize(G, stream=side)
    side.synchronize()
    assert torch.equal(O, want)
    G.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = flare.orthogonalize(G)
    G.copy_(src)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)


def test_refusals():
    G = torch.zeros(2, 8, 12, device="cuda")
    with pytest.raises(ValueError, match="matrices"):
        flare.orthogonalize(torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError, match="CUDA"):
        flare.orthogonalize(G.cpu())
    with pytest.raises(TypeError, match="unsupported dtype"):
        flare.orthogonalize(G.double())
    with pytest.raises(ValueError, match="adjacent columns"):
        flare.orthogonalize(G.mT)
    with pytest.raises(ValueError, match="shape"):
        flare.orthogonalize(G, out=torch.zeros(2, 8, 11, device="cuda"))
    with pytest.raises(TypeError, match="float32"):
        flare.orthogonalize(G, out=G.bfloat16())
    for kw, status in ((dict(steps=0), flare.ERR_INVALID_ARG), (dict(steps=65), flare.ERR_UNSUPPORTED), (dict(eps=-1.0), flare.ERR_UNSUPPORTED),
                       (dict(coefficients=(float("nan"), 0.0, 0.0)), flare.ERR_UNSUPPORTED), (dict(coefficients=(5.0, 3.0, 1.0)), flare.ERR_UNSUPPORTED)):
        with pytest.raises(flare.FlareError) as e:
            flare.orthogonalize(G, **kw)
        assert e.value.status == status, kw
    with pytest.raises(ValueError, match="shape"):
        flare.muon_update(G, torch.zeros(2, 8, 11, device="cuda"), G, lr=0.1)
    with pytest.raises(TypeError, match="float32"):
        flare.muon_update(G, G.bfloat16(), G, lr=0.1)
    with pytest.raises(ValueError, match="contiguous"):
        flare.muon_update(torch.zeros(2, 8, 24, device="cuda")[..., :12], G, G, lr=0.1)
    with pytest.raises(flare.FlareError) as e:
        flare.muon_update(G, G, G, lr=float("inf"))
    assert e.value.status == flare.ERR_INVALID_ARG
    lib = flare.load()
    desc = flare.FlareOrthDesc(count=1, rows=300, cols=300, steps=5, coefficients=(ctypes.c_float * 3)(*flare.NEWTON_SCHULZ), eps=1e-7)
    need = lib.flare_orthogonalize_workspace_bytes(ctypes.byref(desc))
    A = torch.zeros(300, 300, device="cuda")
    p = ctypes.c_void_p(A.data_ptr())
    assert lib.flare_orthogonalize(ctypes.byref(desc), p, p, p, need - 1, None) == flare.ERR_WORKSPACE_TOO_SMALL
