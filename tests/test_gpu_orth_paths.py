"""Every way in which matrices are orthogonalised, by sizes and counts that lead there, against float64 (needs a B200).

Bounds: those of the products in float16 halves, whichever kernel does them (tests.test_gpu_orth).
"""
import math

import pytest
import torch

from paper_2508_12594_b200 import flare
from tests.test_gpu_orth import DT, ENTRY, ULP, close, gradient, reference

pytestmark = pytest.mark.gpu

BLOCK, TEAM, PAIRS, CLUSTER = flare.ORTH_BLOCK, flare.ORTH_TEAM, flare.ORTH_PAIRS, flare.ORTH_CLUSTER

# (count, rows, cols), and what runs it
ONE_BLOCK = [(8, 256, 16), (200, 16, 48), (5, 128, 128), (3, 100, 70)]
TEAMS = [
    (1, 2047, 2500),             # more tiles than blocks, the upper half of a square one a block each
    (1, 1500, 1500),
    (1, 2601, 1003),             # tall, tiles whose sums several blocks share
    (2, 1003, 2601), (2, 2601, 1003), (3, 1100, 1100), (5, 700, 700), (20, 400, 900), (20, 900, 400),    # two teams to twenty
    (80, 130, 200),              # a block is a team
    (149, 65, 520), (150, 520, 65),   # more matrices than teams
]
PAIR = [
    (200, 130, 130),             # one tile, most of it empty
    (150, 130, 900), (150, 900, 130),
    (40, 512, 512), (4, 2048, 2048),  # whole tiles, the upper half of them
    (1, 2500, 2500), (3, 1500, 1500), (1, 3000, 2200), (1, 2200, 3001),   # partial tiles, wide and tall
]
CLUSTERS = [(40, 129, 129), (34, 400, 100), (150, 100, 400), (296, 400, 100), (16, 129, 258), (1, 516, 129), (1, 129, 129)]
PATHS = [(s, BLOCK) for s in ONE_BLOCK] + [(s, TEAM) for s in TEAMS] + [(s, PAIRS) for s in PAIR] + [(s, CLUSTER) for s in CLUSTERS]
NAMES = {BLOCK: "block", TEAM: "team", PAIRS: "pairs", CLUSTER: "cluster"}
each = pytest.mark.parametrize("shape,path", PATHS, ids=lambda v: NAMES[v] if isinstance(v, int) else "x".join(map(str, v)))


def lead_there(shape, path):
    plan = flare.orthogonalize_plan(*shape)
    assert plan[0] == path, f"{shape}: by {plan}"
    return plan


@each
def test_against_float64(shape, path):
    lead_there(shape, path)
    for dtype in ("f32", "bf16", "f16")[:2 if math.prod(shape) % 3 else 3]:
        G = gradient(*shape, dtype=dtype, seed=shape[1])
        O = flare.orthogonalize(G, check=True)
        close(O, reference(G))
        assert torch.equal(flare.orthogonalize(G), O)                 # bit for bit


def test_more_matrices_than_teams_and_clusters():
    assert lead_there((150, 520, 65), TEAM)[2] < 150
    assert lead_there((296, 400, 100), CLUSTER)[2] < 296
    assert 1 < lead_there((3, 1100, 1100), TEAM)[2] < 148


@pytest.mark.parametrize("shape,path", [((200, 130, 130), PAIRS), ((150, 900, 130), PAIRS), ((3, 1500, 1500), PAIRS), ((1, 2200, 3001), PAIRS), ((40, 512, 512), PAIRS),
                                        ((1, 2601, 1003), TEAM), ((2, 1003, 2601), TEAM), ((5, 700, 700), TEAM), ((1, 2047, 2500), TEAM), ((149, 65, 520), TEAM),
                                        ((150, 100, 400), CLUSTER), ((16, 129, 258), CLUSTER)], ids=str)
@pytest.mark.parametrize("weights,grads", [("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32")])
def test_update(shape, path, weights, grads):
    """The optimiser's step: bounds as in tests.test_gpu_orth.test_muon; in place the same bits."""
    lead_there(shape, path)
    gen = torch.Generator(device="cuda").manual_seed(shape[1])
    w = torch.randn(*shape, device="cuda", generator=gen).to(DT[weights])
    m, g = gradient(*shape, seed=1), gradient(*shape, grads, seed=2)
    lr, mu, decay, nesterov = 0.05, 0.9, 0.1, weights != "bf16"
    m64 = mu * m.double() + (1 - mu) * g.double()
    u = mu * m64 + (1 - mu) * g.double() if nesterov else m64
    rho = math.sqrt(max(1.0, shape[1] / shape[2]))
    O = reference(u)
    w64 = (1 - lr * decay) * w.double() - lr * rho * O
    w_out, m_out = torch.empty_like(w), torch.empty_like(m)
    got_w, got_m = flare.muon_update(w, m, g, lr, momentum=mu, weight_decay=decay, nesterov=nesterov, w_out=w_out, m_out=m_out, check=True)
    assert ((got_m.double() - m64).abs() <= 4 * 2.0 ** -24 * (m.double().abs() + g.double().abs())).all()
    rms = O.square().mean((-2, -1), keepdim=True).sqrt()
    bound = max(ULP[w.dtype], 4 * 2.0 ** -24) * w64.abs() + 4 * 2.0 ** -24 * w.double().abs() + lr * rho * ENTRY * rms + (2.0 ** -25 if weights == "f16" else 0.0)
    assert ((got_w.double() - w64).abs() <= bound).all()
    flare.muon_update(w, m, g, lr, momentum=mu, weight_decay=decay, nesterov=nesterov, check=True)
    assert torch.equal(w, got_w) and torch.equal(m, got_m)


@pytest.mark.parametrize("shape,path", [((200, 130, 130), PAIRS), ((150, 900, 130), PAIRS), ((3, 1500, 1500), PAIRS), ((3, 1100, 1100), TEAM), ((20, 900, 400), TEAM),
                                        ((149, 65, 520), TEAM), ((296, 400, 100), CLUSTER)], ids=str)
def test_strides_in_place_and_one_bad_matrix(shape, path):
    lead_there(shape, path)
    count, rows, cols = shape
    wide = torch.full((count, rows + 3, cols + 5), 3.0, device="cuda", dtype=torch.bfloat16)
    G = wide[:, 1:1 + rows, 2:2 + cols]
    G.copy_(gradient(*shape, dtype="bf16", seed=4))
    G[1, 3, 7] = float("nan")
    G[2, rows - 1, cols - 1] = float("inf")
    want = flare.orthogonalize(G.contiguous(), check=True)
    assert want[1].isnan().all() and want[2].isnan().all()
    sound = [0] + list(range(3, count))
    close(want[sound], reference(G[sound]))
    flare.orthogonalize(G, out=G, check=True)
    assert torch.equal(G[sound], want[sound]) and G[1:3].isnan().all()
    G.copy_(torch.full_like(want, 3.0))
    assert (wide == 3).all()


@pytest.mark.parametrize("shape,path", [((8, 256, 16), BLOCK), ((1, 1003, 2601), TEAM), ((3, 1100, 1100), TEAM), ((40, 512, 512), PAIRS), ((16, 129, 258), CLUSTER)], ids=str)
def test_captured(shape, path):
    """In a graph, replayed on other inputs than it was captured with."""
    lead_there(shape, path)
    G = gradient(*shape, seed=1)
    other = gradient(*shape, seed=2)
    want = flare.orthogonalize(other)
    flare.orthogonalize(G)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O = flare.orthogonalize(G)
    G.copy_(other)
    for _ in range(2):
        O.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)


def test_more_elements_than_32_bits_count():
    """2.2 billion of them: the first, the last and some matrices in between."""
    shape = (32767, 256, 264)
    lead_there(shape, PAIRS)
    G = torch.empty(shape, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(7)
    for i in range(0, shape[0], 4096):
        G[i:i + 4096].normal_(generator=gen)
    O = flare.orthogonalize(G, check=True)
    for i in (0, 1, 15886, 31775, 31776, 32765, 32766):
        close(O[i], reference(G[i]))
    del G, O
    torch.cuda.empty_cache()
