"""GPU parity of the gradients of the expert layer, against 64 bits.

Bars.  Small integers make every partial sum an fp32 number: results must agree bit for bit after the one rounding.  On normal data
a sum of n exact products in fp32, in any order, is within n u of the sum of their magnitudes (u = 2^-24); then half a step of the
output's type.
"""
import numpy as np
import pytest

from test_gpu_expert8 import m, routed  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

CASES = [  # tokens, hidden, out_features, experts, top_k, capacity factor, padded, zipf
    (1, 8, 8, 1, 1, 0.0, 0, 0.0),
    (1, 256, 64, 8, 2, 0.0, 0, 0.0),                   # experts without rows
    (5, 72, 136, 4, 2, 0.0, 0, 0.0),
    (64, 128, 128, 4, 1, 0.0, 0, 0.0),
    (65, 520, 264, 3, 2, 0.5, 0, 0.0),
    (200, 264, 520, 16, 3, 0.7, 1, 0.8),
    (700, 1032, 72, 2, 1, 0.0, 0, 0.0),
    (1100, 392, 648, 4, 2, 1.25, 0, 1.2),
    (1500, 136, 1160, 5, 2, 0.9, 1, 0.0),
    (300, 64, 200, 64, 8, 0.0, 0, 1.2),
    (2600, 776, 520, 2, 1, 0.0, 0, 0.0),
    (3300, 2312, 136, 6, 2, 0.0, 0, 0.6),              # large tiles of dx, ragged ones of every length last
    (3300, 2056, 2312, 6, 2, 1.1, 1, 0.0),             # large tiles of both
    (4000, 1288, 200, 60, 8, 0.8, 0, 0.9),             # large tiles of dx, ragged ones in place
]


def act(dtype):
    import torch
    return torch.float32 if dtype == "f32" else torch.bfloat16


def make(rows, H, N, E, dtype, exact, seed=5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def t(*shape):
        v = torch.randint(-3, 4, shape, generator=g, device="cuda").float() if exact else torch.randn(shape, generator=g, device="cuda")
        return v.to(act(dtype))

    return t(rows, N), t(rows, H), t(E, N, H)


def run(m, cfg, ws, tabs, rows, N, dtype, exact, which="both", seed=5):
    import torch
    H, E = cfg.hidden, cfg.experts
    dy, x, w = make(rows, H, N, E, dtype, exact, seed)
    used = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for e in range(E):
        used[tabs["offsets"][e]:tabs["offsets"][e] + tabs["kept"][e]] = True
    dy[~used] = float("nan")                           # rows of no expert reach nothing
    x[~used] = float("nan")
    dx, dw = torch.full((rows + 1, H), 3.0, dtype=act(dtype), device="cuda"), torch.full((E * N + 1, H), 3.0, dtype=act(dtype), device="cuda")
    m.monta_expert_linear_backward(cfg, dy, x if which != "dx" else None, w if which != "dw" else None, N,
                                   dx[:rows] if which != "dw" else None, dw[:E * N].view(E, N, H) if which != "dx" else None, ws)
    torch.cuda.synchronize()
    assert bool((dx[rows] == 3.0).all()) and bool((dw[E * N] == 3.0).all()) and bool((dx[:rows][~used] == 3.0).all())
    return dy, x, w, dx[:rows], dw[:E * N].view(E, N, H)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exact", [1, 0])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_gradients(m, case, dtype, exact):  # noqa: F811
    import torch
    T, H, N, E, k, cf, padded, zipf = case
    cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k, cf, padded, zipf=zipf)
    dy, x, w, dx, dw = run(m, cfg, ws, tabs, rows, N, dtype, exact)
    half = U if dtype == "f32" else 2.0 ** -8
    for e in range(E):
        n = int(tabs["kept"][e])
        seg = slice(int(tabs["offsets"][e]), int(tabs["offsets"][e]) + n)
        a, b, c = dy[seg].double(), x[seg].double(), w[e].double()
        for got, want, mag, terms in ((dx[seg], a @ c, a.abs() @ c.abs(), N), (dw[e], a.T @ b, a.abs().T @ b.abs(), n)):
            if exact:
                assert torch.equal(got.double(), want.to(act(dtype)).double()), (e, terms)
            else:
                assert bool(((got.double() - want).abs() <= terms * U * mag + half * want.abs()).all()), (e, terms)


LONG = [  # experts with so many rows and so few weights that the walk over the rows is what takes time
    (5000, 72, 64, 2, 2, 0.0, 0, 0.4),                 # a single tile of dw for each
    (130, 136, 72, 7, 3, 0.0, 0, 2.0),                 # from a few rows to all of them
    (7000, 504, 392, 4, 2, 0.0, 0, 0.4),
    (4100, 776, 264, 8, 2, 0.9, 1, 0.0),
    (10500, 504, 512, 4, 4, 0.0, 0, 0.0),              # and so many rows that dx goes in its largest tiles
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", LONG, ids=lambda c: "-".join(map(str, c)))
def test_long_walks(m, case, dtype):  # noqa: F811
    test_gradients(m, case, dtype, 1)
    test_gradients(m, case, dtype, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_either_alone(m, dtype):  # noqa: F811
    import torch
    cfg, ws, tabs, rows = routed(m, 150, 136, dtype, 4, 2, 0.8)
    _, _, _, dx, dw = run(m, cfg, ws, tabs, rows, 200, dtype, 0)
    assert torch.equal(run(m, cfg, ws, tabs, rows, 200, dtype, 0, "dx")[3], dx)
    assert torch.equal(run(m, cfg, ws, tabs, rows, 200, dtype, 0, "dw")[4], dw)


def test_against_differences(m):  # noqa: F811
    """The layer is linear in its rows and in its weights: differences of monta_expert_linear's own definition are the gradient exactly, so on
    integers d loss = <dy, y(x + e) - y(x)> is a whole number."""
    import torch
    cfg, ws, tabs, rows = routed(m, 40, 64, "f32", 3, 2)
    dy, x, w, dx, dw = run(m, cfg, ws, tabs, rows, 48, "f32", 1)
    y0, y1 = torch.zeros((rows, 48), device="cuda"), torch.zeros((rows, 48), device="cuda")
    m.monta_expert_linear(cfg, x, w, 48, y0, ws)
    for r, h in ((0, 0), (17, 63), (rows - 1, 31)):
        x2 = x.clone()
        x2[r, h] += 1
        m.monta_expert_linear(cfg, x2, w, 48, y1, ws)
        assert (dy * (y1 - y0)).sum().item() == dx[r, h].item()
    for e, n, h in ((0, 0, 0), (2, 47, 63)):
        w2 = w.clone()
        w2[e, n, h] += 1
        m.monta_expert_linear(cfg, x, w2, 48, y1, ws)
        assert (dy * (y1 - y0)).sum().item() == dw[e, n, h].item()


def test_graph(m):  # noqa: F811
    """Captured and replayed, with eager work and other problems between the replays."""
    import torch
    cfg, ws, tabs, rows = routed(m, 500, 264, "bf16", 4, 2)
    dy, x, w = make(rows, 264, 392, 4, "bf16", 0)
    dx, dw = torch.zeros((rows, 264), dtype=x.dtype, device="cuda"), torch.zeros_like(w)
    m.monta_expert_linear_backward(cfg, dy, x, w, 392, dx, dw, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.monta_expert_linear_backward(cfg, dy, x, w, 392, dx, dw, ws)
    for seed in (8, 9, 10):
        for t, s in zip((dy, x, w), make(rows, 264, 392, 4, "bf16", 0, seed)):
            t.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = dx.clone(), dw.clone()
        dx.zero_(), dw.zero_()
        m.monta_expert_linear_backward(cfg, dy, x, w, 392, dx, dw, ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
