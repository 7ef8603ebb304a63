"""GPU: the gate projection's gradients where the products cancel each other, and where they need the whole range of a logit's gradient.

Bars, with u = 2^-24 and h = eps / 2 of the activation type: a gradient of a logit is multiplied in three parts of 8 bits, whose products are exact,
and n gradients that are not zero make 3 n products and an addition each: (3 n + 8) u of the terms' magnitudes; dx is rounded once more: h.
"""
import pytest

from test_gpu_gate_grad import inputs, layer, make, run, test_what_is_not_finite as what_is_not_finite
from test_gpu_norm import U, half, m, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E", [(70, 136, 2), (333, 520, 16), (200, 264, 40), (150, 1032, 100), (257, 200, 256)])
def test_experts_that_cancel(m, T, H, E, dtype):  # noqa: F811
    """Two experts of a token with opposite weights, whose gradients differ by 2^-17 of them: what is left of dx is as near as fp32 products leave it."""
    import torch
    cfg = make(m, T, H, E, dtype)
    _, x, w, _ = inputs(T, H, E, dtype, 7, add=False)
    first = w[0].clone()
    w[::2], w[1::2] = first, -first
    g, at = torch.Generator(device="cuda").manual_seed(8), torch.arange(T, device="cuda")
    a = torch.randint(0, (E + 1) // 2, (T,), generator=g, device="cuda") * 2
    b = torch.randint(0, E // 2, (T,), generator=g, device="cuda") * 2 + 1
    v = torch.randn(T, generator=g, device="cuda")
    dl = torch.zeros((T, E), device="cuda")
    dl[at, a], dl[at, b] = v, v * (1 + 2.0 ** -17 * torch.randn(T, generator=g, device="cuda"))
    dx, _ = run(m, cfg, dl, x, w, None, dw=False)
    want, mag = dl.double() @ w.double(), dl.double().abs() @ w.double().abs()
    assert bool(((dx.double() - want).abs() <= want.abs() * half(dtype) + mag * (3 * 2 + 8) * U).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E", [(40, 136, 3), (150, 200, 24), (100, 264, 60), (70, 520, 100), (90, 72, 256)])
def test_largest_numbers(m, T, H, E, dtype):  # noqa: F811
    """Finite gradients beyond the largest bf16 number, 3.39e38, are finite in their products."""
    import torch
    cfg = make(m, T, H, E, dtype)
    _, x, w, _ = inputs(T, H, E, dtype, 5, add=False)
    x, w = x * 2.0 ** -12, w * 2.0 ** -12
    dl, at = torch.zeros((T, E), device="cuda"), torch.arange(T, device="cuda")
    dl[at, at % E] = torch.where(at % 2 == 0, 3.4028234663852886e38, -3.395e38)
    dx, dw = run(m, cfg, dl, x, w, None)
    d = dl.double()
    for got, want, mag, h, n in ((dx, d @ w.double(), d.abs() @ w.double().abs(), half(dtype), 1),
                                 (dw, d.t() @ x.double(), d.abs().t() @ x.double().abs(), 0, -(-T // E))):
        assert bool(((got.double() - want).abs() <= want.abs() * h + mag * (3 * n + 8) * U).all())


@pytest.mark.parametrize("E", [65, 100, 128, 129, 256])
def test_what_is_not_finite_over_many_experts(m, E):  # noqa: F811
    what_is_not_finite(m, E, "bf16")


@pytest.mark.parametrize("E", [40, 100, 256])
def test_many_experts_beyond_2gib(m, E):  # noqa: F811
    """2.3 GB of rows over the experts' forms of their own: all rows are alike, and sums over tokens have few bits."""
    import torch
    T, H = 70003, 16384
    cfg = make(m, T, H, E, "bf16")
    dl = ((torch.arange(E, device="cuda") % 7 - 3) * 0.25).expand(T, E).contiguous()
    x, w = normal(1, H, "bf16", 1).expand(T, H).contiguous(), normal(E, H, "bf16", 2)
    dx, dw = run(m, cfg, dl, x, w, x)
    d = dl[0].double()
    want, mag = d @ w.double() + x[0].double(), d.abs() @ w.double().abs() + x[0].double().abs()
    assert bool(((dx[0].double() - want).abs() <= want.abs() * 2.0 ** -8 + mag * (3 * E + 8) * U).all()) and bool((dx == dx[0]).all())
    sums = T * d[:, None] * x[0].double()
    shares = max(1, m.monta_gate_backward_scratch_bytes(cfg) // (E * H * 4))
    assert bool(((dw.double() - sums).abs() <= sums.abs() * (T // shares + 64 + shares) * U).all())


@pytest.mark.parametrize("E,T", [(40, 600), (100, 600), (256, 333)])
def test_step_of_many_experts_in_a_graph_and_beside_another(m, E, T):  # noqa: F811
    """A bf16 router's training step, captured and replayed with eager work between the replays, and two of them at once on streams of their own."""
    import torch
    cfg, t, o, step = layer(m, "bf16", T=T, E=E)
    _, t2, o2, step2 = layer(m, "bf16", T=T, E=E)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (50, 51, 52):
        for u in (t, t2):
            u["x"].copy_(normal(cfg.tokens, cfg.hidden, "bf16", seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step2()
        torch.cuda.synchronize()
        for name in o:
            assert torch.equal(o[name], o2[name]), name
            o[name].zero_()
            o2[name].zero_()
    del graph
    step2()
    pair, side = [layer(m, "bf16", T=T, E=E) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    for one in pair:
        one[1]["x"].copy_(t2["x"])
    torch.cuda.synchronize()
    for _ in range(4):
        for s, one in zip(side, pair):
            with torch.cuda.stream(s):
                one[3]()
    torch.cuda.synchronize()
    for one in pair:
        for name in o2:
            assert torch.equal(one[2][name], o2[name]), name
