"""GPU parity of the gate projection's gradients against 64 bits, and of the way from the losses back to the norm's input as a whole.

Bars, with u = 2^-24 and h = eps / 2 of the activation type:
  - dx adds E products and dadd in fp32: (E + 8) u of the terms' magnitudes.  With bf16 activations a gradient of a logit is multiplied as two
    bf16 numbers: v in [2^e, 2^(e+1)) leaves at most half a step, 2^(e-8); that is a bf16 number itself or lies below it, in binades whose half
    step is at most 2^(e-9-8), so the two leave 2^-17 of v.  Rounded once: h.
  - dw adds a share of the products in fp32, every so many steps of 16 or 32 tokens, then the shares: tokens / shares + 64 + shares additions; three bf16 numbers leave 2^(e-18-8), 2^-26 of v, a
    quarter of a u.
"""
import numpy as np
import pytest

from test_gpu_norm import U, dt, half, m, normal  # noqa: F401

pytestmark = pytest.mark.gpu


def make(m, T, H, E, dtype):  # noqa: F811
    return m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, E, 1, 1, 1, 1)


def scratch(n):
    import torch
    return torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")


def inputs(T, H, E, dtype, seed, add=True):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dl = torch.randn((T, E), generator=g, device="cuda") * torch.exp(2 * torch.randn((T, E), generator=g, device="cuda"))
    return dl, normal(T, H, dtype, seed + 1), normal(E, H, dtype, seed + 2), normal(T, H, dtype, seed + 3) if add else None


def run(m, cfg, dl, x, w, add, dx=True, dw=True):  # noqa: F811
    import torch
    T, H, E = cfg.tokens, cfg.hidden, cfg.experts
    dxb = torch.full((T + 1, H), 5.0, device="cuda", dtype=x.dtype) if dx else None
    dwb = torch.full((E + 1, H), 5.0, device="cuda") if dw else None
    m.monta_gate_backward(cfg, dl, x if dw else None, w if dx else None, add if dx else None, dxb[:T] if dx else None, dwb[:E] if dw else None,
                          scratch(m.monta_gate_backward_scratch_bytes(cfg)) if dw else None)
    torch.cuda.synchronize()
    assert not dx or bool((dxb[T] == 5).all())
    assert not dw or bool((dwb[E] == 5).all())
    return dxb[:T] if dx else None, dwb[:E] if dw else None


def check(m, cfg, dl, x, w, add, dx, dw):  # noqa: F811
    T, H, E = cfg.tokens, cfg.hidden, cfg.experts
    bf16 = cfg.dtype == m.BF16
    d, a, b = dl.double(), x.double(), w.double()
    want, mag = d @ b, d.abs() @ b.abs()
    if add is not None:
        want, mag = want + add.double(), mag + add.double().abs()
    assert bool(((dx.double() - want).abs() <= want.abs() * half("bf16" if bf16 else "f32") + mag * ((E + 8) * U + (2.0 ** -17 if bf16 else 0))).all())
    shares = max(1, m.monta_gate_backward_scratch_bytes(cfg) // (E * H * 4))
    chain = T // shares + 64 + shares
    assert bool(((dw.double() - d.t() @ a).abs() <= (d.abs().t() @ a.abs()) * chain * U).all())


SIZES = [(1, 8, 1), (1, 4096, 8), (15, 64, 3), (17, 72, 16), (64, 256, 17), (100, 264, 32), (333, 520, 10), (1000, 136, 33), (129, 1032, 64), (700, 512, 65),
         (50, 4104, 8), (257, 336, 128), (300, 128, 129), (65, 2056, 200), (1111, 200, 256), (4097, 96, 8), (3000, 1024, 64), (2, 16, 256), (9000, 40, 100),
         (31, 8, 40), (513, 16392, 5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E", SIZES)
def test_gradients(m, T, H, E, dtype):  # noqa: F811
    import torch
    cfg = make(m, T, H, E, dtype)
    dl, x, w, add = inputs(T, H, E, dtype, T + E)
    dx, dw = run(m, cfg, dl, x, w, add)
    check(m, cfg, dl, x, w, add, dx, dw)
    plain, dw2 = run(m, cfg, dl, x, w, None)
    check(m, cfg, dl, x, w, None, plain, dw2)
    assert torch.equal(dw2, dw)                        # the same again: a fixed order of additions
    # either one alone
    only, none = run(m, cfg, dl, x, w, add, dw=False)
    assert none is None and torch.equal(only, dx)
    none, only = run(m, cfg, dl, x, w, add, dx=False)
    assert none is None and torch.equal(only, dw)
    # in place
    both = add.clone()
    m.monta_gate_backward(cfg, dl, x, w, both, both, dw2, scratch(m.monta_gate_backward_scratch_bytes(cfg)))
    assert torch.equal(both, dx)


@pytest.mark.parametrize("T,H,E", [(32833, 4104, 40), (16400, 8200, 100)])
def test_many_elements(m, T, H, E):  # noqa: F811
    """From 2^27 elements of x on, 33 to 128 experts have a form of their own."""
    test_gradients(m, T, H, E, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E", [4, 40])
def test_what_is_not_finite(m, E, dtype):  # noqa: F811
    """A NaN or infinity reaches what it is a factor of, and nothing else: rows of dx and columns of dw."""
    import torch
    T, H = 150, 200
    cfg = make(m, T, H, E, dtype)
    dl, x, w, add = inputs(T, H, E, dtype, 3)
    dx, dw = run(m, cfg, dl, x, w, add)
    x[149, 7], add[11, 100] = float("nan"), float("inf")
    dx2, dw2 = run(m, cfg, dl, x, w, add)
    assert bool(torch.isnan(dw2[:, 7]).all()) and torch.equal(dw2[:, 8:], dw[:, 8:]) and torch.equal(dw2[:, :7], dw[:, :7])
    assert dx2[11, 100].item() == float("inf")
    dx2[11, 100] = dx[11, 100]
    assert torch.equal(dx2, dx)
    dl[77, 2] = float("nan")
    dx2, dw2 = run(m, cfg, dl, x, w, None)
    assert bool(torch.isnan(dx2[77]).all()) and bool(torch.isnan(dw2[2]).all()) and bool(torch.isfinite(dw2[3, 8:]).all())
    assert bool(torch.isfinite(dx2[torch.arange(T, device="cuda") != 77]).all())


@pytest.mark.parametrize("E", [8, 100])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_on_4_bytes(m, E, dtype):  # noqa: F811
    """dlogits needs no more than the alignment of its numbers."""
    import torch
    T, H = 70, 136
    cfg = make(m, T, H, E, dtype)
    dl, x, w, add = inputs(T, H, E, dtype, 11)
    store = torch.empty(T * E + 3, device="cuda")
    want = run(m, cfg, dl, x, w, add)
    for at in (1, 2, 3):
        part = store[at:at + T * E].view(T, E)
        part.copy_(dl)
        assert all(torch.equal(a, b) for a, b in zip(run(m, cfg, part, x, w, add), want))


def test_rows_beyond_2gib(m):  # noqa: F811
    import torch
    T, H, E = 70003, 16384, 3                          # 2.3 GB of rows
    cfg = make(m, T, H, E, "bf16")
    dl = torch.ones((T, E), device="cuda")
    dl[:, 1], dl[:, 2] = 0.5, -2.0
    x, w = normal(1, H, "bf16", 1).expand(T, H).contiguous(), normal(E, H, "bf16", 2)
    dx, dw = run(m, cfg, dl, x, w, x)
    want = (dl[0].double() @ w.double() + x[0].double())
    mag = dl[0].double().abs() @ w.double().abs() + x[0].double().abs()
    assert bool(((dx[0].double() - want).abs() <= want.abs() * 2.0 ** -8 + mag * (E + 8) * U).all()) and bool((dx == dx[0]).all())
    sums = dl.double().sum(0)[:, None] * x[0].double()
    shares = max(1, m.monta_gate_backward_scratch_bytes(cfg) // (E * H * 4))
    assert bool(((dw.double() - sums).abs() <= sums.abs() * (T // shares + 64 + shares) * U).all())


def layer(m, dtype, T=600, H=264, E=12, k=3, seed=7):  # noqa: F811
    """A router's training step from the residual stream to its losses and back, on buffers of its own."""
    import torch
    cfg = m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, E, k, 1, 1, 1, 0.9)
    b = m.alloc_buffers(cfg, np.zeros((T, E), np.float32))
    t = {"x": normal(T, H, dtype, seed) + 0.5, "res": normal(T, H, dtype, seed + 1), "w": (1 + 0.1 * normal(1, H, "f32", seed + 2)[0]).to(dt(dtype)),
         "b": (0.1 * normal(1, H, "f32", seed + 3)[0]).to(dt(dtype)), "wg": normal(E, H, dtype, seed + 4, H ** -0.5), "dback": normal(T, H, dtype, seed + 5),
         "dres": normal(T, H, dtype, seed + 6), "mask": (torch.arange(T, device="cuda") % 10 < 9).to(torch.uint8), "dl": torch.tensor([2.0, 0.3], device="cuda") * T,
         "dg": normal(T, k, "f32", seed + 7)}
    like = {"s": t["x"], "n": t["x"], "dn": t["x"], "dx": t["x"]}
    o = {name: torch.empty_like(v) for name, v in like.items()}
    o.update(losses=torch.empty(2, device="cuda"), counts=torch.empty(E + 1, dtype=torch.int32, device="cuda"), means=torch.empty(E, device="cuda"),
             dlogits=torch.empty((T, E), device="cuda"), dwg=torch.empty((E, H), device="cuda"), dw=torch.empty(H, device="cuda"), db=torch.empty(H, device="cuda"))
    s = [scratch(f(cfg)) for f in (m.monta_route_loss_scratch_bytes, m.monta_gate_backward_scratch_bytes, m.monta_layernorm_scratch_bytes)]

    def step():
        m.monta_layernorm(cfg, t["x"], t["res"], t["w"], t["b"], 1e-5, o["s"], o["n"])
        m.monta_gate(cfg, o["n"], t["wg"], b.logits)
        m.monta_route(cfg, b.logits, b.topk_idx, b.gates, b.ws)
        m.monta_route_loss(cfg, b.logits, b.topk_idx, t["mask"], o["losses"], o["counts"], o["means"], s[0])
        m.monta_route_backward(cfg, b.logits, b.topk_idx, b.gates, t["dg"], t["mask"], t["dl"], o["counts"], o["dlogits"])
        m.monta_gate_backward(cfg, o["dlogits"], o["n"], t["wg"], t["dback"], o["dn"], o["dwg"], s[1])
        m.monta_layernorm_backward(cfg, o["s"], t["w"], 1e-5, o["dn"], t["dres"], o["dx"], o["dw"], o["db"], s[2])

    o.update(logits=b.logits, gates=b.gates, idx=b.topk_idx)
    return cfg, t, o, step


def test_router_training_step(m):  # noqa: F811
    """fp32: the whole run against the same differentiated in 64 bits.  Each link is held to its own bar elsewhere; over the links errors of about
    300 u of a quantity of size 1 to 30 add up, magnified by at most the norms of the links' Jacobians (below 8 each here)."""
    import torch
    cfg, t, o, step = layer(m, "f32")
    step()
    torch.cuda.synchronize()
    T, E, k = cfg.tokens, cfg.experts, cfg.top_k
    x, w, b, wg = (t[n].double().requires_grad_() for n in ("x", "w", "b", "wg"))
    s = x + t["res"].double()
    n = torch.nn.functional.layer_norm(s, (cfg.hidden,), w, b, 1e-5)
    logits = n @ wg.t()
    keep, idx = t["mask"] != 0, o["idx"].long()
    assert bool(((logits - o["logits"]).abs() <= 1e-4).all())
    live = logits[keep]
    p = torch.softmax(live, 1)
    f = torch.bincount(idx[keep].reshape(-1), minlength=E).double() * E / (k * int(keep.sum()))
    balance, z = (f * p.mean(0)).sum(), (torch.logsumexp(live, 1) ** 2).mean()
    assert abs(o["losses"][0].item() - balance.item()) <= 1e-5 and abs(o["losses"][1].item() - z.item()) <= 1e-4
    gates = torch.softmax(torch.gather(live, 1, idx[keep]), 1)
    whole = (gates * t["dg"][keep].double()).sum() + (n * t["dback"].double()).sum() + (s * t["dres"].double()).sum() + balance * t["dl"][0].double() + z * t["dl"][1].double()
    for name, want in zip(("dx", "dw", "db", "dwg"), torch.autograd.grad(whole, [x, w, b, wg])):
        got = o[name].double()
        assert (got - want).norm().item() <= 1e-4 * want.norm().item(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_step_in_a_graph_and_beside_another(m, dtype):  # noqa: F811
    """Captured and replayed, with eager work between the replays; two layers at once on streams of their own."""
    import torch
    cfg, t, o, step = layer(m, dtype)
    _, t2, o2, step2 = layer(m, dtype)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (50, 51, 52):
        for u in (t, t2):
            u["x"].copy_(normal(cfg.tokens, cfg.hidden, dtype, seed))
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
    want = layer(m, dtype, seed=60)
    want[3]()
    pair, side = [layer(m, dtype, seed=60) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, one in zip(side, pair):
            with torch.cuda.stream(s):
                one[3]()
    torch.cuda.synchronize()
    for one in pair:
        for name in one[2]:
            assert torch.equal(one[2][name], want[2][name]), name
