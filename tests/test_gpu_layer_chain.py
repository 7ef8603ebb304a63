"""The operators together, as a layer uses them: serving in 8 bits, and a training step, forward and backward.

Bars.  Every stage's error is at most its number of additions times u = 2^-24 of its terms' magnitudes, plus half a step of the
activation type where it stores one.  Run with magnitudes in the place of values, the same chain carries these along, so the chain's
result is within (all additions times u + all roundings) of the chain of magnitudes, to first order.
"""
import numpy as np
import pytest

from test_gpu_expert8 import m  # noqa: F401

pytestmark = pytest.mark.gpu
U, EPS = 2.0 ** -24, 1e-5


def act(dtype):
    import torch
    return torch.float32 if dtype == "f32" else torch.bfloat16


def half(dtype):
    return U if dtype == "f32" else 2.0 ** -8


def normal(shape, dtype, seed, scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


SHAPES = [(1, 256, 4, 2, 1, 1, 0.0, 0), (48, 512, 8, 2, 2, 2, 0.0, 0), (240, 272, 6, 3, 1, 4, 0.8, 0), (512, 128, 16, 4, 2, 1, 0.6, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E,k,tp,S,cf,padded", SHAPES)
def test_serving(m, T, H, E, k, tp, S, cf, padded, dtype):  # noqa: F811
    """norm (16 bits to the gate, 8 bits to the experts), gate, the slice pipeline on 8-bit rows, 8-bit experts, combine."""
    import torch
    from paper_2411_00662_amd import buffers
    a, N, nb = act(dtype), H, -(-H // 128)
    cfg = m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, E, k, 1, tp, S, cf, 1, padded)
    moved, row8 = m.monta_fp8_rows(cfg)
    L = m.monta_ws_layout_query(cfg)
    x, res, w = normal((T, H), a, 1), normal((T, H), a, 2), (1 + 0.2 * normal((H,), torch.float32, 3)).to(a)
    wg = normal((E, H), a, 4, H ** -0.5)
    wc, wsc = normal((E, N, H), torch.float32, 5, 40.0).clamp(-448, 448).to(torch.float8_e4m3fn), 0.001 + 0.001 * torch.rand((E, -(-N // 128), nb), device="cuda")
    s, out = torch.empty_like(x), torch.empty_like(x)
    rows = torch.empty((T, row8), dtype=torch.uint8, device="cuda")
    stage, final = (torch.full((L.max_rows, row8), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2))
    logits, gates, idx = torch.empty((T, E), device="cuda"), torch.empty((T, k), device="cuda"), torch.empty((T, k), dtype=torch.int32, device="cuda")
    ws = torch.empty(L.ws_bytes, dtype=torch.uint8, device="cuda")
    y, o = torch.zeros((L.max_rows, N), dtype=a, device="cuda"), torch.empty((T, N), dtype=a, device="cuda")
    m.monta_ws_init(cfg, ws)
    m.monta_rmsnorm(cfg, x, res, w, EPS, s, out, rows)
    m.monta_gate(cfg, out, wg, logits)
    m.monta_route_dispatch_regather(moved, logits, rows, idx, gates, stage, final, ws)
    m.monta_expert_linear_fp8(cfg, final, wc, wsc, N, y, ws)
    m.monta_combine(cfg, y, gates, o, ws)
    torch.cuda.synchronize()
    tabs = buffers.read_tables(cfg, ws)
    pos = torch.from_numpy(tabs["pos_final"]).cuda().long()
    t, j = (pos >= 0).nonzero(as_tuple=True)
    assert torch.equal(final[pos[t, j]], rows[t]), "8-bit rows travel bit for bit"
    v = rows[:, :H].contiguous().view(torch.float8_e4m3fn).double() * rows[:, H:H + 4 * nb].contiguous().view(torch.float32).double().repeat_interleave(128, 1)[:, :H]
    we = wc.double() * wsc.double().repeat_interleave(128, 1)[:, :N].repeat_interleave(128, 2)[:, :, :H]
    want, mag = torch.zeros((T, N), dtype=torch.float64, device="cuda"), torch.zeros((T, N), dtype=torch.float64, device="cuda")
    for e in range(E):
        sel = idx[t, j] == e
        g = gates[t[sel], j[sel]].double()[:, None]
        want.index_add_(0, t[sel], g * (v[t[sel]] @ we[e].T))
        mag.index_add_(0, t[sel], g * (v[t[sel]].abs() @ we[e].abs().T))
    # bf16: the 8-bit instruction loses less than 15 products' 2^-13 of the largest of 16, at most 15 / 2^13 of the sum of magnitudes
    tol = ((H + 60) * U + (15 * 2.0 ** -13 if dtype == "bf16" else 0)) * mag + 2 * half(dtype) * mag
    assert bool(((o.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E,k,tp,S,cf,padded", SHAPES + [(1200, 264, 4, 2, 1, 1, 1.0, 0)])
def test_training_step(m, T, H, E, k, tp, S, cf, padded, dtype):  # noqa: F811
    """norm, gate, routing and dispatch, experts, combine; back through the combine, the experts, the dispatch (the combine with gates
    of one) and the norm.  The choices and the gates are the library's; the gates are leaves."""
    import torch
    from paper_2411_00662_amd import buffers
    a, N = act(dtype), H
    cfg = m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, E, k, 1, tp, S, cf, 1, padded)
    L = m.monta_ws_layout_query(cfg)
    x, res, w = normal((T, H), a, 1), normal((T, H), a, 2), (1 + 0.2 * normal((H,), torch.float32, 3)).to(a)
    wg, we = normal((E, H), a, 4, H ** -0.5), normal((E, N, H), a, 5, H ** -0.5)
    dout, dsum = normal((T, N), a, 6, 0.5), normal((T, H), a, 7)
    new = lambda *shape: torch.empty(shape, dtype=a, device="cuda")  # noqa: E731
    s, out, o, dn, dx, dw_e = new(T, H), new(T, H), new(T, N), new(T, H), new(T, H), new(E, N, H)
    stage, final, y, dy, dfinal = (torch.zeros((L.max_rows, H), dtype=a, device="cuda") for _ in range(5))
    logits, gates, dgates = torch.empty((T, E), device="cuda"), torch.empty((T, k), device="cuda"), torch.empty((T, k), device="cuda")
    idx, ones, dw = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.ones((T, k), device="cuda"), torch.empty(H, device="cuda")
    ws, scratch = torch.empty(L.ws_bytes, dtype=torch.uint8, device="cuda"), torch.empty(m.monta_rmsnorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    m.monta_ws_init(cfg, ws)
    m.monta_rmsnorm(cfg, x, res, w, EPS, s, out)
    m.monta_gate(cfg, out, wg, logits)
    m.monta_route_dispatch_regather(cfg, logits, out, idx, gates, stage, final, ws)
    m.monta_expert_linear(cfg, final, we, N, y, ws)
    m.monta_combine(cfg, y, gates, o, ws)
    m.monta_combine_backward(cfg, dout, y, gates, dy, dgates, ws)
    m.monta_expert_linear_backward(cfg, dy, final, we, N, dfinal, dw_e, ws)
    m.monta_combine(cfg, dfinal, ones, dn, ws)
    m.monta_rmsnorm_backward(cfg, s, w, EPS, dn, dsum, dx, dw, scratch)
    torch.cuda.synchronize()
    pos = torch.from_numpy(buffers.read_tables(cfg, ws)["pos_final"]).cuda().long()
    t, j = (pos >= 0).nonzero(as_tuple=True)

    # the same in 64 bits, by autograd from the stored sum
    leaf = lambda v: v.double().requires_grad_()  # noqa: E731
    s64, w64, we64, g64 = leaf(s), leaf(w), leaf(we), leaf(gates)
    n64 = s64 / ((s64 ** 2).mean(1, keepdim=True) + EPS).sqrt() * w64
    want = torch.zeros((T, N), dtype=torch.float64, device="cuda")
    for e in range(E):
        sel = idx[t, j] == e
        want = want.index_add(0, t[sel], g64[t[sel], j[sel]][:, None] * (n64[t[sel]] @ we64[e].T))
    (want * dout.double()).sum().backward()

    # chains of magnitudes
    nm, d, gd = n64.detach().abs(), dout.double().abs(), gates.double()
    om, dgm, dnm, dwm = (torch.zeros(q, dtype=torch.float64, device="cuda") for q in ((T, N), (T, k), (T, H), (E, N, H)))
    for e in range(E):
        sel = idx[t, j] == e
        ts, gs, wm = t[sel], gd[t[sel], j[sel]][:, None], we[e].double().abs()
        ym = nm[ts] @ wm.T
        om.index_add_(0, ts, gs * ym)
        dgm[ts, j[sel]] = (d[ts] * ym).sum(1)
        dnm.index_add_(0, ts, gs * d[ts] @ wm)
        dwm[e] = (gs * d[ts]).T @ nm[ts]
    r = 1 / ((s.double() ** 2).mean(1, keepdim=True) + EPS).sqrt()
    sm, gm = s.double().abs(), dnm * w.double().abs()
    dxm = r * (gm + sm * r ** 2 * (gm * sm).mean(1, keepdim=True)) + dsum.double().abs()
    adds, h = (2 * H + 2 * N + T + 400) * U, half(dtype)
    for name, got, ref, mag, roundings in (
            ("out", o, want.detach(), om, 3), ("dgates", dgates, g64.grad, dgm, 2), ("dw_exp", dw_e, we64.grad, dwm, 3),
            ("dweight", dw, w64.grad, (dnm * sm * r).sum(0), 4), ("dx", dx, s64.grad + dsum.double(), dxm, 5)):
        off = (got.double() - ref).abs()
        assert bool((off <= (adds + roundings * h * 1.05) * mag).all()), (name, (off / mag.clamp_min(1e-300)).max().item())


def test_two_streams(m):  # noqa: F811
    """Two layers at once, each on a stream of its own, one handed over by the argument and one the current one; the results are those of the calls one after
    the other."""
    import torch
    from test_gpu_expert8 import problem, routed
    made = []
    for T, H, N, E, seed in ((700, 512, 520, 4, 1), (90, 1040, 264, 8, 2)):
        cfg, ws, _, rows = routed(m, T, H, "bf16", E, 2, seed=seed)
        packed, wc, wsc, _, _ = problem(m, cfg, rows, N, False, seed)
        a = torch.bfloat16
        t = dict(x=normal((T, H), a, seed), w=normal((H,), a, seed + 10), dy=normal((rows, N), a, seed + 20), fin=normal((rows, H), a, seed + 30),
                 we=normal((E, N, H), a, seed + 40), gates=normal((T, 2), torch.float32, seed + 50))
        new = lambda *s, d=a: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
        out = dict(n=new(T, H), r8=new(T, m.monta_fp8_rows(cfg)[1], d=torch.uint8), y=new(rows, N), dx=new(rows, H), dw=new(E, N, H),
                   dfin=new(rows, H), dg=new(T, 2, d=torch.float32), dn=new(T, H), dnw=new(H, d=torch.float32))
        scratch = new(m.monta_rmsnorm_scratch_bytes(cfg), d=torch.uint8)

        def calls(stream, cfg=cfg, ws=ws, packed=packed, wc=wc, wsc=wsc, t=t, out=out, N=N, scratch=scratch):
            m.monta_rmsnorm(cfg, t["x"], None, t["w"], EPS, None, out["n"], out["r8"], stream=stream)
            m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, out["y"], ws, stream=stream)
            m.monta_combine_backward(cfg, t["x"], t["fin"], t["gates"], out["dfin"], out["dg"], ws, stream=stream)
            m.monta_expert_linear_backward(cfg, t["dy"], t["fin"], t["we"], N, out["dx"], out["dw"], ws, stream=stream)
            m.monta_rmsnorm_backward(cfg, t["x"], t["w"], EPS, out["n"], None, out["dn"], out["dnw"], scratch, stream=stream)

        calls(None)
        torch.cuda.synchronize()
        made.append((calls, out, {k: v.clone() for k, v in out.items()}))
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for _, out, _ in made:
            for v in out.values():
                v.zero_()
        torch.cuda.synchronize()
        made[0][0](side.cuda_stream)
        with torch.cuda.stream(other):
            made[1][0](None)
        torch.cuda.synchronize()
        for _, out, want in made:
            assert all(torch.equal(out[k], want[k]) for k in want), [k for k in want if not torch.equal(out[k], want[k])]
