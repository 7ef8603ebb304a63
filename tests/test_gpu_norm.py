"""GPU parity of the root-mean-square norm, its 8-bit rows, its gradient, and the gradient of the combine, against 64 bits.

Bars, with u = 2^-24 (half a step of fp32) and h = eps / 2 of the activation type:
  - a row's sums run over at most 16 elements of a lane, 6 moves between lanes and 16 waves: fewer than 40 additions, so a sum is within
    40 u of the sum of its terms' magnitudes; the norm takes half of that (a square root), a division, a root and two products: 24 u;
  - outputs of the activation type are rounded once more: h;
  - a code is off by half a step of e4m3: 2^-4 of the value, or 2^-10 of the scale below the smallest normal number (2^-6); the factor
    448 / amax and the value before it are off by 28 u together;
  - the weight's gradient adds up a row of terms per token, in chains of tokens / 512 rows, 16 groups, 32 + 16 partial sums.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
FLOOR = 2.0 ** -40
FLOOR_SCALE = float(np.float32(FLOOR / 448))          # a scale is an fp32 quotient, rounded once


@pytest.fixture(scope="module")
def m():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_00662_amd as mod
    mod.binding.lib()
    return mod


def dt(name):
    import torch
    return torch.float32 if name == "f32" else torch.bfloat16


def half(name):
    return U if name == "f32" else 2.0 ** -8


def make(m, T, H, dtype, **kw):
    return m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, kw.pop("E", 1), kw.pop("k", 1), 1, 1, 1, **kw)


def normal(T, H, dtype, seed, scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((T, H), generator=g, device="cuda") * scale).to(dt(dtype))


def run_norm(m, x, residual, w, dtype, eps=1e-5, fp8=True, out=True):
    import torch
    T, H = x.shape
    cfg = make(m, T, H, dtype)
    s = torch.full_like(x, 7.0) if residual is not None else None
    o = torch.full_like(x, 7.0) if out else None
    rows = torch.full((T + 1, m.monta_fp8_rows(cfg)[1]), 0x5a, dtype=torch.uint8, device="cuda") if fp8 else None
    m.monta_rmsnorm(cfg, x, residual, w, eps, s, o, rows[:T] if fp8 else None)
    torch.cuda.synchronize()
    if fp8:
        assert bool((rows[T] == 0x5a).all()), "monta_rmsnorm wrote past the last row"
    return s, o, rows[:T] if fp8 else None


def split(rows, H):
    """Packed rows -> (codes as fp64, scales as fp64), after a look at the zeros behind them."""
    import torch
    nb = -(-H // 128)
    assert bool((rows[:, H + 4 * nb:] == 0).all())
    return (rows[:, :H].contiguous().view(torch.float8_e4m3fn).to(torch.float64),
            rows[:, H:H + 4 * nb].contiguous().view(torch.float32).to(torch.float64))


def want_norm(x, residual, w, eps):
    import torch
    s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    s64 = s.double()
    v = s64 / ((s64 ** 2).mean(1, keepdim=True) + eps).sqrt() * w.double()
    return s, v


SIZES = [(1, 16), (1, 4096), (3, 128), (5, 112), (17, 256), (33, 528), (9, 1040), (7, 2048), (300, 512), (4, 5120), (3, 7168), (2, 8192), (2100, 96),
         (4500, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", SIZES + [(2, 16384)])
@pytest.mark.parametrize("residual", [0, 1])
def test_norm(m, T, H, dtype, residual):
    import torch
    if dtype == "f32" and H > 8192:
        pytest.skip("rows beyond 32 KiB")
    x, r = normal(T, H, dtype, 1, 1.7), normal(T, H, dtype, 2) if residual else None
    w = 1 + 0.3 * normal(1, H, "f32", 3)[0]
    w = w.to(x.dtype)
    s, out, rows = run_norm(m, x, r, w, dtype)
    want_s, v = want_norm(x, r, w, 1e-5)
    if residual:
        assert torch.equal(s, want_s)
    assert bool(((out.double() - v).abs() <= v.abs() * (half(dtype) + 28 * U)).all())
    codes, scales = split(rows, H)
    nb = -(-H // 128)
    pad = torch.zeros((T, nb * 128), dtype=torch.float64, device="cuda")
    pad[:, :H] = v.abs()
    amax = pad.view(T, nb, 128).amax(2).clamp_min(FLOOR)
    assert bool(((scales - amax / 448).abs() <= amax / 448 * 28 * U).all())
    sc = scales.repeat_interleave(128, 1)[:, :H]
    assert bool(((codes * sc - v).abs() <= torch.maximum(v.abs() * 2.0 ** -4, sc * 2.0 ** -10) + v.abs() * 32 * U).all())
    assert bool((codes.abs() <= 448).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_parts(m, dtype):
    """Each output alone, and buffers that are the inputs themselves."""
    import torch
    T, H = 37, 656
    x, r, w = normal(T, H, dtype, 4), normal(T, H, dtype, 5), normal(1, H, dtype, 6)[0].contiguous()
    s, out, rows = run_norm(m, x, r, w, dtype)
    assert torch.equal(run_norm(m, x, r, w, dtype, out=False)[2], rows)
    assert torch.equal(run_norm(m, x, r, w, dtype, fp8=False)[1], out)
    cfg = make(m, T, H, dtype)
    for sum_is, out_is in ((0, 1), (1, 0), (1, None), (0, None), (None, 0)):
        bufs = [x.clone(), r.clone()]
        s2 = torch.empty_like(x) if sum_is is None else bufs[sum_is]
        o2 = torch.empty_like(x) if out_is is None else bufs[out_is]
        m.monta_rmsnorm(cfg, bufs[0], bufs[1], w, 1e-5, s2, o2)
        assert torch.equal(s2, s) and torch.equal(o2, out)
    y = x.clone()
    m.monta_rmsnorm(cfg, y, None, w, 1e-5, None, y)
    assert torch.equal(y, run_norm(m, x, None, w, dtype)[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_edges(m, dtype):
    """Rows of zeros, tiny blocks, a single large value, NaN and infinities that stay in their rows, the smallest and largest magnitudes."""
    import torch
    T, H = 8, 272
    x = normal(T, H, dtype, 7)
    x[0] = 0
    x[1, 128:256] = 1e-20                              # a block below the floor of the scales
    x[2] = 0
    x[2, 5] = 3.0
    x[3, 17] = float("nan")
    x[4, 200] = float("inf")
    x[5] *= 1e-15                                      # squares of 1e-30: the mean is far below eps
    x[6] *= 1e15
    w = torch.ones(H, device="cuda", dtype=x.dtype)
    _, out, rows = run_norm(m, x, None, w, dtype)
    _, v = want_norm(x, None, w, 1e-5)
    codes, scales = split(rows, H)
    for t in (0, 1, 2, 5, 6, 7):
        assert bool(((out[t].double() - v[t]).abs() <= v[t].abs() * (half(dtype) + 28 * U)).all()), t
        assert bool(torch.isfinite(codes[t]).all()) and bool(torch.isfinite(scales[t]).all())
        sc = scales[t].repeat_interleave(128)[:H]
        assert bool(((codes[t] * sc - v[t]).abs() <= torch.maximum(v[t].abs() * 2.0 ** -4, sc * 2.0 ** -10) * (1 + 2.0 ** -17)).all()), t
    assert bool((out[0] == 0).all()) and bool((codes[0] == 0).all()) and bool((scales[0] == FLOOR_SCALE).all())
    assert scales[1, 1].item() == FLOOR_SCALE
    assert bool(torch.isnan(out[3]).all()) and bool(torch.isnan(codes[3]).all())
    assert bool(torch.isnan(out[4, 200])) and bool(torch.isnan(codes[4, 200]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dsum", [0, 1])
@pytest.mark.parametrize("T,H", SIZES + [(513, 4096), (1500, 520), (2, 16384)])
def test_norm_backward(m, T, H, dtype, dsum):
    import torch
    if dtype == "f32" and H > 8192:
        pytest.skip("rows beyond 32 KiB")
    eps = 1e-5
    s, d, w = normal(T, H, dtype, 11, 1.5), normal(T, H, dtype, 12), (1 + 0.3 * normal(1, H, "f32", 13)[0]).to(dt(dtype))
    t = normal(T, H, dtype, 14) if dsum else None
    cfg = make(m, T, H, dtype)
    dx, dw = torch.full_like(s, 9.0), torch.full((H + 1,), 9.0, device="cuda")
    scratch = torch.empty(m.monta_rmsnorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    m.monta_rmsnorm_backward(cfg, s, w, eps, d, t, dx, dw[:H], scratch)
    torch.cuda.synchronize()
    assert dw[H].item() == 9.0
    a, b, g = s.double(), d.double(), d.double() * w.double()
    r = 1 / ((a ** 2).mean(1, keepdim=True) + eps).sqrt()
    proj = (g * a).mean(1, keepdim=True) * r ** 2
    want = r * (g - a * proj) + (t.double() if dsum else 0)
    mag = r * (g.abs() + a.abs() * r ** 2 * (g * a).abs().mean(1, keepdim=True)) + (t.double().abs() if dsum else 0)
    assert bool(((dx.double() - want).abs() <= want.abs() * half(dtype) + mag * 96 * U).all())
    terms = b * a * r
    assert bool(((dw[:H].double() - terms.sum(0)).abs() <= (T // 512 + 120) * U * terms.abs().sum(0)).all())
    # the same again: a fixed order of additions; and in place
    dw2, bufs = torch.empty(H, device="cuda"), [s.clone(), d.clone()] + ([t.clone()] if dsum else [])
    for at in range(len(bufs)):
        c = [u.clone() for u in bufs]
        m.monta_rmsnorm_backward(cfg, c[0], w, eps, c[1], c[2] if dsum else None, c[at], dw2, scratch)
        assert torch.equal(c[at], dx) and torch.equal(dw2, dw[:H])


def test_norm_backward_against_differences(m):
    """fp32: the gradients against central differences of the norm itself, in 64 bits."""
    import torch
    T, H, eps, step = 3, 64, 1e-3, 1e-4
    s, d, w = normal(T, H, "f32", 21), normal(T, H, "f32", 22), 1 + 0.2 * normal(1, H, "f32", 23)[0]
    cfg = make(m, T, H, "f32")
    dx, dw = torch.empty_like(s), torch.empty(H, device="cuda")
    m.monta_rmsnorm_backward(cfg, s, w, eps, d, None, dx, dw, torch.empty(m.monta_rmsnorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))

    def loss(a, g):
        return (a / ((a ** 2).mean(1, keepdim=True) + eps).sqrt() * g * d.double()).sum(1)

    a, g = s.double(), w.double()
    for h in (0, 13, 63):
        e = torch.zeros(H, dtype=torch.float64, device="cuda")
        e[h] = step
        # third derivatives of the norm are below 50 here (values of about 1, eps 1e-3): the difference is within 50 step^2 / 6 of it
        assert bool((((loss(a + e, g) - loss(a - e, g)) / (2 * step) - dx[:, h].double()).abs() <= 1e-6).all())
        assert abs(((loss(a, g + e) - loss(a, g - e)).sum() / (2 * step) - dw[h].double()).item()) <= 1e-6


def routed(m, T, H, dtype, E, k, cf, padded=0, seed=31):
    import torch
    from paper_2411_00662_amd import buffers
    cfg = m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, E, k, 1, 1, 1, cf, 1, padded)
    b = m.alloc_buffers(cfg, np.random.default_rng(seed).normal(size=(T, E)).astype(np.float32))
    m.monta_route(cfg, b.logits, b.topk_idx, b.gates, b.ws)
    torch.cuda.synchronize()
    return cfg, b, buffers.read_tables(cfg, b.ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,E,k,cf,padded", [
    (1, 16, 1, 1, 0.0, 0), (1, 4096, 8, 2, 0.0, 0), (5, 128, 4, 4, 0.0, 0), (64, 40, 8, 3, 0.5, 0), (257, 528, 16, 8, 0.75, 1), (40, 1040, 64, 32, 1.0, 0),
    (33, 2048, 8, 2, 2.0, 1), (9, 5120, 4, 1, 0.3, 0), (6, 8192, 8, 2, 0.0, 0), (700, 96, 6, 5, 0.9, 0)])
def test_combine_backward(m, T, H, E, k, cf, padded, dtype):
    import torch
    cfg, b, tabs = routed(m, T, H, dtype, E, k, cf, padded)
    rows = b.final.shape[0]
    pos = torch.from_numpy(tabs["pos_final"]).cuda().long()
    y, d = normal(rows, H, dtype, 32), normal(T, H, dtype, 33)
    live = pos >= 0
    used = torch.zeros(rows, dtype=torch.bool, device="cuda")
    used[pos[live]] = True
    y[~used] = float("nan")                            # rows of no choice are not read ...
    dy, dg = torch.full((rows + 1, H), 5.0, device="cuda", dtype=y.dtype), torch.full((T * k + 1,), 5.0, device="cuda")
    m.monta_combine_backward(cfg, d, y, b.gates, dy[:rows], dg[:T * k].view(T, k), b.ws)
    torch.cuda.synchronize()
    assert bool((dy[:rows][~used] == 5.0).all()) and bool((dy[rows] == 5.0).all()) and dg[T * k].item() == 5.0        # ... nor written
    got = dg[:T * k].view(T, k).double()
    assert bool((got[~live] == 0).all())
    t, j = live.nonzero(as_tuple=True)
    at = pos[t, j]
    terms = d[t].double() * y[at].double()
    assert bool(((got[t, j] - terms.sum(1)).abs() <= 48 * U * terms.abs().sum(1)).all())
    want = d[t].double() * b.gates[t, j].double()[:, None]
    assert bool(((dy[at].double() - want).abs() <= want.abs() * (half(dtype) + 2 * U)).all())


def test_graph_streams_and_large_offsets(m):
    """Captured and replayed with eager work between the replays; on another stream; rows beyond 2^31 bytes."""
    import torch
    T, H = 2000, 1024
    cfg = make(m, T, H, "bf16")
    w = normal(1, H, "bf16", 41)[0].contiguous()
    x, r, d = normal(T, H, "bf16", 42), normal(T, H, "bf16", 43), normal(T, H, "bf16", 44)
    s, out, dx = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    rows = torch.empty((T, m.monta_fp8_rows(cfg)[1]), dtype=torch.uint8, device="cuda")
    dw, scratch = torch.empty(H, device="cuda"), torch.empty(m.monta_rmsnorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")

    def step():
        m.monta_rmsnorm(cfg, x, r, w, 1e-5, s, out, rows)
        m.monta_rmsnorm_backward(cfg, s, w, 1e-5, d, r, dx, dw, scratch)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (50, 51, 52):
        x.copy_(normal(T, H, "bf16", seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (s, out, rows, dx, dw)]
        for t in (s, out, rows, dx, dw):
            t.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (s, out, rows, dx, dw)))
    del graph
    T, H = 70000, 16384                                # 2.3 GB of rows
    x = normal(1, H, "bf16", 45).expand(T, H).contiguous()
    w = normal(1, H, "bf16", 46)[0].contiguous()
    cfg = make(m, T, H, "bf16")
    m.monta_rmsnorm(cfg, x, None, w, 1e-5, None, x)
    torch.cuda.synchronize()
    assert torch.equal(x[0], x[T - 1]) and torch.equal(x[T // 2], x[T - 1]) and bool((x == x[0]).all())


def test_most_tokens(m):
    """2^31 - 1 tokens: the walk's counter passes 2^31."""
    import torch
    T, H = 2 ** 31 - 1, 8
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    cfg = make(m, T, H, "bf16")
    x = torch.ones((T, H), dtype=torch.bfloat16, device="cuda")
    x[-1], x[5] = 3.0, float("nan")
    w = torch.full((H,), 2.0, dtype=torch.bfloat16, device="cuda")
    m.monta_rmsnorm(cfg, x, None, w, 0.0, None, x)
    torch.cuda.synchronize()
    for part in x.split(1 << 28):
        bad = (part != 2.0).any(1)                     # of a row of equal numbers every norm is one
        if part.data_ptr() == x.data_ptr():
            assert bool(bad[5]) and int(bad.sum()) == 1 and bool(torch.isnan(x[5]).all())
        else:
            assert not bool(bad.any())
    del x, part, bad
    torch.cuda.empty_cache()
