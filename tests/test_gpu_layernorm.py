"""GPU parity of the layer norm, its 8-bit rows and its gradient against 64 bits.

Bars, with u = 2^-24 (half a step of fp32), h = eps / 2 of the activation type, A the mean magnitude of a row, s its spread, r = 1 / s:
  - a row's sums run over at most 16 elements of a lane, 6 moves between lanes and 4 between waves: fewer than 40 additions, so the mean is
    off by at most 40 u A, as is the mean of a wave's share;
  - the sum of squares has that error of the shares' means once (2 times 40 u A / s of it) and 44 u from squaring and adding: r is off by
    (22 + 80 A r) u;
  - v = (s - m) r w + b: 40 u A r |w| from the mean, then r, the difference, two products and a sum;
  - outputs of the activation type are rounded once more: h; a code is off by half a step of e4m3, 2^-4 of the value, or 2^-10 of the
    scale below the smallest normal number;
  - dx has r up to three times over and two more means: 3 (22 + 80 A r) + 40 + 14 u of the sum of its terms' magnitudes;
  - the gradients of weight and bias add up a term per token, in chains of tokens / 512 rows, 16 groups, 32 + 16 partial sums.
"""
import pytest

from test_gpu_norm import FLOOR, FLOOR_SCALE, U, dt, half, m, make, normal, split  # noqa: F401

pytestmark = pytest.mark.gpu


def run_norm(m, x, residual, w, b, dtype, eps=1e-5, fp8=True, out=True):  # noqa: F811
    import torch
    T, H = x.shape
    cfg = make(m, T, H, dtype)
    s = torch.full_like(x, 7.0) if residual is not None else None
    o = torch.full((T + 1, H), 7.0, device="cuda", dtype=x.dtype) if out else None
    rows = torch.full((T + 1, m.monta_fp8_rows(cfg)[1]), 0x5a, dtype=torch.uint8, device="cuda") if fp8 else None
    m.monta_layernorm(cfg, x, residual, w, b, eps, s, o[:T] if out else None, rows[:T] if fp8 else None)
    torch.cuda.synchronize()
    assert not fp8 or bool((rows[T] == 0x5a).all()), "monta_layernorm wrote past the last row"
    assert not out or bool((o[T] == 7.0).all()), "monta_layernorm wrote past the last row"
    return s, o[:T] if out else None, rows[:T] if fp8 else None


def want_norm(x, residual, w, b, eps):
    """-> the sum, v, and how far fp32 may be from v."""
    import torch
    s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    a, w = s.double(), w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    c = a - a.mean(1, keepdim=True)
    r = 1 / ((c ** 2).mean(1, keepdim=True) + eps).sqrt()
    far = a.abs().mean(1, keepdim=True) * r
    t = c * r * w
    bar = U * (40 * far * w.abs() + t.abs() * (28 + 80 * far) + 2 * (t.abs() + b.abs()))
    return s, t + b, bar


def check_codes(rows, v, bar):
    import torch
    T, H = v.shape
    codes, scales = split(rows, H)
    nb = -(-H // 128)
    pad, worst = torch.zeros((2, T, nb * 128), dtype=torch.float64, device="cuda")
    pad[:, :H], worst[:, :H] = v.abs(), bar
    amax, off = pad.view(T, nb, 128).amax(2).clamp_min(FLOOR), worst.view(T, nb, 128).amax(2)
    assert bool(((scales - amax / 448).abs() <= (amax * 4 * U + off) / 448).all())
    sc = scales.repeat_interleave(128, 1)[:, :H]
    assert bool(((codes * sc - v).abs() <= torch.maximum(v.abs() * 2.0 ** -4, sc * 2.0 ** -10) + 2 * bar + v.abs() * 8 * U).all())
    assert bool((codes.abs() <= 448).all())


def params(H, dtype, seed):
    return (1 + 0.3 * normal(1, H, "f32", seed)[0]).to(dt(dtype)), (0.2 * normal(1, H, "f32", seed + 1)[0]).to(dt(dtype))


# every number of lanes of a row, waves without a vector, waves with a few
SIZES = [(1, 16), (1, 4096), (3, 128), (5, 112), (17, 256), (33, 528), (9, 1040), (7, 2048), (300, 512), (4, 5120), (3, 7168), (2, 8192), (2100, 96),
         (4500, 16), (3, 4112), (5, 2064), (40, 192), (9, 320), (1030, 384), (21, 768), (2000, 1024), (11, 1536)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H", SIZES + [(2, 16384)])
@pytest.mark.parametrize("residual", [0, 1])
def test_norm(m, T, H, dtype, residual):  # noqa: F811
    import torch
    if dtype == "f32" and H > 8192:
        pytest.skip("rows beyond 32 KiB")
    x, res = normal(T, H, dtype, 1, 1.7) + 0.7, normal(T, H, dtype, 2) if residual else None
    w, b = params(H, dtype, 3)
    s, out, rows = run_norm(m, x, res, w, b, dtype)
    want_s, v, bar = want_norm(x, res, w, b, 1e-5)
    if residual:
        assert torch.equal(s, want_s)
    assert bool(((out.double() - v).abs() <= v.abs() * half(dtype) + bar * 1.01).all())
    check_codes(rows, v, bar)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts(m, dtype):  # noqa: F811
    """Each output alone, no bias, and buffers that are the inputs themselves."""
    import torch
    T, H = 37, 656
    x, res = normal(T, H, dtype, 4), normal(T, H, dtype, 5)
    w, b = params(H, dtype, 6)
    s, out, rows = run_norm(m, x, res, w, b, dtype)
    assert torch.equal(run_norm(m, x, res, w, b, dtype, out=False)[2], rows)
    assert torch.equal(run_norm(m, x, res, w, b, dtype, fp8=False)[1], out)
    none, zero = (run_norm(m, x, res, w, bias, dtype) for bias in (None, torch.zeros_like(b)))
    assert all(torch.equal(p, q) for p, q in zip(none, zero))
    cfg = make(m, T, H, dtype)
    for sum_is, out_is in ((0, 1), (1, 0), (1, None), (0, None), (None, 0)):
        bufs = [x.clone(), res.clone()]
        s2 = torch.empty_like(x) if sum_is is None else bufs[sum_is]
        o2 = torch.empty_like(x) if out_is is None else bufs[out_is]
        m.monta_layernorm(cfg, bufs[0], bufs[1], w, b, 1e-5, s2, o2)
        assert torch.equal(s2, s) and torch.equal(o2, out)
    y = x.clone()
    m.monta_layernorm(cfg, y, None, w, b, 1e-5, None, y)
    assert torch.equal(y, run_norm(m, x, None, w, b, dtype)[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [80, 208, 368, 496, 976, 1040, 2064, 7168, 16384])
def test_edges(m, H, dtype):  # noqa: F811
    """Rows of equal numbers, a mean far above the spread, one large value, NaN and infinities that stay in their rows, small and large magnitudes."""
    import torch
    H = H // 2 // 16 * 16 if dtype == "f32" else H
    x = normal(10, H, dtype, 7)
    base = x.clone()
    x[0] = 3.0
    x[1] = 1000.0 + (4.0 if dtype == "bf16" else 1.0) * torch.randint(-2, 3, (H,), device="cuda", generator=torch.Generator("cuda").manual_seed(8))
    x[2] = 0
    x[2, 5] = 300.0
    x[3, 17] = float("nan")
    x[4, H - 1] = float("inf")
    x[5] *= 1e-15
    x[6] *= 1e15
    x[7, 0], x[7, 1] = float("inf"), float("-inf")
    w, b = torch.ones(H, device="cuda", dtype=x.dtype), torch.zeros(H, device="cuda", dtype=x.dtype)
    _, out, rows = run_norm(m, x, None, w, b, dtype)
    _, v, bar = want_norm(x, None, w, b, 1e-5)
    good = [0, 1, 2, 5, 6, 8, 9]
    assert bool(((out.double() - v).abs() <= v.abs() * half(dtype) + bar * 1.01)[good].all())
    check_codes(rows[good], v[good], bar[good])
    codes, scales = split(rows, H)
    # a sum of H equal numbers of 2 bits is exact
    assert bool((out[0] == 0).all()) and bool((codes[0] == 0).all()) and bool((scales[0] == FLOOR_SCALE).all())
    for t in (3, 4, 7):
        assert bool(torch.isnan(out[t]).all()) and bool(torch.isnan(codes[t]).all())
    ref = run_norm(m, base, None, w, b, dtype)
    assert all(torch.equal(p[t], q[t]) for p, q in zip((out, rows), ref[1:]) for t in (8, 9))
    zero = make(m, 10, H, dtype)
    o = torch.empty_like(x)
    m.monta_layernorm(zero, x, None, w, b, 0.0, None, o)
    torch.cuda.synchronize()
    assert bool(torch.isnan(o[0]).all()) and bool(torch.isfinite(o[[1, 2, 5, 6, 8, 9]]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dsum", [0, 1])
@pytest.mark.parametrize("T,H", SIZES + [(513, 4096), (1500, 520), (2, 16384), (1, 8192), (4, 4096), (5, 4096), (8, 1024), (9, 1024), (63, 128), (65, 120), (1155, 1040), (1100, 1536), (600, 4096), (1030, 768)])
def test_backward(m, T, H, dtype, dsum):  # noqa: F811
    import torch
    if dtype == "f32" and H > 8192:
        pytest.skip("rows beyond 32 KiB")
    eps = 1e-5
    s, d = normal(T, H, dtype, 11, 1.5) - 0.6, normal(T, H, dtype, 12)
    w, _ = params(H, dtype, 13)
    t = normal(T, H, dtype, 15) if dsum else None
    cfg = make(m, T, H, dtype)
    dx = torch.full((T + 1, H), 9.0, device="cuda", dtype=s.dtype)
    dw, db = (torch.full((H + 1,), 9.0, device="cuda") for _ in range(2))
    scratch = torch.empty(m.monta_layernorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda")
    m.monta_layernorm_backward(cfg, s, w, eps, d, t, dx[:T], dw[:H], db[:H], scratch)
    torch.cuda.synchronize()
    assert dw[H].item() == 9.0 and db[H].item() == 9.0 and bool((dx[T] == 9.0).all())
    dx = dx[:T]
    a, b = s.double(), d.double()
    g, c = b * w.double(), a - a.mean(1, keepdim=True)
    r = 1 / ((c ** 2).mean(1, keepdim=True) + eps).sqrt()
    n, far = c * r, a.abs().mean(1, keepdim=True) * r
    want = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) + (t.double() if dsum else 0)
    # (s - m) is off by 40 u A: its share of n, and of the mean of g n
    mag = r * (g.abs() + g.abs().mean(1, keepdim=True) + (n.abs() + 1) * ((g * n).abs().mean(1, keepdim=True) + g.abs().mean(1, keepdim=True)))
    mag = mag + (t.double().abs() if dsum else 0)
    assert bool(((dx.double() - want).abs() <= want.abs() * half(dtype) + mag * (120 + 320 * far) * U).all())
    chain = T // 512 + 120
    for got, terms, bar in ((dw, b * n, (b * n).abs() * (chain + 28 + 80 * far) + b.abs() * 40 * far), (db, b, b.abs() * chain)):
        assert bool(((got[:H].double() - terms.sum(0)).abs() <= U * bar.sum(0)).all())
    # the same again: a fixed order of additions; without the bias's gradient; and in place
    dw2, bufs = torch.empty(H, device="cuda"), [s.clone(), d.clone()] + ([t.clone()] if dsum else [])
    for at in range(len(bufs)):
        u, db2 = [v.clone() for v in bufs], torch.empty(H, device="cuda") if at == 0 else None
        m.monta_layernorm_backward(cfg, u[0], w, eps, u[1], u[2] if dsum else None, u[at], dw2, db2, scratch)
        assert torch.equal(u[at], dx) and torch.equal(dw2, dw[:H]) and (at or torch.equal(db2, db[:H]))


def test_backward_against_differences(m):  # noqa: F811
    """fp32: the gradients against central differences of the norm itself, in 64 bits."""
    import torch
    T, H, eps, step = 3, 64, 1e-3, 1e-4
    s, d = normal(T, H, "f32", 21), normal(T, H, "f32", 22)
    w, b = params(H, "f32", 23)
    cfg = make(m, T, H, "f32")
    dx, dw, db = torch.empty_like(s), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    m.monta_layernorm_backward(cfg, s, w, eps, d, None, dx, dw, db, torch.empty(m.monta_layernorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))

    def loss(a, g, c):
        n = a - a.mean(1, keepdim=True)
        return ((n / ((n ** 2).mean(1, keepdim=True) + eps).sqrt() * g + c) * d.double()).sum(1)

    a, g, c = s.double(), w.double(), b.double()
    for h in (0, 13, 63):
        e = torch.zeros(H, dtype=torch.float64, device="cuda")
        e[h] = step
        # third derivatives of the norm are below 50 here (values of about 1, eps 1e-3): the difference is within 50 step^2 / 6 of it
        assert bool((((loss(a + e, g, c) - loss(a - e, g, c)) / (2 * step) - dx[:, h].double()).abs() <= 1e-6).all())
        assert abs(((loss(a, g + e, c) - loss(a, g - e, c)).sum() / (2 * step) - dw[h].double()).item()) <= 1e-6
        assert abs(((loss(a, g, c + e) - loss(a, g, c - e)).sum() / (2 * step) - db[h].double()).item()) <= 1e-6


def test_streamed(m):  # noqa: F811
    """From 192 MiB on rows are streamed past the cache: the same bits, whatever the number of rows, and rows beyond 2^31 bytes."""
    import torch
    for dtype, H in (("bf16", 4096), ("f32", 520)):
        part, T = 1000, (1 << 29) // (H * (2 if dtype == "bf16" else 4))
        x, d = normal(part, H, dtype, 31).repeat(T // part, 1), normal(part, H, dtype, 32).repeat(T // part, 1)
        w, b = params(H, dtype, 33)
        small, large = make(m, part, H, dtype), make(m, x.shape[0], H, dtype)
        outs = []
        for cfg in (small, large):
            n = cfg.tokens
            o, dx = torch.empty_like(x[:n]), torch.empty_like(x[:n])
            dw, db = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
            m.monta_layernorm(cfg, x[:n], None, w, b, 1e-5, None, o)
            m.monta_layernorm_backward(cfg, x[:n], w, 1e-5, d[:n], None, dx, dw, db,
                                       torch.empty(m.monta_layernorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))
            outs.append((o, dx))
        for a, c in zip(*outs):
            assert bool((c.view(-1, part, H) == a).all())
    T, H = 70000, 16384                                # 2.3 GB of rows
    x = normal(1, H, "bf16", 45).expand(T, H).contiguous()
    w, b = params(H, "bf16", 46)
    m.monta_layernorm(make(m, T, H, "bf16"), x, None, w, b, 1e-5, None, x)
    torch.cuda.synchronize()
    assert bool((x == x[0]).all()) and bool((x[0] != 0).any())
