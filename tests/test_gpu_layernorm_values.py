"""GPU: the layer norm and its gradient where a row's mean is far above its spread, against 64 bits.

Bars, with u = 2^-24, h = eps / 2 of the activation type, A the mean magnitude of a row, s its spread, r = 1 / sqrt(s^2 + eps), and fewer than 40 additions to
a sum (16 elements of a lane, 6 moves between lanes, 4 between waves):
  - the first mean is off by e = 40 u A; the second, that of the differences from the first, corrects it: what remains is 40 u of those differences'
    mean magnitude, s + e at most.  Of a normalised element that is 40 u (1 + F) with F = e r = 40 u A r, where the first mean alone leaves F itself;
  - a difference from the mean is off by u of that from the first mean and u of its own: (1 + F) u and |n| u of a normalised one;
  - the squares' sum: 44 u, and twice the differences' errors: 2 (1 + F) u, of which r has a half: (23 + F) u;
  - v = n w + b: |w| (41 + 41 F) u, |n w| (30 + F) u with root, quotient and products, 2 u of both terms;
  - dx = r (g - mean(g) - n mean(g n)) + dsum: each factor's share by the same, in sum below (160 + 90 F) u of the terms' magnitudes.
"""
import pytest

from test_gpu_layernorm import check_codes, make, params, run_norm
from test_gpu_norm import U, dt, half, m, normal  # noqa: F401

pytestmark = pytest.mark.gpu
LEVELS = (10.1, 1234.567, 12345.678, -98765.4)


def level_rows(H, dtype, seed):
    """Of each level: equal numbers; all but one; numbers within 4 steps of each other; and within 1 / 1000 (bf16: 32 steps)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = []
    for a in LEVELS:
        base = torch.full((H,), a, device="cuda").to(dt(dtype))
        one = base.clone()
        step = abs(base[0].item()) * 2.0 ** (-22 if dtype == "f32" else -7)
        one[H // 3] += step
        few = base + step * torch.randint(-2, 3, (H,), generator=g, device="cuda")
        wide = base.float() * (1 + 1e-3 * torch.randn(H, generator=g, device="cuda")) if dtype == "f32" else base + step * torch.randint(-16, 17, (H,), generator=g, device="cuda")
        rows += [r.to(dt(dtype)) for r in (base, one, few, wide)]
    return torch.stack(rows)


def statistics(x, eps):
    a = x.double()
    c = a - a.mean(1, keepdim=True)
    r = 1 / ((c ** 2).mean(1, keepdim=True) + eps).sqrt()
    return c * r, r, 40 * U * a.abs().mean(1, keepdim=True) * r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [64, 128, 256, 528, 768, 1040, 2064, 4096, 8192, 16384])
def test_mean_far_above_the_spread(m, H, dtype):  # noqa: F811
    if dtype == "f32" and H > 8192:
        pytest.skip("rows beyond 32 KiB")
    x = level_rows(H, dtype, H)
    w, b = params(H, dtype, 3)
    _, out, rows = run_norm(m, x, None, w, b, dtype)
    n, r, F = statistics(x, 1e-5)
    t = n * w.double()
    v = t + b.double()
    bar = U * (w.double().abs() * (41 + 41 * F) + t.abs() * (30 + F) + 2 * (t.abs() + b.double().abs()))
    assert bool(((out.double() - v).abs() <= v.abs() * half(dtype) + bar * 1.01).all())
    check_codes(rows, v, bar)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dsum", [0, 1])
@pytest.mark.parametrize("H", [64, 128, 256, 528, 768, 1040, 2064, 4096, 8192, 16384])
def test_gradient_of_a_mean_far_above_the_spread(m, H, dtype, dsum):  # noqa: F811
    if dtype == "f32" and H > 8192:
        pytest.skip("rows beyond 32 KiB")
    check_gradient(m, level_rows(H, dtype, H), dtype, 1e-5, dsum)


def check_gradient(m, x, dtype, eps, dsum, small=False):  # noqa: F811
    import torch
    T, H = x.shape
    d, t = normal(T, H, dtype, 5), normal(T, H, dtype, 6) if dsum else None
    w, _ = params(H, dtype, 7)
    cfg = make(m, T, H, dtype)
    dx, dw, db = torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    m.monta_layernorm_backward(cfg, x, w, eps, d, t, dx, dw, db, torch.empty(m.monta_layernorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    n, r, F = statistics(x, eps)
    # squares below 2^-126 are held to 2^-150 each, and so is their mean: r is off by 2^-150 r^2 of itself
    S = r ** 2 * 2.0 ** -126 if small else 0
    b = d.double()
    g = b * w.double()
    gm, gn = g.abs().mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    want = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True)) + (t.double() if dsum else 0)
    mag = r * (g.abs() + gm + (n.abs() + 1) * (gn + gm)) + (t.double().abs() if dsum else 0)
    assert bool(((dx.double() - want).abs() <= want.abs() * half(dtype) + mag * (160 + 90 * F + 4 * S) * U).all())
    for got, terms, bar in ((dw, b * n, (b * n).abs() * (T // 256 + 120 + 30 + F + S) + b.abs() * (41 + 41 * F)), (db, b, b.abs() * (T // 256 + 120))):
        assert bool(((got.double() - terms.sum(0)).abs() <= U * bar.sum(0)).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [16, 64, 96, 128, 256, 528, 768, 1040, 2064, 4096, 8192])
def test_rows_keep_to_themselves(m, H, dtype):  # noqa: F811
    """Rows with a mean far above their spread, and with a NaN, among others: those have the bits that they have among their like."""
    import torch
    T = 37
    x, d = normal(T, H, dtype, 11), normal(T, H, dtype, 12)
    w, b = params(H, dtype, 13)
    mixed = x.clone()
    mixed[1::4] += 1000
    mixed[7::8, H // 2] = float("nan")
    cfg = make(m, T, H, dtype)
    same = torch.ones(T, dtype=torch.bool, device="cuda")
    same[1::4] = same[7::8] = False
    outs = []
    for s in (x, mixed):
        dx, dw, db = torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        m.monta_layernorm_backward(cfg, s, w, 1e-5, d, None, dx, dw, db, torch.empty(m.monta_layernorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))
        outs.append((run_norm(m, s, None, w, b, dtype, fp8=False)[1], dx, db))
    for one, other in list(zip(*outs))[:2]:
        assert torch.equal(one[same], other[same]) and bool(torch.isnan(other[7::8]).all()) and bool(torch.isfinite(other[1::4]).all())
    assert torch.equal(outs[0][2], outs[1][2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [3e-20, 1e-10, 1e15])
@pytest.mark.parametrize("H", [64, 768, 2064, 8192])
def test_gradient_of_small_and_large_rows(m, H, dtype, scale):  # noqa: F811
    """eps of zero: the square of r is no fp32 number where the spread is below 5e-20, but the gradient is."""
    check_gradient(m, (normal(9, H, "f32", H).double() * scale).to(dt(dtype)), dtype, 0.0, 0, small=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [3e-20, 1e15])
@pytest.mark.parametrize("H", [64, 768, 2064, 8192])
def test_rms_gradient_of_small_and_large_rows(m, H, dtype, scale):  # noqa: F811
    """The same of the norm without a mean, its bars as there."""
    import torch
    x = (normal(9, H, "f32", H).double() * scale).to(dt(dtype))
    d, (w, _) = normal(9, H, dtype, 5), params(H, dtype, 7)
    cfg = make(m, 9, H, dtype)
    dx, dw = torch.empty_like(x), torch.empty(H, device="cuda")
    m.monta_rmsnorm_backward(cfg, x, w, 0.0, d, None, dx, dw, torch.empty(m.monta_rmsnorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    a, b = x.double(), d.double()
    r = 1 / (a ** 2).mean(1, keepdim=True).sqrt()
    n, g, S = a * r, b * w.double(), r ** 2 * 2.0 ** -126
    want = r * (g - n * (g * n).mean(1, keepdim=True))
    mag = r * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= want.abs() * half(dtype) + mag * (160 + 4 * S) * U).all())
    assert bool(((dw.double() - (b * n).sum(0)).abs() <= U * ((b * n).abs() * (150 + S)).sum(0)).all())
