"""GPU: what the norm makes of infinities, NaN and magnitudes whose squares are no fp32 numbers, as its documentation says, for every
number of lanes that a row has."""
import pytest

from test_gpu_norm import FLOOR_SCALE, dt, m, normal, run_norm, split  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [80, 496, 1040, 2064, 7168, 16384])
def test_rows_out_of_the_ordinary(m, H, dtype):  # noqa: F811
    import torch
    H = H // 2 // 16 * 16 if dtype == "f32" else H
    at = H // 2 + 1
    x, res = normal(9, H, dtype, 1), normal(9, H, dtype, 2)
    w = torch.full((H,), 1.5, device="cuda", dtype=dt(dtype))
    base = run_norm(m, x, res, w, dtype)
    x[1, at] = float("nan")
    x[3, at] = float("-inf")
    x[5, at], res[5, at] = float("inf"), float("-inf")          # their sum is NaN
    x[7], res[7] = 0, 0
    s, out, rows = run_norm(m, x, res, w, dtype)
    for t in (0, 2, 4, 6, 8):
        assert all(torch.equal(a[t], b[t]) for a, b in zip((s, out, rows), base)), t
    codes, scales = split(rows, H)
    rest = torch.arange(H, device="cuda") != at
    for t in (1, 5):
        assert bool(torch.isnan(out[t]).all()) and bool(torch.isnan(codes[t]).all())
    assert bool(torch.isnan(out[3, at])) and bool(torch.isnan(codes[3, at])) and bool((out[3][rest] == 0).all()) and bool((codes[3][rest] == 0).all())
    assert bool((out[7] == 0).all()) and bool((codes[7] == 0).all()) and bool((scales[7] == FLOOR_SCALE).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [16, 528, 4112])
def test_eps_of_zero(m, H, dtype):  # noqa: F811
    """Zeros: NaN; squares that are all zero: infinities where the row is not; and of large and small rows the norm is that of the row at scale one."""
    import torch
    cfg = m.make_cfg(5, H, m.FP32 if dtype == "f32" else m.BF16, 1, 1, 1, 1, 1)
    w = torch.ones(H, device="cuda", dtype=dt(dtype))
    x = normal(1, H, dtype, 3).expand(5, H).contiguous()
    x[0] *= 2.0 ** 50
    x[1] *= 2.0 ** -40
    x[3] = 0
    x[4] = 0
    x[4, ::2] = -2.0 ** -80
    out = torch.empty_like(x)
    m.monta_rmsnorm(cfg, x, None, w, 0.0, None, out)
    torch.cuda.synchronize()
    # a power of two changes no rounding: squares and their sums stay above the subnormal fp32 numbers, but for values below 2^-23 of the largest
    u = 2.0 ** -24
    for t in (0, 1):
        assert bool(((out[t].double() - out[2].double()).abs() <= out[2].double().abs() * (2 * u if dtype == "f32" else 2.0 ** -7)).all()), t
    assert bool(torch.isnan(out[3]).all())
    assert bool((out[4, ::2] == float("-inf")).all()) and bool(torch.isnan(out[4, 1::2]).all())
