"""GPU: the layer norm and its gradient from 192 MiB on, whose rows are streamed past the cache: every output, the weight's and the bias's gradients
among them, with many rounds of rows in a workgroup; and the gradient of rows beyond 2^31 bytes.

The large batch is a small one over and over: rows have the same bits; the gradients of weight and bias are that many times the small one's sums in 64 bits, with
bars as in test_gpu_layernorm: a term has the errors of its normalised element, (28 + 80 F) u of it and 40 F u of the output's gradient with F = A r, and a chain of
tokens / 256 rows (one row a workgroup of 256), 120 more for groups and partial sums."""
import pytest

from test_gpu_layernorm import make, params, run_norm
from test_gpu_norm import U, m, normal  # noqa: F401

pytestmark = pytest.mark.gpu


def gradient(m, x, w, d, t, dtype, in_place=False):  # noqa: F811
    import torch
    T, H = x.shape
    cfg = make(m, T, H, dtype)
    dx, dw, db = d if in_place else torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    m.monta_layernorm_backward(cfg, x, w, 1e-5, d, t, dx, dw, db, torch.empty(m.monta_layernorm_scratch_bytes(cfg), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return dx, dw, db


def check_params(x, d, dw, db, times):
    a, b, T = x.double(), d.double(), x.shape[0] * times
    c = a - a.mean(1, keepdim=True)
    r = 1 / ((c ** 2).mean(1, keepdim=True) + 1e-5).sqrt()
    n, far, chain = c * r, a.abs().mean(1, keepdim=True) * r, T // 256 + 120
    for got, terms, bar in ((dw, b * n, (b * n).abs() * (chain + 28 + 80 * far) + b.abs() * 40 * far), (db, b, b.abs() * chain)):
        assert bool(((got.double() - terms.sum(0) * times).abs() <= U * bar.sum(0) * times).all())


@pytest.mark.parametrize("dsum", [0, 1])
@pytest.mark.parametrize("dtype,part,times,H", [("bf16", 1000, 9, 4096), ("bf16", 997, 17, 2048), ("bf16", 1000, 68, 512), ("bf16", 500, 9, 8192), ("bf16", 1003, 300, 120),
                                                ("f32", 1000, 34, 520), ("f32", 1001, 9, 2048), ("f32", 300, 9, 8192)])
def test_streamed_batches(m, dtype, part, times, H, dsum):  # noqa: F811
    import torch
    x, res, d, t = (normal(part, H, dtype, seed) for seed in (1, 2, 3, 4))
    w, b = params(H, dtype, 5)
    fp8 = H % 16 == 0
    many = [v.repeat(times, 1) for v in (x, res, d, t)]
    small, large = run_norm(m, x, res, w, b, dtype, fp8=fp8), run_norm(m, many[0], many[1], w, b, dtype, fp8=fp8)
    assert many[0].numel() * many[0].element_size() * 3 >= 192 << 20
    for one, all_ in zip(small, large):
        assert one is None or bool((all_.reshape(times, part, -1).view(torch.uint8) == one.reshape(part, -1).view(torch.uint8)).all())
    got = gradient(m, x, w, d, t if dsum else None, dtype)
    dx, dw, db = gradient(m, many[0], w, many[2], many[3] if dsum else None, dtype)
    assert bool((dx.view(times, part, H) == got[0]).all())
    check_params(x, d, got[1], got[2], 1)
    check_params(x, d, dw, db, times)


@pytest.mark.parametrize("dtype,H", [("bf16", 16384), ("f32", 1024)])
def test_gradient_beyond_2gib(m, dtype, H):  # noqa: F811
    """2.3 GB of rows, in place, and the last rows other ones than the first."""
    import torch
    part, times = 1000, 70 if dtype == "bf16" else 560
    x, d = normal(part, H, dtype, 7), normal(part, H, dtype, 8)
    w, _ = params(H, dtype, 9)
    want = gradient(m, x, w, d, None, dtype)[0]
    dx, dw, db = gradient(m, x.repeat(times, 1), w, d.repeat(times, 1), None, dtype, in_place=True)
    assert dx.numel() * dx.element_size() > 1 << 31 and bool((dx.view(times, part, H) == want).all())
    check_params(x, d, dw, db, times)
