"""GPU: the router's losses and gradient of tokens that have no probabilities, and of NaN of either kind."""
import pytest

from test_gpu_router import inputs, m, make, run_grad, run_loss  # noqa: F401

pytestmark = pytest.mark.gpu
# every number of lanes of a token; one workgroup, and several
SIZES = [(3, 2, 1), (300, 4, 2), (5000, 4, 2), (300, 7, 2), (4097, 8, 2), (129, 16, 4), (2050, 33, 8), (8192, 64, 8), (100, 100, 4), (1111, 255, 8)]


@pytest.mark.parametrize("T,E,k", SIZES)
def test_tokens_without_probabilities(m, T, E, k):  # noqa: F811
    """-infinity throughout, NaN throughout or +infinity give NaN in both losses, the means and the token's gradients; masked, nothing."""
    import torch
    logits, idx, gates, dgates, _ = inputs(T, E, k, T + E)
    cfg, one = make(m, T, E, k), torch.ones(2, device="cuda")
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    at = T // 2
    mask[at] = 0
    want = run_loss(m, cfg, logits, idx, mask)
    grad = run_grad(m, cfg, logits, idx, gates, dgates, mask, one, want[1])
    for values in (float("-inf"), float("nan"), None):
        bad = logits.clone()
        if values is None:
            bad[at, E // 2] = float("inf")
        else:
            bad[at] = values
        got = run_loss(m, cfg, bad, idx, None)
        assert bool(torch.isnan(got[0]).all()) and bool(torch.isnan(got[2]).all()), (values, got[0])
        assert got[1][E].item() == T and got[1][:E].sum().item() == T * k
        d = run_grad(m, cfg, bad, idx, gates, dgates, None, one, got[1])
        rest = torch.arange(T, device="cuda") != at
        assert bool(torch.isnan(d[at]).all()) and bool(torch.isfinite(d[rest]).all())
        assert all(torch.equal(a, b) for a, b in zip(run_loss(m, cfg, bad, idx, mask), want))
        assert torch.equal(run_grad(m, cfg, bad, idx, gates, dgates, mask, one, want[1]), grad)


@pytest.mark.parametrize("bits", [0x7f800001, 0x7fa00000, -0x400001, 0x7fc00000, -1])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_any_nan_counts_as_minus_infinity(m, T, E, k, bits):  # noqa: F811
    """Signalling and quiet ones, first in a token's row, last, and between."""
    import torch
    logits, idx, gates, dgates, _ = inputs(T, E, k, T + E, renorm=0)
    cfg, one = make(m, T, E, k, 0), torch.ones(2, device="cuda")
    which = torch.zeros((T, E), dtype=torch.bool, device="cuda")
    t = torch.arange(T, device="cuda")
    which[t, t % E] = True
    which[::3, 0] = which[::5, E - 1] = True
    which[t, (t + 1) % E] = False                      # one logit at least is a number
    nan = torch.where(which, torch.full_like(logits, 0).view(torch.int32) + bits, logits.view(torch.int32)).view(torch.float32)
    none = torch.where(which, float("-inf"), logits)
    got, want = run_loss(m, cfg, nan, idx, None), run_loss(m, cfg, none, idx, None)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool(torch.isfinite(want[0]).all())
    assert torch.equal(run_grad(m, cfg, nan, idx, gates, dgates, None, one, got[1]), run_grad(m, cfg, none, idx, gates, dgates, None, one, got[1]))
