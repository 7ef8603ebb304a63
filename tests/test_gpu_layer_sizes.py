"""Sizes at the ends of what the norm, the experts and their gradients take, against 64 bits."""
import pytest

from test_gpu_norm import half, m, normal  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def needs(gib):
    import torch
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB")


@pytest.fixture(autouse=True)
def _memory_back():
    yield
    import torch
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,H,keep", [(2 ** 26 + 5, 8, 1 << 10), (2 ** 24 + 3, 520, 1 << 8)])
def test_combine_backward_of_many_tokens(m, T, H, keep):  # noqa: F811
    """More tokens than a launch has waves, or workgroups, for.  Every keep-th token and the last one have a row; the tables are laid
    down as a routing leaves them.  Bars as in test_gpu_norm.py."""
    import torch
    needs(32)
    cfg = m.make_cfg(T, H, m.BF16, 1, 1, 1, 1, 1, 1.0 / keep)
    L = m.monta_ws_layout_query(cfg)
    at = torch.cat([torch.arange(0, T - keep + 1, keep, device="cuda"), torch.tensor([T - 1], device="cuda")])
    rows = at.numel()
    assert rows <= L.max_rows
    ws = torch.zeros(L.ws_bytes, dtype=torch.uint8, device="cuda")
    pos = ws[L.off_pos_final:L.off_pos_final + 4 * T].view(torch.int32)
    pos.fill_(-1)
    pos[at] = torch.randperm(rows, device="cuda", dtype=torch.int32)
    row = pos[at].long()
    d = torch.empty((T, H), dtype=torch.bfloat16, device="cuda").normal_()
    y, gates = normal(L.max_rows, H, "bf16", 1), torch.rand((T, 1), device="cuda")
    dy, dg = torch.full_like(y, 5.0), torch.full((T + 1,), 5.0, device="cuda")
    m.monta_combine_backward(cfg, d, y, gates, dy, dg[:T].view(T, 1), ws)
    torch.cuda.synchronize()
    assert dg[T].item() == 5.0 and bool((dy[rows:] == 5.0).all())
    terms = d[at].double() * y[row].double()
    assert bool(((dg[at].double() - terms.sum(1)).abs() <= 48 * U * terms.abs().sum(1)).all())
    dg[at] = 0
    assert not bool(dg[:T].any())                      # dropped choices
    want = d[at].double() * gates[at].double()
    assert bool(((dy[row].double() - want).abs() <= want.abs() * (half("bf16") + 2 * U)).all())
