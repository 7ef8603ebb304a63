"""Sizes at the ends of what the norm, the experts and their gradients take, against 64 bits: beyond the memory-side cache (256 MiB), where
loads and stores are streamed past it, beyond 2^31 bytes, and more tokens than a launch has workgroups for.  Bars as in
test_gpu_norm.py, test_gpu_expert8.py and test_gpu_expert_grad.py."""
import pytest

import test_gpu_expert8 as experts8
import test_gpu_expert_grad as grads
import test_gpu_norm as norms
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


BEYOND = 340_000_000                                    # bytes
ROWS = [80, 496, 1040, 2064, 8176, 16384]               # elements of bf16: one for each number of lanes that a row has; fp32 half of them


def rows_of(H, dtype, parts):
    """(tokens, hidden): parts rows of a token are BEYOND in all."""
    H = H // 2 // 16 * 16 if dtype == "f32" else H
    return int(BEYOND / (parts * H * (4 if dtype == "f32" else 2))), H


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [0, 1])
@pytest.mark.parametrize("H", ROWS)
def test_norm_beyond_the_cache(m, H, residual, dtype):  # noqa: F811
    T, H = rows_of(H, dtype, 4 if residual else 2)
    norms.test_norm(m, T, H, dtype, residual)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dsum", [0, 1])
@pytest.mark.parametrize("H", ROWS)
def test_norm_backward_beyond_the_cache(m, H, dsum, dtype):  # noqa: F811
    T, H = rows_of(H, dtype, 4 if dsum else 3)
    norms.test_norm_backward(m, T, H, dtype, dsum)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", ROWS)
def test_combine_backward_beyond_the_cache(m, H, dtype):  # noqa: F811
    """Three choices of eight experts, four tenths of them dropped."""
    T, H = rows_of(H, dtype, 1 + 2 * 1.8)
    norms.test_combine_backward(m, T, H, 8, 3, 0.6, 0, dtype)


@pytest.mark.parametrize("T,N,E,k", [(120, 2056, 16, 8), (24, 2056, 16, 4)])
@pytest.mark.parametrize("H", [4104, 4224])
def test_weights_beyond_the_cache(m, T, N, E, k, H):  # noqa: F811
    """dw of more than 256 MiB for many and for few rows, on rows that are whole 64-byte half lines and on others; off them as a whole:
    the same bits."""
    import torch
    grads.test_gradients(m, (T, H, N, E, k, 0.0, 0, 0.0), "bf16", 1)
    cfg, ws, tabs, rows = experts8.routed(m, T, H, "bf16", E, k)
    dy, x, w, _, dw = grads.run(m, cfg, ws, tabs, rows, N, "bf16", 0)
    n = E * N * H
    for by in (8, 32):                                 # 16 bytes, which leaves parts of half lines, and 64
        off = torch.full((n + 64,), 3.0, dtype=torch.bfloat16, device="cuda")
        m.monta_expert_linear_backward(cfg, dy, x, None, N, None, off[by:by + n].view(E, N, H), ws)
        torch.cuda.synchronize()
        assert torch.equal(off[by:by + n].view(E, N, H), dw) and bool((off[:by] == 3.0).all()) and bool((off[by + n:] == 3.0).all())


def spread(n, count=64):
    """Row numbers at both ends and evenly between."""
    import torch
    return torch.unique(torch.cat([torch.linspace(0, n - 1, count, dtype=torch.float64).long(), torch.arange(min(n, 8)), n - 1 - torch.arange(min(n, 8))])).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,N,E", [(140000, 8192, 256, 2), (140000, 256, 8192, 2), (600, 4096, 4224, 64)])
def test_gradients_beyond_2_31_bytes(m, T, H, N, E, dtype):  # noqa: F811
    """x and dx, dy, and w and dw of more than 2^31 bytes in turn.  Small integers: every sum is an fp32 number, whatever its order."""
    import torch
    needs(64)
    cfg, ws, tabs, rows = experts8.routed(m, T, H, dtype, E, 1)
    dy, x, w, dx, dw = grads.run(m, cfg, ws, tabs, rows, N, dtype, 1)
    act = grads.act(dtype)
    for e in range(E):
        a, n = int(tabs["offsets"][e]), int(tabs["kept"][e])
        at = a + spread(n)
        assert torch.equal(dx[at], (dy[at].double() @ w[e].double()).to(act)), e
        assert torch.equal(dw[e], (dy[a:a + n].float().T.contiguous() @ x[a:a + n].float()).to(act)), e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,N,E", [(300000, 8192, 256, 2), (300000, 256, 4096, 2), (600, 4096, 8448, 64)])
def test_experts8_beyond_2_31_bytes(m, T, H, N, E, dtype):  # noqa: F811
    """Rows, results and weights of more than 2^31 bytes in turn; exact as in test_gpu_expert8.py."""
    import torch
    needs(64)
    cfg, ws, tabs, rows = experts8.routed(m, T, H, dtype, E, 1)
    packed, wc, wsc, xc, xs = experts8.problem(m, cfg, rows, N, True)
    y = torch.full((rows + 1, N), 3.0, dtype=grads.act(dtype), device="cuda")
    m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y[:rows], ws)
    torch.cuda.synchronize()
    assert bool((y[rows] == 3.0).all())
    for e in range(E):
        at = int(tabs["offsets"][e]) + spread(int(tabs["kept"][e]))
        v = xc[at].double() * xs[at].double().repeat_interleave(128, 1)[:, :H]
        u = wc[e].double() * wsc[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :H]
        assert torch.equal(y[at], (v @ u.T).to(y.dtype)), e


def test_combine_backward_beyond_2_31_bytes(m):  # noqa: F811
    needs(48)
    norms.test_combine_backward(m, 90000, 8192, 4, 2, 0.0, 0, "bf16")
