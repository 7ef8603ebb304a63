"""GPU parity of the 8-bit expert layer on values out of the ordinary: every code, and scales that are infinite.  Codes of small integers
and scales that are powers of two make all sums fp32 numbers: what is finite agrees bit for bit after the one rounding."""
import pytest

from test_gpu_expert8 import m, problem, routed  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [  # tokens, hidden, out_features, experts, top_k: one for each way of walking along the hidden axis
    (2, 8208, 24, 8, 2),                               # few tiles, 16 features, 65 blocks
    (90, 4112, 40, 3, 2),                              # few tiles, 32 features, 33 blocks
    (96, 528, 520, 16, 3),                             # 32 x 64
    (512, 400, 1000, 2, 1),                            # 32 x 128, fp32 64 x 128
    (1200, 384, 1160, 5, 2),                           # 128 x 128
    (3300, 400, 2056, 6, 2),                           # 256 x 256 and lower ones
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [0, -1])
@pytest.mark.parametrize("case", SHAPES, ids=str)
def test_infinite_scales(m, case, block, dtype):  # noqa: F811
    """The first or the last block of a tile's weights has an infinite scale: an infinity of the block's sign, NaN where the block's sum is zero, as in
    64 bits, and every other feature as it is without."""
    import torch
    T, H, N, E, k = case
    cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k)
    packed, wc, wsc, xc, xs = problem(m, cfg, rows, N, True)
    wsc[:, -1, block] = float("inf")                   # the last block of 128 features
    first = (N - 1) // 128 * 128
    y = torch.full((rows, N), 3.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y, ws)
    torch.cuda.synchronize()
    nb = wsc.shape[2]
    for e in range(E):
        seg = slice(int(tabs["offsets"][e]), int(tabs["offsets"][e] + tabs["kept"][e]))
        want = torch.zeros((seg.stop - seg.start, N), dtype=torch.float64, device="cuda")
        for b in range(nb):
            cut = slice(b * 128, min(H, b * 128 + 128))
            part = xc[seg, cut].double() @ wc[e][:, cut].double().T
            want += part * (xs[seg, b:b + 1].double() * wsc[e, :, b].double().repeat_interleave(128)[:N])
        want, got = want.to(y.dtype), y[seg]
        assert torch.equal(got[:, :first], want[:, :first]), e
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num()), e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SHAPES, ids=str)
def test_every_code(m, case, dtype):  # noqa: F811
    """Row r has one code, number r % 256, at one place and zeros elsewhere; the weights have 1 there: the results are the codes' values."""
    import torch
    T, H, N, E, k = case
    cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k)
    at, nb = H - 3, -(-H // 128)
    packed = torch.zeros((rows, m.monta_fp8_rows(cfg)[1]), dtype=torch.uint8, device="cuda")
    codes = (torch.arange(rows, device="cuda") * 37 % 256).to(torch.uint8)
    packed[:, at] = codes
    packed[:, H:H + 4 * nb] = torch.ones((rows, nb), device="cuda").view(torch.uint8)
    wc = torch.zeros((E, N, H), dtype=torch.uint8, device="cuda")
    wc[:, :, at] = 0x38                                # 1.0
    y = torch.full((rows, N), 3.0, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    m.monta_expert_linear_fp8(cfg, packed, wc, torch.ones((E, -(-N // 128), nb), device="cuda"), N, y, ws)
    torch.cuda.synchronize()
    used = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for e in range(E):
        used[int(tabs["offsets"][e]):int(tabs["offsets"][e] + tabs["kept"][e])] = True
    want = torch.where(used, codes.view(torch.float8_e4m3fn).float(), torch.full((), 3.0, device="cuda")).to(y.dtype)[:, None].expand(rows, N)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(y.nan_to_num(), want.nan_to_num())
