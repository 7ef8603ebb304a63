"""GPU parity of the forms of the 8-bit expert layer and of the gradients that no case of test_gpu_expert8.py and test_gpu_expert_grad.py
takes, with segments of chosen lengths, so that tiles of every height end them.  Bars as there."""
import numpy as np
import pytest

import test_gpu_expert8 as experts8
import test_gpu_expert_grad as grads
from test_gpu_expert8 import m, routed  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# rows behind the last whole tile of 256: none, few, one short tile, and the first and last of every count of 16 or 32 rows that a loop is compiled for
ENDS = [0, 1, 3, 16, 17, 32, 33, 64, 65, 96, 128, 129, 150, 160, 161, 192, 193, 224, 225, 255]
IN_PLACE = ENDS + [256, 257, 321, 511]                  # rows of each expert
LAST = [512 + n for n in ENDS[1:]] + [0]

GRADS = [  # tokens, hidden, out_features, experts, top_k, capacity factor, padded, zipf
    (64, 2056, 1160, 16, 2, 0.0, 0, 0.0),              # few rows, many weights: a launch for each gradient
    (360, 392, 200, 64, 8, 0.0, 0, 0.8),               # dx in tiles of 64 x 128, dw in 128 x 128
]
GRADS_TO = [  # rows of the experts, hidden, out_features
    (IN_PLACE, 1544, 520),                             # large tiles of dx, ragged ones in place; those of at most 64 rows walk two halves
    (IN_PLACE, 1792, 1032),
    (LAST, 1544, 520),
    (LAST, 1032, 2056),                                # large tiles of both
]
EXPERTS8 = [  # tokens, hidden, out_features, experts, top_k, capacity factor, padded, slices, tp, zipf
    (256, 528, 1032, 64, 8, 0.0, 0, 2, 1, 0.6),        # bf16 in tiles of 64 x 128
    (300, 8320, 392, 40, 8, 0.0, 0, 1, 1, 1.0),        # the same, 65 blocks
]
EXPERTS8_TO = [  # rows of the experts, hidden, out_features
    (IN_PLACE, 256, 1288), (IN_PLACE, 272, 1288), (IN_PLACE, 8448, 1032), (LAST, 256, 1288), (LAST, 400, 1160),
]


def routed_to(m, loads, H, dtype, seed=7):  # noqa: F811
    """Every token to one expert, so many to each."""
    import torch
    from paper_2411_00662_amd import buffers
    rng = np.random.default_rng(seed)
    to = rng.permutation(np.repeat(np.arange(len(loads)), loads))
    logits = rng.normal(size=(len(to), len(loads))).astype(np.float32)
    logits[np.arange(len(to)), to] += 50
    cfg = m.make_cfg(len(to), H, m.FP32 if dtype == "f32" else m.BF16, len(loads), 1, 1, 1, 1)
    L = m.monta_ws_layout_query(cfg)
    ws = torch.zeros(L.ws_bytes, dtype=torch.uint8, device="cuda")
    idx, gates = torch.empty((len(to), 1), dtype=torch.int32, device="cuda"), torch.empty((len(to), 1), device="cuda")
    m.monta_ws_init(cfg, ws)
    m.monta_route(cfg, torch.from_numpy(logits).cuda(), idx, gates, ws)
    torch.cuda.synchronize()
    tabs = buffers.read_tables(cfg, ws)
    assert tabs["kept"].tolist() == list(loads)
    return cfg, ws, tabs, int(L.max_rows)


def check_gradients(m, cfg, ws, tabs, rows, N, dtype, exact):  # noqa: F811
    import torch
    dy, x, w, dx, dw = grads.run(m, cfg, ws, tabs, rows, N, dtype, exact)
    half = U if dtype == "f32" else 2.0 ** -8
    for e in range(cfg.experts):
        n = int(tabs["kept"][e])
        seg = slice(int(tabs["offsets"][e]), int(tabs["offsets"][e]) + n)
        a, b, c = dy[seg].double(), x[seg].double(), w[e].double()
        for name, got, want, mag, terms in (("dx", dx[seg], a @ c, a.abs() @ c.abs(), N), ("dw", dw[e], a.T @ b, a.abs().T @ b.abs(), n)):
            if exact:
                assert torch.equal(got.double(), want.to(grads.act(dtype)).double()), (name, e, n)
            else:
                assert bool(((got.double() - want).abs() <= terms * U * mag + half * want.abs()).all()), (name, e, n)
    return dx, dw


def ids(case):
    return "-".join("last" if v is LAST else "in_place" if v is IN_PLACE else str(v) for v in case)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", GRADS + GRADS_TO + grads.CASES[-4:-3], ids=ids)
def test_gradients(m, case, dtype):  # noqa: F811
    """Both gradients, and each alone: the same bits."""
    import torch
    if len(case) == 3:
        loads, H, N = case
        cfg, ws, tabs, rows = routed_to(m, loads, H, dtype)
    else:
        T, H, N, E, k, cf, padded, zipf = case
        cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k, cf, padded, zipf=zipf)
    check_gradients(m, cfg, ws, tabs, rows, N, dtype, 1)
    dx, dw = check_gradients(m, cfg, ws, tabs, rows, N, dtype, 0)
    assert torch.equal(grads.run(m, cfg, ws, tabs, rows, N, dtype, 0, "dx")[3], dx)
    assert torch.equal(grads.run(m, cfg, ws, tabs, rows, N, dtype, 0, "dw")[4], dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", EXPERTS8, ids=ids)
def test_experts8(m, case, dtype):  # noqa: F811
    T, H, N, E, k, cf, padded, S, tp, zipf = case
    cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k, cf, padded, S, tp, zipf)
    experts8.check(m, cfg, ws, tabs, rows, N, dtype, True)
    experts8.check(m, cfg, ws, tabs, rows, N, dtype, True, slices=range(S), seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", EXPERTS8_TO, ids=ids)
def test_experts8_by_length(m, case, dtype):  # noqa: F811
    loads, H, N = case
    cfg, ws, tabs, rows = routed_to(m, loads, H, dtype)
    experts8.check(m, cfg, ws, tabs, rows, N, dtype, True)
    if H < 1024:
        experts8.check(m, cfg, ws, tabs, rows, N, dtype, False)
