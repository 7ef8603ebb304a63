"""GPU parity of the expert layer on 8-bit rows and weights, against 64 bits.

Bars.  Codes that are small integers with scales that are powers of two make every product, every sum of a block and every partial
sum of the scaled blocks an fp32 number: results must agree bit for bit after the one rounding, which pins every index.  On
random codes:
  - fp32: exact products, additions in fp32: H u of the sum of the magnitudes (u = 2^-24) and 4 u for the scales and their product;
  - bf16: the 8-bit matrix instruction lines up the products of a few neighbours (at most 16 here) with the largest and cuts what lies
    more than 13 bits below it: 15 products lose less than 2^-13 of the largest each; then as above, and half a step of bf16.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def m():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_00662_amd as mod
    mod.binding.lib()
    return mod


def routed(m, T, H, dtype, E, k, cf=0.0, padded=0, slices=1, tp=1, zipf=0.0, seed=1):
    import torch
    from paper_2411_00662_amd import buffers
    cfg = m.make_cfg(T, H, m.FP32 if dtype == "f32" else m.BF16, E, k, 1, tp, slices, cf, 1, padded)
    logits = np.random.default_rng(seed).normal(size=(T, E)) - zipf * np.log(np.arange(1, E + 1))
    L = m.monta_ws_layout_query(cfg)
    ws = torch.zeros(L.ws_bytes, dtype=torch.uint8, device="cuda")
    idx, gates = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    m.monta_ws_init(cfg, ws)
    m.monta_route(cfg, torch.from_numpy(logits.astype(np.float32)).cuda(), idx, gates, ws)
    torch.cuda.synchronize()
    return cfg, ws, buffers.read_tables(cfg, ws), int(L.max_rows)


def problem(m, cfg, rows, N, exact, seed=2):
    """(8-bit rows, weight codes, weight scales, and both as 64-bit values and scales)"""
    import torch
    H, E = cfg.hidden, cfg.experts
    nb = -(-H // 128)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def codes(*shape):
        if exact:
            return torch.randint(-2, 3, shape, generator=g, device="cuda").float().to(torch.float8_e4m3fn)
        return (torch.randn(shape, generator=g, device="cuda") * 60).clamp(-448, 448).to(torch.float8_e4m3fn)

    def scales(*shape):
        if exact:
            return 2.0 ** torch.randint(-1, 2, shape, generator=g, device="cuda").float()
        return torch.rand(shape, generator=g, device="cuda") * 0.02 + 0.001

    xc, xs, wc, ws = codes(rows, H), scales(rows, nb), codes(E, N, H), scales(E, -(-N // 128), nb)
    packed = torch.full((rows, m.monta_fp8_rows(cfg)[1]), 0x7f, dtype=torch.uint8, device="cuda")       # NaN behind the scales
    packed[:, :H] = xc.view(torch.uint8)
    packed[:, H:H + 4 * nb] = xs.view(torch.uint8)
    return packed, wc, ws, xc, xs


def check(m, cfg, ws_buf, tabs, rows, N, dtype, exact, slices=(-1,), seed=2):
    import torch
    H, E = cfg.hidden, cfg.experts
    packed, wc, wsc, xc, xs = problem(m, cfg, rows, N, exact, seed)
    kept, first = tabs["kept"], tabs["offsets"]
    used = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for e in range(E):
        used[first[e]:first[e] + kept[e]] = True
    packed[~used] = 0x7f                               # rows of no expert hold NaN: they must not reach a result
    act = torch.float32 if dtype == "f32" else torch.bfloat16
    y = torch.full((rows + 1, N), 3.0, dtype=act, device="cuda")
    for j in slices:
        m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y[:rows], ws_buf, j)
    torch.cuda.synchronize()
    assert bool((y[rows] == 3.0).all()) and bool((y[:rows][~used] == 3.0).all())
    xv = xc.double() * xs.double().repeat_interleave(128, 1)[:, :H]
    for e in range(E):
        seg = slice(int(first[e]), int(first[e] + kept[e]))
        if kept[e] == 0:
            continue
        w = wc[e].double() * wsc[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :H]
        want, got = xv[seg] @ w.T, y[seg].double()
        if exact:
            assert torch.equal(got, want.to(act).double()), f"expert {e}"
            continue
        mag = xv[seg].abs() @ w.abs().T
        if dtype == "f32":
            tol = (H + 4) * U * mag
        else:
            cut = torch.zeros_like(want)
            for h in range(0, H, 16):
                cut += (xv[seg, None, h:h + 16] * w[None, :, h:h + 16]).abs().amax(2)
            tol = 15 * 2.0 ** -13 * cut + (H + 4) * U * mag + want.abs() * 2.0 ** -8
        assert bool(((got - want).abs() <= tol).all()), f"expert {e}: {((got - want).abs() / tol).max().item()}"


CASES = [  # tokens, hidden, out_features, experts, top_k, capacity factor, padded, slices, tp, zipf
    (1, 16, 8, 1, 1, 0.0, 0, 1, 1, 0.0),
    (1, 4096, 256, 8, 2, 0.0, 0, 1, 1, 0.0),
    (7, 128, 136, 4, 2, 0.0, 0, 1, 1, 0.0),
    (16, 144, 72, 8, 2, 0.5, 0, 1, 1, 0.0),
    (40, 1040, 264, 4, 4, 0.0, 0, 1, 1, 0.0),
    (64, 8320, 64, 2, 1, 0.0, 0, 1, 1, 0.0),           # 65 blocks: the weights' scales are fetched twice
    (96, 528, 520, 16, 3, 0.7, 1, 1, 1, 0.8),
    (300, 256, 128, 3, 2, 0.0, 0, 1, 1, 0.0),
    (512, 400, 1000, 2, 1, 0.0, 0, 1, 1, 0.0),
    (1200, 384, 1160, 5, 2, 1.25, 0, 3, 2, 1.2),
    (2048, 272, 2056, 4, 2, 0.9, 1, 4, 1, 0.0),
    (900, 128, 8, 64, 8, 0.0, 0, 1, 1, 1.2),
    (3300, 256, 2304, 6, 2, 0.0, 0, 1, 1, 0.0),        # large tiles, ragged ones of every length last
    (3300, 400, 2056, 6, 2, 0.0, 0, 2, 1, 0.6),
    (1100, 8320, 1032, 8, 4, 0.0, 1, 1, 1, 0.3),
    (4000, 144, 1288, 60, 8, 0.8, 0, 1, 1, 0.9),       # large tiles and lower ones, fewer steps than stages
    (1500, 8336, 1032, 40, 4, 0.0, 0, 1, 1, 1.2),      # the same, 66 blocks
    (5, 12288, 136, 3, 2, 0.0, 0, 1, 1, 0.0),          # walks that begin at different blocks and go round: 96 of them,
    (40, 8192, 520, 8, 2, 0.0, 0, 2, 1, 0.0),          # 64
    (3, 65536, 72, 2, 1, 0.0, 0, 1, 1, 0.0),           # and 512, the longest rows
    (2, 8208, 24, 8, 2, 0.0, 0, 1, 1, 0.0),            # few tiles, whose waves share the blocks: 65 of them
    (90, 4112, 40, 3, 2, 0.0, 1, 2, 1, 0.7),           # the same, several row tiles
    (12, 4096, 4096, 8, 2, 0.0, 0, 1, 1, 0.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_exact(m, case, dtype):
    T, H, N, E, k, cf, padded, S, tp, zipf = case
    cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k, cf, padded, S, tp, zipf)
    check(m, cfg, ws, tabs, rows, N, dtype, True)
    if S > 1:
        check(m, cfg, ws, tabs, rows, N, dtype, True, slices=range(S), seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(3, 4096, 64, 4, 2), (48, 1040, 136, 4, 2), (200, 528, 264, 2, 1), (700, 256, 1032, 2, 1)], ids=str)
def test_random(m, case, dtype):
    T, H, N, E, k = case
    cfg, ws, tabs, rows = routed(m, T, H, dtype, E, k)
    check(m, cfg, ws, tabs, rows, N, dtype, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(3300, 400, 2056, 6, 2, 2, 0.6), (40, 8192, 520, 8, 2, 2, 0.0), (90, 4112, 40, 3, 2, 2, 0.7), (2048, 272, 2056, 4, 2, 4, 0.0),
                                  (4096, 256, 520, 16, 2, 4, 1.2)], ids=str)
def test_slices_are_the_whole(m, case, dtype):
    """Slice after slice or all at once, on codes whose sums are rounded: the same bits; and again: the same bits."""
    import torch
    T, H, N, E, k, S, zipf = case
    cfg, ws, _, rows = routed(m, T, H, dtype, E, k, slices=S, zipf=zipf)
    packed, wc, wsc, _, _ = problem(m, cfg, rows, N, False)
    y = [torch.zeros((rows, N), dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda") for _ in range(3)]
    m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y[0], ws)
    for j in range(S):
        m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y[1], ws, j)
    m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y[2], ws)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2])


def test_special_codes(m):
    """A NaN code or an infinite scale stays in its row; largest and smallest codes multiply as the numbers they are."""
    import torch
    cfg, ws, tabs, rows = routed(m, 64, 256, "bf16", 2, 1)
    packed, wc, wsc, xc, xs = problem(m, cfg, rows, 128, True)
    base = torch.zeros((rows, 128), dtype=torch.bfloat16, device="cuda")
    m.monta_expert_linear_fp8(cfg, packed, wc, wsc, 128, base, ws)
    packed[3, 70] = 0x7f
    packed[9, 256:260] = torch.tensor([0, 0, 0x80, 0x7f], dtype=torch.uint8, device="cuda")     # +inf
    y = torch.zeros_like(base)
    m.monta_expert_linear_fp8(cfg, packed, wc, wsc, 128, y, ws)
    same = torch.ones(rows, dtype=torch.bool, device="cuda")
    same[[3, 9]] = False
    assert torch.equal(y[same], base[same]) and bool(torch.isnan(y[3]).all()) and not bool(torch.isfinite(y[9]).any())
    one = torch.zeros_like(packed)
    one[:, 256:264] = torch.ones((rows, 2), device="cuda").view(torch.uint8)
    values = torch.arange(127, dtype=torch.uint8, device="cuda")                     # every positive finite code, one in each row
    n = min(rows, 127)
    one[:n, 5] = values[:n].flip(0) if n < 127 else values
    wone = torch.zeros((2, 128, 256), dtype=torch.uint8, device="cuda")
    wone[:, :, 5] = 0x38                                                             # 1.0
    m.monta_expert_linear_fp8(cfg, one, wone, torch.ones_like(wsc), 128, y, ws)
    want = one[:n, 5].contiguous().view(torch.float8_e4m3fn).float().to(torch.bfloat16)
    assert torch.equal(y[:n], want[:, None].expand(n, 128))


def test_graph(m):
    """Captured, replayed with eager work between, two problems whose replays follow one another."""
    import torch
    made = []
    for T, H, N, E in ((64, 512, 256, 4), (600, 640, 520, 3)):
        cfg, ws, tabs, rows = routed(m, T, H, "bf16", E, 2)
        packed, wc, wsc, _, _ = problem(m, cfg, rows, N, False)
        y = torch.zeros((rows, N), dtype=torch.bfloat16, device="cuda")
        m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.monta_expert_linear_fp8(cfg, packed, wc, wsc, N, y, ws)
        made.append((graph, y, y.clone(), (packed, wc, wsc, ws)))        # a replay reads the buffers again: they stay
    for _ in range(3):
        for graph, y, _, _ in made:
            y.zero_()
        torch.cuda.synchronize()
        for graph, _, _, _ in made:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for _, y, want, _ in made)
