"""The operators around the expert layer whose speed counts, each in its plain form and as the framework's call.

A case is one pass through one of them:

  norm          root-mean-square norm of a token's row, the residual's addition before it, and with `fp8` the
                normalised row a second time in 8 bits (e4m3) with a scale for each block of 128 elements
  norm_grad     its gradient: by the input and by the weight
  experts8      the expert layer on such 8-bit rows and on 8-bit weights with a scale for each 128 x 128 block: one
                matrix product per expert, of as many rows as were routed to it
  experts_grad  the gradient of the expert layer by its rows and by its weights
  combine_grad  the gradient of the combine: rows of the experts' output and gates

`run` computes them in elementary torch operations in 32 bits, or, where `own` is true, by the library's calls.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 128                      # elements that share a scale
E4M3_MAX = 448.0
AMAX_FLOOR = 2.0 ** -40          # a block whose values are all below it is scaled as if its largest were this


def _case(kind, T, H, dtype, name=None, E=1, k=1, N=0, cf=0.0, zipf=0.0, padded=0, residual=0, fp8=0):
    c = {"kind": kind, "tokens": T, "hidden": H, "dtype": dtype, "experts": E, "top_k": k, "out_features": N,
         "capacity_factor": float(cf), "zipf": float(zipf), "padded": padded, "residual": residual, "fp8": fp8}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of a serving loop, on its way to the gate (16 bits) and to the experts (8 bits): launch latency
        _case("norm", 1, 4096, "bf16", "norm_token", residual=1, fp8=1),
        # the 8K batch of the sparse layer of 8 experts
        _case("norm", 8192, 4096, "bf16", "norm_batch", residual=1, fp8=1),
        # 32 bits, a width that ends inside a block of 128, no residual
        _case("norm", 1155, 528, "f32", "norm_f32_odd", fp8=1),
        # training on the same batch, with the gradient that arrives along the residual
        _case("norm_grad", 8192, 4096, "bf16", "norm_grad_batch", residual=1),
        _case("norm_grad", 1155, 516, "f32", "norm_grad_f32_odd"),
        # one decoding step of 64 sequences: every expert's weights for a few rows each
        _case("experts8", 64, 4096, "bf16", "experts8_decode", E=8, k=2, N=4096),
        # long segments: prefill of the sparse layer of 8 experts
        _case("experts8", 8192, 4096, "bf16", "experts8_batch", E=8, k=2, N=4096, cf=2.0),
        # fine-grained experts with a skewed load and drops: segments of every length
        _case("experts8", 4096, 7168, "bf16", "experts8_skewed", E=64, k=8, N=2048, cf=1.25, zipf=1.2),
        # training: both gradients of the expert layer on the 8K batch
        _case("experts_grad", 8192, 4096, "bf16", "experts_grad_batch", E=8, k=2, N=4096, cf=2.0),
        # 32 bits, odd sizes, drops, the capacity-padded layout
        _case("experts_grad", 1155, 516, "f32", "experts_grad_f32_odd", E=10, k=3, N=516, cf=0.7, padded=1),
        # the way back through the combine, on the same batch and with eight choices of which many were dropped
        _case("combine_grad", 8192, 4096, "bf16", "combine_grad_batch", E=8, k=2, cf=2.0),
        _case("combine_grad", 8192, 7168, "bf16", "combine_grad_skewed", E=64, k=8, cf=1.25, zipf=1.2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm_grad", "experts8", "experts8", "experts_grad", "combine_grad"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        bpe = 4 if dtype == "f32" else 2
        fp8 = int(kind == "experts8" or (kind == "norm" and rng.random() < 0.7))
        unit = 16 if fp8 else 16 // bpe
        H = unit * max(1, _log(rng, 64, 8192) // unit) if rng.random() < 0.5 else rng.choice([512, 1024, 2048, 4096, 5120, 7168, 8192])
        if kind in ("norm", "norm_grad"):
            T = _log(rng, 1, 65536)
            if T * H * bpe > 8192 * 4096 * 2:
                continue
            return _case(kind, T, H, dtype, residual=rng.randint(0, 1), fp8=fp8)
        E = rng.choice([2, 4, 8, 8, 16, 32, 64, rng.randint(2, 64)])
        k = min(E, rng.choice([1, 2, 2, 4, 6, 8]))
        T = _log(rng, 1, 8192)
        cf, zipf = rng.choice([(0.0, 0.0), (2.0, 0.0), (1.25, 0.0), (1.25, 1.2), (0.7, 0.8)])
        unit = 16 // bpe
        N = 0 if kind == "combine_grad" else unit * max(1, _log(rng, 64, 8192) // unit)
        c = _case(kind, T, H, dtype, E=E, k=k, N=N, cf=cf, zipf=zipf, padded=int(cf > 0 and rng.random() < 0.2))
        rows = _max_rows(c)
        if kind == "combine_grad":
            if rows * H * bpe > 45000 * 7168 * 2:
                continue
        elif rows * H * N > (16384 * 4096 * 4096 if dtype == "bf16" else 16384 * 1024 * 1024) or E * H * N * bpe > 2 << 30:
            continue
        # the plain form pads every expert to the largest one's rows
        if zipf == 0.0 and cf == 0.0 and kind != "combine_grad" and E * T * H * 4 > 4 << 30:
            continue
        return c


def _capacity(c):
    T, E, k, cf = c["tokens"], c["experts"], c["top_k"], c["capacity_factor"]
    cf = torch.tensor(cf, dtype=torch.float32).item()
    return T if cf <= 0 else min(T, math.ceil(cf * T * k / E))


def _max_rows(c):
    ec = c["experts"] * _capacity(c)
    return ec if c["padded"] else min(c["tokens"] * c["top_k"], ec)


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _fp8_row_bytes(H):
    """Codes, then a 32-bit scale for each block, in whole 128-byte lines."""
    return (H + 4 * _blocks(H) + 127) // 128 * 128


# ------------------------------------------------------------------------------------------------ inputs


def _quantise(v, rows_per_scale):
    """float32 [R, H] -> (codes [R, H], scales [R / rows_per_scale, blocks]), a scale for each rows_per_scale x 128 block."""
    R, H = v.shape
    nr, nb = -(-R // rows_per_scale), _blocks(H)
    full = torch.zeros((nr * rows_per_scale, nb * BLOCK), dtype=v.dtype, device=v.device)
    full[:R, :H] = v
    tiles = full.view(nr, rows_per_scale, nb, BLOCK)
    amax = tiles.abs().amax(dim=(1, 3)).clamp_min(AMAX_FLOOR)
    codes = (tiles * (E4M3_MAX / amax)[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
    return codes.view(nr * rows_per_scale, nb * BLOCK)[:R, :H].to(torch.float8_e4m3fn), amax / E4M3_MAX


def _cfg(m, c):
    return m.make_cfg(c["tokens"], c["hidden"], m.FP32 if c["dtype"] == "f32" else m.BF16, c["experts"], c["top_k"], 1, 1, 1,
                      c["capacity_factor"], 1, c["padded"])


class _State:
    pass


def _plan(c, logits):
    """The routing of a layer, in torch: gates [T, k], row of each pair (-1: dropped), first row and rows of each expert."""
    T, E, k, C = c["tokens"], c["experts"], c["top_k"], _capacity(c)
    top, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    gates, idx = torch.softmax(top[:, :k], dim=1), idx[:, :k]
    flat = idx.reshape(-1)
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    rank = torch.empty_like(flat)
    rank[order] = torch.arange(T * k, device=flat.device) - (torch.cumsum(counts, 0) - counts)[flat[order]]
    kept = counts.clamp_max(C)
    first = torch.arange(E, device=flat.device) * C if c["padded"] else torch.cumsum(kept, 0) - kept
    pos = torch.where(rank < C, first[flat] + rank, torch.full_like(rank, -1)).view(T, k)
    return gates.contiguous(), pos, first, kept


def prepare(case, seed):
    c, s = case, _State()
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, H, E, k, N, dt = c["tokens"], c["hidden"], c["experts"], c["top_k"], c["out_features"], _dtype(c)

    def normal(*shape, scale=1.0, dtype=None):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype or dt).mul_(scale)

    s.c, s.kind, s.H, s.N, s.dt = c, c["kind"], H, N, dt
    if own:                      # what a program that uses the library keeps: its module, the configuration, buffers
        import paper_2411_00662_amd as m
        s.m, s.cfg = m, _cfg(m, c)
    if s.kind in ("norm", "norm_grad"):
        s.w = (1.0 + normal(H, scale=0.2, dtype=torch.float32)).to(dt)
        s.x = normal(T, H, scale=1.5)
        s.residual = normal(T, H) if c["residual"] else None
        if s.kind == "norm":
            s.sum = torch.empty_like(s.x) if c["residual"] else None
            s.out = torch.empty_like(s.x)
            s.rows8 = torch.empty((T, _fp8_row_bytes(H)), dtype=torch.uint8, device="cuda") if c["fp8"] else None
            return s
        s.dout = normal(T, H, scale=0.1)
        s.dx, s.dw = torch.empty_like(s.x), torch.empty(H, dtype=torch.float32, device="cuda")
        if own:
            s.scratch = torch.empty(m.monta_rmsnorm_scratch_bytes(s.cfg), dtype=torch.uint8, device="cuda")
        return s

    logits = _logits(c, g, "cuda")
    s.rows = _max_rows(c)
    s.gates, s.pos, s.first, s.kept = _plan(c, logits)
    s.most = int(s.kept.max().item())
    if own:                      # the routing as the library keeps it
        L = m.monta_ws_layout_query(s.cfg)
        s.ws = torch.empty(L.ws_bytes, dtype=torch.uint8, device="cuda")
        topk = torch.empty((T, k), dtype=torch.int32, device="cuda")
        routed = torch.empty((T, k), dtype=torch.float32, device="cuda")
        m.monta_ws_init(s.cfg, s.ws)
        m.monta_route(s.cfg, logits, topk, routed, s.ws)
    if s.kind == "experts8":
        codes, scales = _quantise(normal(s.rows, H, dtype=torch.float32), 1)
        s.x8 = torch.zeros((s.rows, _fp8_row_bytes(H)), dtype=torch.uint8, device="cuda")
        s.x8[:, :H] = codes.view(torch.uint8)
        s.x8[:, H:H + 4 * _blocks(H)] = scales.contiguous().view(torch.uint8)
        s.w8 = torch.empty((E, N, H), dtype=torch.float8_e4m3fn, device="cuda")
        s.w_scales = torch.empty((E, _blocks(N), _blocks(H)), dtype=torch.float32, device="cuda")
        for e in range(E):
            s.w8[e], s.w_scales[e] = _quantise(normal(N, H, scale=H ** -0.5, dtype=torch.float32), BLOCK)
        s.y = torch.zeros((s.rows, N), dtype=dt, device="cuda")
    elif s.kind == "experts_grad":
        s.x, s.w, s.dy = normal(s.rows, H), normal(E, N, H, scale=H ** -0.5), normal(s.rows, N, scale=0.1)
        s.dx, s.dw = torch.zeros((s.rows, H), dtype=dt, device="cuda"), torch.empty((E, N, H), dtype=dt, device="cuda")
    else:
        s.y, s.dout = normal(s.rows, H), normal(T, H, scale=0.1)
        s.dy, s.dgates = torch.zeros((s.rows, H), dtype=dt, device="cuda"), torch.empty((T, k), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(s):
    return (_run_own if own else _run_plain)[s.kind](s)


def _own_norm(s):
    s.m.monta_rmsnorm(s.cfg, s.x, s.residual, s.w, EPS, s.sum, s.out, s.rows8)
    got = {"out": s.out}
    if s.residual is not None:
        got["sum"] = s.sum
    if s.rows8 is not None:
        got["codes"] = s.rows8[:, :s.H].view(torch.float8_e4m3fn)
        got["scales"] = s.rows8[:, s.H:s.H + 4 * _blocks(s.H)].view(torch.float32)
    return got


def _own_norm_grad(s):
    s.m.monta_rmsnorm_backward(s.cfg, s.x, s.w, EPS, s.dout, s.residual, s.dx, s.dw, s.scratch)
    return {"dx": s.dx, "dw": s.dw}


def _own_experts8(s):
    s.m.monta_expert_linear_fp8(s.cfg, s.x8, s.w8, s.w_scales, s.N, s.y, s.ws)
    return {"y": s.y}


def _own_experts_grad(s):
    s.m.monta_expert_linear_backward(s.cfg, s.dy, s.x, s.w, s.N, s.dx, s.dw, s.ws)
    return {"dx": s.dx, "dw": s.dw}


def _own_combine_grad(s):
    s.m.monta_combine_backward(s.cfg, s.dout, s.y, s.gates, s.dy, s.dgates, s.ws)
    return {"dy": s.dy, "dgates": s.dgates}


_run_own = {"norm": _own_norm, "norm_grad": _own_norm_grad, "experts8": _own_experts8, "experts_grad": _own_experts_grad,
            "combine_grad": _own_combine_grad}


def _plain_norm(s):
    got, t = {}, s.x
    if s.residual is not None:
        t = (s.x.float() + s.residual.float()).to(s.dt)
        got["sum"] = t
    t = t.float()
    v = t * torch.rsqrt((t * t).mean(dim=1, keepdim=True) + EPS) * s.w.float()
    got["out"] = v.to(s.dt)
    if s.c["fp8"]:
        got["codes"], got["scales"] = _quantise(v, 1)
    return got


def _plain_norm_grad(s):
    t, d = s.x.float(), s.dout.float()
    r = torch.rsqrt((t * t).mean(dim=1, keepdim=True) + EPS)
    n = t * r
    g = d * s.w.float()
    dx = r * (g - n * (g * n).mean(dim=1, keepdim=True))
    if s.residual is not None:
        dx = dx + s.residual.float()
    return {"dx": dx.to(s.dt), "dw": (d * n).sum(dim=0)}


def _segments(s):
    """Rows of each expert's segment, [E, most], those past its end at the row behind all others; and the same as truth values."""
    at = torch.arange(s.most, device="cuda")
    live = at < s.kept[:, None]
    return torch.where(live, s.first[:, None] + at, torch.full_like(at, s.rows)), live


def _gather(t, at, live):
    """Rows of t by segment, in 32 bits, zeros past the segments' ends."""
    return t[at.clamp_max(t.shape[0] - 1)].float() * live[..., None]


def _scatter(t, at, rows):
    out = torch.zeros((rows + 1, t.shape[-1]), dtype=t.dtype, device=t.device)
    out[at.reshape(-1)] = t.reshape(-1, t.shape[-1])
    return out[:rows]


def _dequantise(codes, scales, rows_per_scale):
    """The values that codes [..., R, H] stand for, in 32 bits."""
    R, H = codes.shape[-2:]
    s = scales.repeat_interleave(rows_per_scale, dim=-2)[..., :R, :] if rows_per_scale > 1 else scales
    return codes.float() * s.repeat_interleave(BLOCK, dim=-1)[..., :H]


def _rows8(s):
    H = s.H
    return s.x8[:, :H].view(torch.float8_e4m3fn), s.x8[:, H:H + 4 * _blocks(H)].view(torch.float32)


def _plain_experts8(s):
    at, live = _segments(s)
    x = _gather(_dequantise(*_rows8(s), 1), at, live)
    y = torch.bmm(x, _dequantise(s.w8, s.w_scales, BLOCK).transpose(1, 2))
    return {"y": _scatter(y.to(s.dt), at, s.rows)}


def _plain_experts_grad(s):
    at, live = _segments(s)
    dy, x = _gather(s.dy, at, live), _gather(s.x, at, live)
    dx = torch.bmm(dy, s.w.float())
    return {"dx": _scatter(dx.to(s.dt), at, s.rows), "dw": torch.bmm(dy.transpose(1, 2), x).to(s.dt)}


def _plain_combine_grad(s):
    live, d = s.pos >= 0, s.dout.float()
    y = s.y[s.pos.clamp_min(0)].float()
    dgates = (y * d[:, None]).sum(dim=-1) * live
    dy = (d[:, None] * s.gates[..., None]).to(s.dt)
    at = torch.where(live, s.pos, torch.full_like(s.pos, s.rows))
    return {"dy": _scatter(dy, at, s.rows), "dgates": dgates}


_run_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "experts8": _plain_experts8, "experts_grad": _plain_experts_grad,
              "combine_grad": _plain_combine_grad}


# ------------------------------------------------------------------------------------------------ what a pass needs


def _logits(c, g, device):
    logits = torch.randn((c["tokens"], c["experts"]), generator=g, device=device)
    if c["zipf"] > 0:
        logits -= c["zipf"] * torch.log(torch.arange(1, c["experts"] + 1, device=device, dtype=torch.float32))
    return logits


def _typical_load(c):
    """(rows that are kept, experts that have any) for one set of logits of the case's distribution: other sets differ little."""
    idx = torch.topk(_logits(c, torch.Generator().manual_seed(0), "cpu"), c["top_k"], dim=1).indices
    kept = torch.bincount(idx.reshape(-1), minlength=c["experts"]).clamp_max(_capacity(c))
    return int(kept.sum()), int((kept > 0).sum())


def work(case):
    """Bytes that a pass has to read and write once each, and operations."""
    c = case
    T, H, E, k, N = c["tokens"], c["hidden"], c["experts"], c["top_k"], c["out_features"]
    bpe = 4 if c["dtype"] == "f32" else 2
    row = H * bpe
    if c["kind"] == "norm":
        moved = T * row * (4 if c["residual"] else 2) + row + (T * (H + 4 * _blocks(H)) if c["fp8"] else 0)
        return {"bytes": moved, "flops": 6 * T * H}
    if c["kind"] == "norm_grad":
        return {"bytes": T * row * (4 if c["residual"] else 3) + row + 4 * H, "flops": 10 * T * H}
    kept, used = _typical_load(c)
    if c["kind"] == "combine_grad":
        return {"bytes": T * row + 2 * kept * row + T * k * 12, "flops": 3 * kept * H}
    if c["kind"] == "experts8":
        return {"bytes": kept * (H + 4 * _blocks(H)) + used * (N * H + 4 * _blocks(N) * _blocks(H)) + kept * N * bpe,
                "flops": 2 * kept * N * H}
    return {"bytes": kept * (2 * H + N) * bpe + (used + E) * N * H * bpe, "flops": 4 * kept * N * H}


# ------------------------------------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    """The same outputs from the definitions, row by row and expert by expert, in 64 bits."""
    s, f = prepare(case, seed), torch.float64
    c, H = case, s.H
    if s.kind == "norm":
        got = {}
        t = s.x.to(f)
        if s.residual is not None:
            got["sum"] = t + s.residual.to(f)
            t = got["sum"].to(torch.float32).to(s.dt).to(f)         # the norm is that of the sum as it is stored
        got["out"] = t / ((t ** 2).sum(1, keepdim=True) / H + EPS).sqrt() * s.w.to(f)
        if c["fp8"]:
            nb = _blocks(H)
            codes, scales = torch.empty_like(t), torch.empty((c["tokens"], nb), dtype=f, device="cuda")
            for b in range(nb):
                v = got["out"][:, b * BLOCK:(b + 1) * BLOCK]
                scales[:, b] = torch.maximum(v.abs().max(1).values, torch.tensor(AMAX_FLOOR, dtype=f, device="cuda")) / E4M3_MAX
                codes[:, b * BLOCK:(b + 1) * BLOCK] = (v / scales[:, b:b + 1]).to(torch.float32).to(torch.float8_e4m3fn).to(f)
            got["codes"], got["scales"] = codes, scales
        return got
    if s.kind == "norm_grad":
        t, d, w = s.x.to(f), s.dout.to(f), s.w.to(f)
        ms = (t ** 2).sum(1, keepdim=True) / H + EPS
        dot = (d * w * t).sum(1, keepdim=True)
        dx = d * w / ms.sqrt() - t * dot / (H * ms ** 1.5)
        return {"dx": dx if s.residual is None else dx + s.residual.to(f), "dw": (d * t / ms.sqrt()).sum(0)}
    if s.kind == "combine_grad":
        d, y = s.dout.to(f), s.y.to(f)
        dy, dgates = torch.zeros_like(y), torch.zeros(s.pos.shape, dtype=f, device="cuda")
        for j in range(c["top_k"]):
            t = (s.pos[:, j] >= 0).nonzero()[:, 0]
            at = s.pos[t, j]
            dy[at] = d[t] * s.gates[t, j].to(f)[:, None]
            dgates[t, j] = (d[t] * y[at]).sum(1)
        return {"dy": dy, "dgates": dgates}
    first, kept = s.first.tolist(), s.kept.tolist()
    if s.kind == "experts8":
        y = torch.zeros((s.rows, s.N), dtype=f, device="cuda")
        for e in range(c["experts"]):
            seg = slice(first[e], first[e] + kept[e])
            x8, xs = s.x8[seg, :H].contiguous().view(torch.float8_e4m3fn).to(f), s.x8[seg, H:H + 4 * _blocks(H)].contiguous().view(torch.float32).to(f)
            w = s.w8[e].to(f)
            for b in range(_blocks(H)):
                cut = slice(b * BLOCK, min(H, (b + 1) * BLOCK))
                x8[:, cut] *= xs[:, b:b + 1]
                for n in range(_blocks(s.N)):
                    w[n * BLOCK:(n + 1) * BLOCK, cut] *= s.w_scales[e, n, b].to(f)
            y[seg] = x8 @ w.T
        return {"y": y}
    dx, dw = torch.zeros((s.rows, H), dtype=f, device="cuda"), torch.zeros((c["experts"], s.N, H), dtype=f, device="cuda")
    for e in range(c["experts"]):
        seg = slice(first[e], first[e] + kept[e])
        dy = s.dy[seg].to(f)
        dx[seg] = dy @ s.w[e].to(f)
        dw[e] = dy.T @ s.x[seg].to(f)
    return {"dx": dx, "dw": dw}
