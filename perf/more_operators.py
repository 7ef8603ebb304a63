"""What training needs between the layer's loss and the token rows ahead of the gate, each operator in its plain form and as the framework's call.

A case is one pass through one of them:

  layernorm       layer norm of a token's row, the residual's addition before it, and with `fp8` the normalised row a second time in
                  8 bits (e4m3) with a scale for each block of 128 elements
  layernorm_grad  its gradient: by the input, the weight and the bias
  route_loss      the router's balance loss and the mean square of its log partition (z loss), with the pairs that chose each expert,
                  over the tokens that are no padding
  route_grad      from the gradients of the gates and of the two losses to that of the router's logits
  gate_grad       the gradient of the gate projection: by the tokens' rows, added to what reaches them by another way, and by its weights

`run` computes them in elementary torch operations in 32 bits, or, where `own` is true, by the library's calls.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 128                      # elements that share a scale
E4M3_MAX = 448.0
AMAX_FLOOR = 2.0 ** -40          # a block whose values are all below it is scaled as if its largest were this
LOSS_WEIGHTS = (1e-2, 1e-3)      # of the balance loss and of the z loss in the whole one


def _case(kind, T, H=64, dtype="f32", name=None, E=1, k=1, zipf=0.0, renorm=1, cf=0.0, padding=0, losses=1, other=0, fp8=0):
    c = {"kind": kind, "tokens": T, "hidden": H, "dtype": dtype, "experts": E, "top_k": k, "zipf": float(zipf), "renorm": renorm,
         "capacity_factor": float(cf), "padding": padding, "losses": losses, "other": other, "fp8": fp8}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of a serving loop through the norm ahead of the gate (16 bits) and the experts (8 bits): launch latency
        _case("layernorm", 1, 4096, "bf16", "layernorm_token", other=1, fp8=1),
        # the 8K batch of the sparse layer of 8 experts
        _case("layernorm", 8192, 4096, "bf16", "layernorm_batch", other=1, fp8=1),
        # 32 bits, a width that ends inside a block of 128, no residual
        _case("layernorm", 1155, 528, "f32", "layernorm_f32_odd", fp8=1),
        # training on the same batch, with the gradient that arrives along the residual
        _case("layernorm_grad", 8192, 4096, "bf16", "layernorm_grad_batch", other=1),
        _case("layernorm_grad", 1155, 516, "f32", "layernorm_grad_f32_odd"),
        # the smallest named workload's router: launches and host work are all there is
        _case("route_loss", 256, name="route_loss_tiny", E=4, k=2),
        # fine-grained experts with a skewed load, the ends of the sequences padding: the largest named workload's router
        _case("route_loss", 65536, name="route_loss_skewed", E=64, k=8, zipf=1.2, padding=1),
        # the router of the sparse layer of 8 experts, gates renormalised over two winners
        _case("route_grad", 8192, name="route_grad_batch", E=8, k=2, cf=2.0),
        # the library's limit of 256 experts, the softmax over all of them, many dropped pairs, padding
        _case("route_grad", 32768, name="route_grad_256", E=256, k=8, zipf=1.2, renorm=0, cf=1.25, padding=1),
        # gate projection of the sparse layer of 8 experts, with the gradient that comes back through the dispatch
        _case("gate_grad", 8192, 4096, "bf16", "gate_grad_batch", E=8, k=2, other=1),
        # ... of the largest named workload
        _case("gate_grad", 65536, 7168, "bf16", "gate_grad_skewed", E=64, k=8, zipf=1.2),
        # 32 bits, odd sizes
        _case("gate_grad", 1155, 516, "f32", "gate_grad_f32_odd", E=10, k=3, other=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["layernorm", "layernorm_grad", "route_loss", "route_grad", "gate_grad", "gate_grad"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        bpe = 4 if dtype == "f32" else 2
        fp8 = int(kind == "layernorm" and rng.random() < 0.6)
        unit = 16 if fp8 else 16 // bpe
        H = unit * max(1, _log(rng, 64, 8192) // unit) if rng.random() < 0.5 else rng.choice([512, 1024, 2048, 4096, 5120, 7168, 8192])
        T = _log(rng, 1, 65536)
        other = rng.randint(0, 1)
        if kind in ("layernorm", "layernorm_grad"):
            if T * H * bpe > 8192 * 4096 * 2:
                continue
            return _case(kind, T, H, dtype, other=other, fp8=fp8)
        E = rng.choice([2, 4, 8, 8, 16, 32, 64, 128, 256, rng.randint(2, 256)])
        k = min(E, rng.choice([1, 2, 2, 4, 6, 8]))
        zipf = rng.choice([0.0, 0.0, 0.8, 1.2])
        if kind == "gate_grad":
            if T * H * E > 65536 * 7168 * 64 // (1 if dtype == "bf16" else 4) or T * H * bpe > 65536 * 7168 * 2:
                continue
            return _case(kind, T, H, dtype, E=E, k=k, zipf=zipf, other=other)
        return _case(kind, T, E=E, k=k, zipf=zipf, renorm=rng.choice([1, 1, 0]), cf=rng.choice([0.0, 2.0, 1.25, 0.7]),
                     padding=rng.randint(0, 1), losses=int(kind == "route_loss" or rng.random() < 0.8))


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _fp8_row_bytes(H):
    """Codes, then a 32-bit scale for each block, in whole 128-byte lines."""
    return (H + 4 * _blocks(H) + 127) // 128 * 128


# ------------------------------------------------------------------------------------------------ inputs


class _State:
    pass


def _choices(c, logits):
    """The router's choices in torch: expert ids and gates [T, k]."""
    top, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    top, idx = top[:, :c["top_k"]], idx[:, :c["top_k"]]
    gates = torch.softmax(top, dim=1) if c["renorm"] else torch.gather(torch.softmax(logits, dim=1), 1, idx)
    return idx.to(torch.int32).contiguous(), gates.contiguous()


def _kept(c, idx):
    """Which pairs a capacity leaves: the first ones of each expert, in token order."""
    T, E, k = c["tokens"], c["experts"], c["top_k"]
    if c["capacity_factor"] <= 0:
        return torch.ones((T, k), dtype=torch.bool, device=idx.device)
    C = min(T, math.ceil(c["capacity_factor"] * T * k / E))
    flat = idx.reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=E)
    rank = torch.empty_like(flat)
    rank[order] = torch.arange(T * k, device=flat.device) - (torch.cumsum(counts, 0) - counts)[flat[order]]
    return (rank < C).view(T, k)


def prepare(case, seed):
    c, s = case, _State()
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, H, E, k, dt = c["tokens"], c["hidden"], c["experts"], c["top_k"], _dtype(c)

    def normal(*shape, scale=1.0, dtype=None):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype or dt).mul_(scale)

    s.c, s.kind, s.H, s.dt = c, c["kind"], H, dt
    if own:                      # what a program that uses the library keeps: its module, the configuration, buffers
        import paper_2411_00662_amd as m
        s.m = m
        s.cfg = m.make_cfg(T, H, m.FP32 if c["dtype"] == "f32" else m.BF16, E, k, 1, 1, 1, c["capacity_factor"], c["renorm"])

    def scratch(nbytes):
        return torch.empty(nbytes, dtype=torch.uint8, device="cuda")

    if s.kind in ("layernorm", "layernorm_grad"):
        s.w, s.b = (1.0 + normal(H, scale=0.2, dtype=torch.float32)).to(dt), normal(H, scale=0.1)
        # channels with an offset of their own, as the stream of a deep model has them
        s.x = normal(T, H, scale=1.5) + normal(H)
        s.other = normal(T, H) if c["other"] else None
        s.out = torch.empty_like(s.x)
        if s.kind == "layernorm":
            s.sum = torch.empty_like(s.x) if c["other"] else None
            s.rows8 = scratch(T * _fp8_row_bytes(H)).view(T, -1) if c["fp8"] else None
            return s
        s.dout = normal(T, H, scale=0.1)
        s.dw, s.db = (torch.empty(H, dtype=torch.float32, device="cuda") for _ in range(2))
        if own:
            s.scratch = scratch(m.monta_layernorm_scratch_bytes(s.cfg))
        return s

    s.logits = normal(T, E, dtype=torch.float32)
    if c["zipf"] > 0:
        s.logits -= c["zipf"] * torch.log(torch.arange(1, E + 1, device="cuda", dtype=torch.float32))
    s.idx, s.gates = _choices(c, s.logits)
    if s.kind == "gate_grad":
        # large at the choices, small everywhere from the losses
        s.dlogits = normal(T, E, scale=1e-4, dtype=torch.float32)
        s.dlogits.scatter_add_(1, s.idx.long(), normal(T, k, scale=0.02, dtype=torch.float32))
        s.x, s.w = normal(T, H), normal(E, H, scale=H ** -0.5)
        s.other = normal(T, H, scale=0.1) if c["other"] else None
        s.dx, s.dw = torch.empty_like(s.x), torch.empty((E, H), dtype=torch.float32, device="cuda")
        if own:
            s.scratch = scratch(m.monta_gate_backward_scratch_bytes(s.cfg))
        return s
    s.mask = None
    if c["padding"]:             # the last eighth of every 64 tokens is padding
        s.mask = (torch.arange(T, device="cuda") % 64 < 56).to(torch.uint8)
    live = torch.ones(T, dtype=torch.bool, device="cuda") if s.mask is None else s.mask.bool()
    s.counts = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    s.counts[:E] = torch.bincount(s.idx[live].reshape(-1).long(), minlength=E)
    s.counts[E] = live.sum()
    if s.kind == "route_loss":
        s.counts.zero_()
        s.losses, s.means = torch.empty(2, device="cuda"), torch.empty(E, device="cuda")
        if own:
            s.scratch = scratch(m.monta_route_loss_scratch_bytes(s.cfg))
        return s
    s.dgates = normal(T, k, scale=0.1, dtype=torch.float32) * _kept(c, s.idx)
    s.dlosses = torch.tensor(LOSS_WEIGHTS, device="cuda") if c["losses"] else None
    s.dlogits = torch.empty_like(s.logits)
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(s):
    return (_run_own if own else _run_plain)[s.kind](s)


def _own_layernorm(s):
    s.m.monta_layernorm(s.cfg, s.x, s.other, s.w, s.b, EPS, s.sum, s.out, s.rows8)
    got = {"out": s.out}
    if s.other is not None:
        got["sum"] = s.sum
    if s.rows8 is not None:
        got["codes"] = s.rows8[:, :s.H].view(torch.float8_e4m3fn)
        got["scales"] = s.rows8[:, s.H:s.H + 4 * _blocks(s.H)].view(torch.float32)
    return got


def _own_layernorm_grad(s):
    s.m.monta_layernorm_backward(s.cfg, s.x, s.w, EPS, s.dout, s.other, s.out, s.dw, s.db, s.scratch)
    return {"dx": s.out, "dw": s.dw, "db": s.db}


def _own_route_loss(s):
    s.m.monta_route_loss(s.cfg, s.logits, s.idx, s.mask, s.losses, s.counts, s.means, s.scratch)
    return {"losses": s.losses, "counts": s.counts, "means": s.means}


def _own_route_grad(s):
    s.m.monta_route_backward(s.cfg, s.logits, s.idx, s.gates, s.dgates, s.mask, s.dlosses, s.counts, s.dlogits)
    return {"dlogits": s.dlogits}


def _own_gate_grad(s):
    s.m.monta_gate_backward(s.cfg, s.dlogits, s.x, s.w, s.other, s.dx, s.dw, s.scratch)
    return {"dx": s.dx, "dw": s.dw}


_run_own = {"layernorm": _own_layernorm, "layernorm_grad": _own_layernorm_grad, "route_loss": _own_route_loss,
            "route_grad": _own_route_grad, "gate_grad": _own_gate_grad}


def _standard(t):
    """float32 [T, H] -> rows of mean 0 and variance 1, and the factor that made them so."""
    t = t - t.mean(dim=1, keepdim=True)
    r = torch.rsqrt((t * t).mean(dim=1, keepdim=True) + EPS)
    return t * r, r


def _quantise(v):
    """float32 [T, H] -> (codes [T, H], scales [T, blocks])."""
    T, H = v.shape
    full = torch.zeros((T, _blocks(H) * BLOCK), dtype=v.dtype, device=v.device)
    full[:, :H] = v
    tiles = full.view(T, _blocks(H), BLOCK)
    amax = tiles.abs().amax(dim=2).clamp_min(AMAX_FLOOR)
    codes = (tiles * (E4M3_MAX / amax)[..., None]).clamp(-E4M3_MAX, E4M3_MAX)
    return codes.view(T, -1)[:, :H].to(torch.float8_e4m3fn), amax / E4M3_MAX


def _plain_layernorm(s):
    got, t = {}, s.x
    if s.other is not None:
        t = (s.x.float() + s.other.float()).to(s.dt)
        got["sum"] = t
    v = _standard(t.float())[0] * s.w.float() + s.b.float()
    got["out"] = v.to(s.dt)
    if s.c["fp8"]:
        got["codes"], got["scales"] = _quantise(v)
    return got


def _plain_layernorm_grad(s):
    n, r = _standard(s.x.float())
    d = s.dout.float()
    g = d * s.w.float()
    dx = r * (g - g.mean(dim=1, keepdim=True) - n * (g * n).mean(dim=1, keepdim=True))
    if s.other is not None:
        dx = dx + s.other.float()
    return {"dx": dx.to(s.dt), "dw": (d * n).sum(dim=0), "db": d.sum(dim=0)}


def _live(s):
    """1 for a token that counts, 0 for padding, as a column."""
    if s.mask is None:
        return torch.ones((s.c["tokens"], 1), device="cuda")
    return (s.mask != 0).float()[:, None]


def _softmax(logits):
    top = logits.amax(dim=1, keepdim=True)
    e = torch.exp(logits - top)
    z = e.sum(dim=1, keepdim=True)
    return e / z, top + torch.log(z)


def _plain_route_loss(s):
    E, k = s.c["experts"], s.c["top_k"]
    live = _live(s)
    n = live.sum()
    p, lse = _softmax(s.logits)
    means = (p * live).sum(dim=0) / n.clamp_min(1)
    counts = torch.zeros(E + 1, device="cuda", dtype=torch.int64)
    experts = torch.where(live > 0, torch.arange(E, device="cuda"), -1)          # no pair of a padding token matches
    for j in range(k):
        counts[:E] += (s.idx[:, j:j + 1] == experts).sum(dim=0)
    counts[E] = (live > 0).sum()
    share = counts[:E].float() * (E / k) / n.clamp_min(1)
    losses = torch.stack([(share * means).sum(), (lse * lse * live).sum() / n.clamp_min(1)])
    return {"losses": losses, "counts": counts.to(torch.int32), "means": means}


def _plain_route_grad(s):
    E, k = s.c["experts"], s.c["top_k"]
    idx, live = s.idx.long(), _live(s)
    dot = (s.gates * s.dgates).sum(dim=1, keepdim=True)
    p, lse = _softmax(s.logits)
    if s.c["renorm"]:
        d = torch.zeros_like(s.logits).scatter_add_(1, idx, s.gates * (s.dgates - dot))
    else:
        d = torch.zeros_like(s.logits).scatter_add_(1, idx, s.gates * s.dgates) - p * dot
    if s.dlosses is not None:
        n = s.counts[E].float().clamp_min(1)
        share = s.counts[:E].float() * (E / k) / n
        d = d + p * ((share - (p * share).sum(dim=1, keepdim=True)) * (s.dlosses[0] / n) + 2.0 * lse * (s.dlosses[1] / n))
    return {"dlogits": d * live}


def _plain_gate_grad(s):
    dx = s.dlogits @ s.w.float()
    if s.other is not None:
        dx = dx + s.other.float()
    return {"dx": dx.to(s.dt), "dw": s.dlogits.t() @ s.x.float()}


_run_plain = {"layernorm": _plain_layernorm, "layernorm_grad": _plain_layernorm_grad, "route_loss": _plain_route_loss,
              "route_grad": _plain_route_grad, "gate_grad": _plain_gate_grad}


# ------------------------------------------------------------------------------------------------ what a pass needs


def work(case):
    """Bytes that a pass has to read and write once each, and operations."""
    c = case
    T, H, E, k = c["tokens"], c["hidden"], c["experts"], c["top_k"]
    row = H * (4 if c["dtype"] == "f32" else 2)
    if c["kind"] == "layernorm":
        moved = T * row * (4 if c["other"] else 2) + 2 * row + (T * (H + 4 * _blocks(H)) if c["fp8"] else 0)
        return {"bytes": moved, "flops": 8 * T * H}
    if c["kind"] == "layernorm_grad":
        return {"bytes": T * row * (4 if c["other"] else 3) + row + 8 * H, "flops": 14 * T * H}
    if c["kind"] == "gate_grad":
        return {"bytes": T * E * 4 + T * row * (3 if c["other"] else 2) + E * row + E * H * 4, "flops": 4 * T * E * H}
    live = T - sum(1 for t in range(T) if t % 64 >= 56) if c["padding"] else T
    mask = T if c["padding"] else 0
    if c["kind"] == "route_loss":
        return {"bytes": live * (E + k) * 4 + mask + 8 * E + 12, "flops": 6 * live * E}
    # gates that are renormalised over the winners, and no losses: the logits are not needed
    logits = live * E * 4 if c["losses"] or not c["renorm"] else 0
    return {"bytes": logits + live * k * 12 + mask + T * E * 4 + (4 * E + 12 if c["losses"] else 0), "flops": 8 * live * E}


# ------------------------------------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    """The same outputs from the definitions in 64 bits; gradients by differentiating those."""
    s, f = prepare(case, seed), torch.float64
    c, H, E, k, T = case, s.H, case["experts"], case["top_k"], case["tokens"]
    if s.kind == "layernorm":
        got, t = {}, s.x.to(f)
        if s.other is not None:
            got["sum"] = t + s.other.to(f)
            t = got["sum"].to(torch.float32).to(s.dt).to(f)         # the norm is that of the sum as it is stored
        var, mean = torch.var_mean(t, dim=1, correction=0, keepdim=True)
        got["out"] = (t - mean) / (var + EPS).sqrt() * s.w.to(f) + s.b.to(f)
        if c["fp8"]:
            nb = _blocks(H)
            codes, scales = torch.empty_like(t), torch.empty((T, nb), dtype=f, device="cuda")
            for b in range(nb):
                v = got["out"][:, b * BLOCK:(b + 1) * BLOCK]
                scales[:, b] = v.abs().max(1).values.clamp_min(AMAX_FLOOR) / E4M3_MAX
                codes[:, b * BLOCK:(b + 1) * BLOCK] = (v / scales[:, b:b + 1]).to(torch.float32).to(torch.float8_e4m3fn).to(f)
            got["codes"], got["scales"] = codes, scales
        return got
    if s.kind == "layernorm_grad":
        t, w, b = s.x.to(f).requires_grad_(), s.w.to(f).requires_grad_(), torch.zeros(H, dtype=f, device="cuda", requires_grad=True)
        var, mean = torch.var_mean(t, dim=1, correction=0, keepdim=True)
        dx, dw, db = torch.autograd.grad((t - mean) / (var + EPS).sqrt() * w + b, [t, w, b], s.dout.to(f))
        return {"dx": dx if s.other is None else dx + s.other.to(f), "dw": dw, "db": db}
    if s.kind == "gate_grad":
        dw, dx = torch.empty((E, H), dtype=f, device="cuda"), torch.zeros((T, H), dtype=f, device="cuda")
        x, w = s.x.to(f), s.w.to(f)
        for e in range(E):
            d = s.dlogits[:, e].to(f)
            dw[e] = d @ x
            dx += d[:, None] * w[e]
        return {"dx": dx if s.other is None else dx + s.other.to(f), "dw": dw}
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s.mask is None else s.mask != 0
    logits, idx = s.logits.to(f).requires_grad_(), s.idx.long()
    live, n = logits[keep], max(1, int(keep.sum()))
    chosen = torch.bincount(idx[keep].reshape(-1), minlength=E)
    means = torch.softmax(live, dim=1).sum(dim=0) / n
    balance = (chosen.to(f) * E / (n * k) * means).sum()
    z = (torch.logsumexp(live, dim=1) ** 2).sum() / n
    if s.kind == "route_loss":
        counts = torch.cat([chosen, keep.sum()[None]]).to(torch.int32)
        return {"losses": torch.stack([balance, z]).detach(), "counts": counts, "means": means.detach()}
    won = torch.gather(live, 1, idx[keep])
    gates = torch.softmax(won, dim=1) if c["renorm"] else torch.exp(won - torch.logsumexp(live, dim=1, keepdim=True))
    whole = (gates * s.dgates[keep].to(f)).sum()
    if s.dlosses is not None:
        whole = whole + balance * s.dlosses[0].to(f) + z * s.dlosses[1].to(f)
    return {"dlogits": torch.autograd.grad(whole, logits)[0]}
