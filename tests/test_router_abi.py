"""Host-only checks of the layer norm, the router's losses and gradient, and the gate's gradient: sizes, and refusals before any HIP call."""
import ctypes

import pytest

import paper_2411_00662_amd as m
from paper_2411_00662_amd import binding as B

A = [0x1000000000 * (i + 1) for i in range(12)]        # addresses far apart; never dereferenced: validation fails first


def cfg(tokens=8, hidden=512, dtype=m.BF16, experts=4, top_k=2, slices=2, **kw):
    return m.make_cfg(tokens, hidden, dtype, experts, top_k, 1, 1, slices, **kw)


def layernorm(c, x=A[0], residual=A[1], w=A[2], b=A[3], eps=1e-5, s=A[4], out=A[5], out8=A[6]):
    return B.lib().monta_layernorm(ctypes.byref(c), x, residual, w, b, eps, s, out, out8, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), -3), (dict(w=0), -3), (dict(out=0, out8=0), -3), (dict(s=0), -3),
    (dict(residual=0), -1),                                             # a sum of nothing
    (dict(x=A[0] + 8), -5), (dict(residual=A[1] + 4), -5), (dict(w=A[2] + 2), -5), (dict(b=A[3] + 2), -5), (dict(s=A[4] + 8), -5),
    (dict(out=A[5] + 8), -5), (dict(out8=A[6] + 8), -5),
    (dict(eps=-1e-5), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(s=A[0] + 1024), -1), (dict(out=A[0] + 1024), -1), (dict(out=A[4]), -1), (dict(s=A[1] - 16), -1), (dict(out=A[1] + 16), -1),
    (dict(out8=A[0]), -1), (dict(out8=A[1]), -1), (dict(out8=A[2]), -1), (dict(out8=A[3]), -1), (dict(out8=A[4]), -1), (dict(out8=A[5]), -1),
    (dict(s=A[2]), -1), (dict(s=A[3]), -1), (dict(out=A[2]), -1), (dict(out=A[3]), -1)])
def test_layernorm_refuses(kw, code):
    assert layernorm(cfg(), **kw) == code


def test_layernorm_sizes():
    assert layernorm(cfg(hidden=520)) == -1                             # 8-bit rows need whole 16-byte pieces
    assert layernorm(cfg(hidden=16392), out8=0) == -2                   # rows beyond 32 KiB
    assert layernorm(cfg(hidden=8196, dtype=m.FP32), out8=0) == -2
    assert layernorm(cfg(hidden=513)) == -1
    with pytest.raises(m.MontaError) as e:
        m.monta_layernorm_scratch_bytes(cfg(hidden=16392))
    assert e.value.code == -2
    assert m.monta_layernorm_scratch_bytes(cfg(tokens=1, slices=1, hidden=4096)) == 4096 * 8
    assert m.monta_layernorm_scratch_bytes(cfg(tokens=1 << 20, hidden=4096)) <= 1 << 24
    assert B.lib().monta_layernorm_scratch_bytes(ctypes.byref(cfg()), None) == -3


@pytest.mark.parametrize("name", ["monta_layernorm_scratch_bytes", "monta_route_loss_scratch_bytes", "monta_gate_backward_scratch_bytes"])
@pytest.mark.parametrize("hidden,experts", [(128, 4), (1024, 16), (1536, 64), (4096, 100), (8192, 256)])
def test_scratch_for_more_tokens_does_for_fewer(name, hidden, experts):
    for dtype in (m.BF16, m.FP32):
        last = 0
        for tokens in [*range(1, 1200), 1999, 2048, 2049, 4097, 8192, 8193, 16384, 30000, 32769, 65536, 1 << 20, 1 << 24]:
            n = getattr(m, name)(cfg(tokens=tokens, hidden=hidden, dtype=dtype, experts=experts, top_k=1, slices=1))
            assert n >= last, tokens
            last = n


def layernorm_backward(c, s=A[0], w=A[1], eps=1e-5, dout=A[2], dsum=A[3], dx=A[4], dw=A[5], db=A[6], scratch=A[7]):
    return B.lib().monta_layernorm_backward(ctypes.byref(c), s, w, eps, dout, dsum, dx, dw, db, scratch, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(s=0), -3), (dict(w=0), -3), (dict(dout=0), -3), (dict(dx=0), -3), (dict(dw=0), -3), (dict(scratch=0), -3),
    (dict(s=A[0] + 8), -5), (dict(w=A[1] + 8), -5), (dict(dout=A[2] + 8), -5), (dict(dsum=A[3] + 8), -5), (dict(dx=A[4] + 8), -5), (dict(dw=A[5] + 2), -5),
    (dict(db=A[6] + 2), -5), (dict(scratch=A[7] + 4), -5),
    (dict(eps=-1.0), -1), (dict(dx=A[0] + 512), -1), (dict(dx=A[1]), -1), (dict(dw=A[2]), -1), (dict(dw=A[4]), -1), (dict(db=A[5]), -1), (dict(db=A[2]), -1),
    (dict(db=A[5] + 2044), -1), (dict(scratch=A[0]), -1), (dict(scratch=A[1]), -1), (dict(scratch=A[4]), -1), (dict(scratch=A[5]), -1), (dict(scratch=A[6]), -1)])
def test_layernorm_backward_refuses(kw, code):
    assert layernorm_backward(cfg(), **kw) == code
    assert layernorm_backward(cfg(hidden=16392), **kw) in (code, -2)


def route_loss(c, logits=A[0], idx=A[1], mask=A[2], losses=A[3], counts=A[4], means=A[5], scratch=A[6]):
    return B.lib().monta_route_loss(ctypes.byref(c), logits, idx, mask, losses, counts, means, scratch, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(logits=0), -3), (dict(idx=0), -3), (dict(losses=0), -3), (dict(counts=0), -3), (dict(means=0), -3), (dict(scratch=0), -3),
    (dict(logits=A[0] + 2), -5), (dict(idx=A[1] + 1), -5), (dict(losses=A[3] + 2), -5), (dict(counts=A[4] + 2), -5), (dict(means=A[5] + 2), -5),
    (dict(scratch=A[6] + 8), -5),
    (dict(losses=A[0]), -1), (dict(counts=A[1]), -1), (dict(means=A[2]), -1), (dict(means=A[2] + 4), -1), (dict(counts=A[3]), -1), (dict(means=A[3]), -1),
    (dict(means=A[4] + 16), -1), (dict(scratch=A[0]), -1), (dict(scratch=A[1]), -1), (dict(scratch=A[5]), -1)])
def test_route_loss_refuses(kw, code):
    assert route_loss(cfg(), **kw) == code


def test_route_loss_sizes():
    assert route_loss(cfg(top_k=5)) == -1
    assert route_loss(cfg(experts=257)) in (-1, -2)
    assert B.lib().monta_route_loss_scratch_bytes(ctypes.byref(cfg()), None) == -3
    for tokens, experts in ((1, 1), (65536, 64), (2 ** 31 - 1, 256), (2 ** 31 - 1, 1), (8191, 255)):
        n = m.monta_route_loss_scratch_bytes(cfg(tokens=tokens, experts=experts, top_k=1, slices=1))
        assert 8 * (experts + 1) <= n <= 1024 + 512 * 8 * (experts + 1)


def route_backward(c, logits=A[0], idx=A[1], gates=A[2], dgates=A[3], mask=A[4], dlosses=A[5], counts=A[6], dlogits=A[7]):
    return B.lib().monta_route_backward(ctypes.byref(c), logits, idx, gates, dgates, mask, dlosses, counts, dlogits, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(logits=0), -3), (dict(idx=0), -3), (dict(gates=0), -3), (dict(dgates=0, dlosses=0), -3), (dict(counts=0), -3), (dict(dlogits=0), -3),
    (dict(logits=A[0] + 2), -5), (dict(idx=A[1] + 2), -5), (dict(gates=A[2] + 2), -5), (dict(dgates=A[3] + 1), -5), (dict(dlosses=A[5] + 2), -5),
    (dict(counts=A[6] + 2), -5), (dict(dlogits=A[7] + 2), -5),
    (dict(dlogits=A[0]), -1), (dict(dlogits=A[1]), -1), (dict(dlogits=A[2] + 4), -1), (dict(dlogits=A[3]), -1), (dict(dlogits=A[4] - 124), -1),
    (dict(dlogits=A[5]), -1), (dict(dlogits=A[6]), -1)])
def test_route_backward_refuses(kw, code):
    assert route_backward(cfg(), **kw) == code
    assert route_backward(cfg(top_k=5), **kw) == -1


def gate_backward(c, dl=A[0], x=A[1], w=A[2], dadd=A[3], dx=A[4], dw=A[5], scratch=A[6]):
    return B.lib().monta_gate_backward(ctypes.byref(c), dl, x, w, dadd, dx, dw, scratch, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(dl=0), -3), (dict(dx=0, dw=0, dadd=0), -3), (dict(w=0), -3), (dict(x=0), -3), (dict(scratch=0), -3), (dict(dx=0, dadd=0, x=0), -3),
    (dict(dw=0, w=0), -3),
    (dict(dx=0), -1),                                                   # something to add to nothing
    (dict(dl=A[0] + 2), -5), (dict(x=A[1] + 8), -5), (dict(w=A[2] + 8), -5), (dict(dadd=A[3] + 8), -5), (dict(dx=A[4] + 8), -5), (dict(dw=A[5] + 4), -5),
    (dict(scratch=A[6] + 4), -5),
    (dict(dx=A[0]), -1), (dict(dx=A[1]), -1), (dict(dx=A[2]), -1), (dict(dx=A[3] + 1024), -1), (dict(dw=A[0]), -1), (dict(dw=A[1]), -1), (dict(dw=A[2]), -1),
    (dict(x=A[3], dx=A[3]), -1), (dict(w=A[3], dx=A[3]), -1), (dict(dl=A[3], dx=A[3]), -1),          # dadd itself, but another argument, too
    (dict(dw=A[3]), -1), (dict(dw=A[4]), -1), (dict(scratch=A[0]), -1), (dict(scratch=A[4]), -1), (dict(scratch=A[5]), -1)])
def test_gate_backward_refuses(kw, code):
    assert gate_backward(cfg(), **kw) == code


def test_gate_backward_sizes():
    assert gate_backward(cfg(hidden=(1 << 20) + 8)) == -2
    assert gate_backward(cfg(top_k=5)) == -1
    with pytest.raises(m.MontaError) as e:
        m.monta_gate_backward_scratch_bytes(cfg(hidden=(1 << 20) + 8))
    assert e.value.code == -2
    assert B.lib().monta_gate_backward_scratch_bytes(ctypes.byref(cfg()), None) == -3
    for dtype in (m.FP32, m.BF16):
        for tokens, hidden, experts in ((1, 8, 1), (65536, 7168, 64), (2 ** 31 - 1, 16, 256), (2 ** 31 - 1, 1 << 20, 2), (3, 1 << 20, 256), (100000, 64, 9)):
            n = m.monta_gate_backward_scratch_bytes(cfg(tokens=tokens, hidden=hidden, dtype=dtype, experts=experts, top_k=1, slices=1))
            assert n == 16 or (n % (experts * hidden * 4) == 0 and n // (experts * hidden * 4) <= 1024)


CALLS = {
    "monta_layernorm": (["x", "residual", "weight", "bias", "sum", "out", "out_fp8"], dict(eps=1e-5)),
    "monta_layernorm_backward": (["sum", "weight", "dout", "dsum", "dx", "dweight", "dbias", "scratch"], dict(eps=1e-5)),
    "monta_route_loss": (["logits", "topk_idx", "token_mask", "losses", "counts", "means", "scratch"], {}),
    "monta_route_backward": (["logits", "topk_idx", "gates", "dgates", "token_mask", "dlosses", "counts", "dlogits"], {}),
    "monta_gate_backward": (["dlogits", "x", "w_gate", "dadd", "dx", "dw_gate", "scratch"], {}),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_marshalling_refuses(name):
    """Host tensors and other objects by name, before anything else; addresses as they are."""
    import torch
    names, kw = CALLS[name]
    c = cfg()
    for bad in names:
        bufs = {n: A[i] for i, n in enumerate(names)}
        bufs[bad] = torch.zeros(4096)
        with pytest.raises(ValueError, match=f"^{bad}: expected a device tensor$"):
            getattr(m, name)(c, **bufs, **kw, stream=0)
        bufs[bad] = "text"
        with pytest.raises(AttributeError, match="is_cuda"):
            getattr(m, name)(c, **bufs, **kw, stream=0)
        if bad != "token_mask":                                         # bytes lie anywhere
            bufs[bad] = 3
            with pytest.raises(m.MontaError, match=f"^{name}: ") as e:
                getattr(m, name)(c, **bufs, **kw, stream=0)
            assert e.value.code == -5
    bufs = {n: A[i] for i, n in enumerate(names)}
    bufs[names[0]] = None
    with pytest.raises(m.MontaError, match=f"^{name}: ") as e:
        getattr(m, name)(c, **bufs, **kw, stream=0)
    assert e.value.code == -3
    with pytest.raises(m.MontaError) as e:
        getattr(m, name)(cfg(top_k=5), **{n: A[i] for i, n in enumerate(names)}, **kw, stream=0)
    assert e.value.code == -1
    with pytest.raises(TypeError):
        getattr(m, name)("cfg", **{n: A[i] for i, n in enumerate(names)}, **kw, stream=0)
