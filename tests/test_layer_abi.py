"""Host-only checks of the norm, the 8-bit expert layer and the gradients: sizes, and refusals before any HIP call."""
import ctypes

import pytest

import paper_2411_00662_amd as m
from paper_2411_00662_amd import binding as B

A = [0x10000000 * (i + 1) for i in range(12)]          # addresses far apart; never dereferenced: validation fails first


def cfg(tokens=8, hidden=512, dtype=m.BF16, experts=4, top_k=2, slices=2, **kw):
    return m.make_cfg(tokens, hidden, dtype, experts, top_k, 1, 1, slices, **kw)


@pytest.mark.parametrize("hidden,row", [(16, 128), (128, 256), (112, 128), (496, 512), (512, 640), (4096, 4224), (7168, 7424), (528, 640)])
def test_fp8_rows(hidden, row):
    """hidden codes, a 4-byte scale per 128 of them, whole 128-byte lines; moved as bf16 rows of half as many elements."""
    assert row == -(-(hidden + 4 * -(-hidden // 128)) // 128) * 128
    for dtype in (m.FP32, m.BF16):
        c = cfg(hidden=hidden, dtype=dtype, capacity_factor=0.75, renorm=0, padded=1)
        rows, n = m.monta_fp8_rows(c)
        assert n == row and rows.hidden == row // 2 and rows.dtype == m.BF16
        for f, _ in B.monta_cfg._fields_:
            if f not in ("hidden", "dtype"):
                assert getattr(rows, f) == getattr(c, f)
        # one workspace serves both configurations
        a, b = m.monta_ws_layout_query(c), m.monta_ws_layout_query(rows)
        assert all(getattr(a, f) == getattr(b, f) for f, _ in B.monta_ws_layout._fields_)


def test_fp8_rows_refuses():
    lib, c = B.lib(), cfg()
    rows, n = m.monta_cfg(), ctypes.c_int64(0)
    r, p = ctypes.byref(rows), ctypes.byref(n)
    assert lib.monta_fp8_rows(ctypes.byref(c), None, p) == -3
    assert lib.monta_fp8_rows(ctypes.byref(c), r, None) == -3
    assert lib.monta_fp8_rows(None, r, p) == -3
    assert lib.monta_fp8_rows(ctypes.byref(cfg(hidden=520)), r, p) == -1        # not whole 16-byte pieces of codes
    assert lib.monta_fp8_rows(ctypes.byref(cfg(top_k=5)), r, p) == -1


def rmsnorm(c, x=A[0], residual=A[1], w=A[2], eps=1e-5, s=A[3], out=A[4], out8=A[5]):
    return B.lib().monta_rmsnorm(ctypes.byref(c), x, residual, w, eps, s, out, out8, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), -3), (dict(w=0), -3), (dict(out=0, out8=0), -3), (dict(s=0), -3),
    (dict(residual=0), -1),                                             # a sum of nothing
    (dict(x=A[0] + 8), -5), (dict(residual=A[1] + 4), -5), (dict(w=A[2] + 2), -5), (dict(s=A[3] + 8), -5), (dict(out=A[4] + 8), -5),
    (dict(out8=A[5] + 8), -5),
    (dict(eps=-1e-5), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(s=A[0] + 1024), -1), (dict(out=A[0] + 1024), -1), (dict(out=A[3]), -1), (dict(s=A[1] - 16), -1), (dict(out=A[1] + 16), -1),
    (dict(out8=A[0]), -1), (dict(out8=A[1]), -1), (dict(out8=A[2]), -1), (dict(out8=A[3]), -1), (dict(out8=A[4]), -1),
    (dict(s=A[2]), -1), (dict(out=A[2]), -1)])
def test_rmsnorm_refuses(kw, code):
    assert rmsnorm(cfg(), **kw) == code


def test_rmsnorm_sizes():
    assert rmsnorm(cfg(hidden=520)) == -1                               # 8-bit rows need whole 16-byte pieces
    assert rmsnorm(cfg(hidden=16392), out8=0) == -2                     # rows beyond 32 KiB
    assert rmsnorm(cfg(hidden=8196, dtype=m.FP32), out8=0) == -2
    assert rmsnorm(cfg(hidden=513)) == -1
    with pytest.raises(m.MontaError) as e:
        m.monta_rmsnorm_scratch_bytes(cfg(hidden=16392))
    assert e.value.code == -2
    assert m.monta_rmsnorm_scratch_bytes(cfg(tokens=1, slices=1, hidden=4096)) == 4096 * 4
    assert m.monta_rmsnorm_scratch_bytes(cfg(tokens=1 << 20, hidden=4096)) <= 1 << 24


def backward(c, s=A[0], w=A[1], eps=1e-5, dout=A[2], dsum=A[3], dx=A[4], dw=A[5], scratch=A[6]):
    return B.lib().monta_rmsnorm_backward(ctypes.byref(c), s, w, eps, dout, dsum, dx, dw, scratch, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(s=0), -3), (dict(w=0), -3), (dict(dout=0), -3), (dict(dx=0), -3), (dict(dw=0), -3), (dict(scratch=0), -3),
    (dict(s=A[0] + 8), -5), (dict(dsum=A[3] + 8), -5), (dict(dw=A[5] + 2), -5), (dict(scratch=A[6] + 4), -5),
    (dict(eps=-1.0), -1), (dict(dx=A[0] + 512), -1), (dict(dx=A[1]), -1), (dict(dw=A[2]), -1), (dict(dw=A[4]), -1), (dict(scratch=A[0]), -1),
    (dict(scratch=A[1]), -1), (dict(scratch=A[4]), -1), (dict(scratch=A[5]), -1)])
def test_rmsnorm_backward_refuses(kw, code):
    assert backward(cfg(), **kw) == code
    assert backward(cfg(hidden=16392), **kw) in (code, -2)


def combine(c, dout=A[0], y=A[1], gates=A[2], dy=A[3], dgates=A[4], ws=A[5]):
    return B.lib().monta_combine_backward(ctypes.byref(c), dout, y, gates, dy, dgates, ws, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(dout=0), -3), (dict(y=0), -3), (dict(gates=0), -3), (dict(dy=0), -3), (dict(dgates=0), -3), (dict(ws=0), -3),
    (dict(dout=A[0] + 8), -5), (dict(gates=A[2] + 2), -5), (dict(dgates=A[4] + 1), -5), (dict(ws=A[5] + 8), -5),
    (dict(dy=A[1]), -1), (dict(dy=A[0]), -1), (dict(dgates=A[2]), -1), (dict(dy=A[5]), -1), (dict(dgates=A[5]), -1), (dict(dgates=A[3]), -1)])
def test_combine_backward_refuses(kw, code):
    assert combine(cfg(), **kw) == code


def test_combine_backward_sizes():
    assert combine(cfg(hidden=16392)) == -2
    assert combine(cfg(top_k=5)) == -1


def expert8(c, x=A[0], w=A[1], scales=A[2], n=256, y=A[3], ws=A[4], slice=-1):
    return B.lib().monta_expert_linear_fp8(ctypes.byref(c), x, w, scales, n, y, ws, slice, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), -3), (dict(w=0), -3), (dict(scales=0), -3), (dict(y=0), -3), (dict(ws=0), -3),
    (dict(x=A[0] + 8), -5), (dict(w=A[1] + 8), -5), (dict(scales=A[2] + 2), -5), (dict(y=A[3] + 8), -5), (dict(ws=A[4] + 8), -5),
    (dict(n=0), -1), (dict(n=-8), -1), (dict(n=252), -1), (dict(slice=-2), -1), (dict(slice=2), -1),
    (dict(y=A[0]), -1), (dict(y=A[1]), -1), (dict(y=A[2]), -1), (dict(y=A[4]), -1)])
def test_expert_linear_fp8_refuses(kw, code):
    assert expert8(cfg(), **kw) == code


def test_expert_linear_fp8_sizes():
    assert expert8(cfg(hidden=520)) == -1
    assert expert8(cfg(hidden=65536 + 16)) == -2
    assert expert8(cfg(), n=(1 << 20) + 8) == -2
    assert expert8(cfg(tokens=2 ** 31 - 4096, hidden=16, top_k=1, slices=1), n=8) == -2


def grads(c, dy=A[0], x=A[1], w=A[2], n=256, dx=A[3], dw=A[4], ws=A[5]):
    return B.lib().monta_expert_linear_backward(ctypes.byref(c), dy, x, w, n, dx, dw, ws, 0)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=0), -3), (dict(ws=0), -3), (dict(dx=0, dw=0), -3), (dict(w=0), -3), (dict(x=0), -3), (dict(dx=0, x=0), -3), (dict(dw=0, w=0), -3),
    (dict(dy=A[0] + 8), -5), (dict(x=A[1] + 8), -5), (dict(w=A[2] + 8), -5), (dict(dx=A[3] + 8), -5), (dict(dw=A[4] + 8), -5), (dict(ws=A[5] + 4), -5),
    (dict(n=0), -1), (dict(n=4), -1), (dict(dx=A[0]), -1), (dict(dx=A[1]), -1), (dict(dw=A[2]), -1), (dict(dw=A[1]), -1), (dict(dw=A[3]), -1),
    (dict(dx=A[5]), -1)])
def test_expert_linear_backward_refuses(kw, code):
    assert grads(cfg(), **kw) == code


def test_expert_linear_backward_sizes():
    assert grads(cfg(), n=(1 << 20) + 8) == -2
    assert grads(cfg(hidden=(1 << 20) + 8)) == -2
    assert grads(cfg(tokens=2 ** 31 - 4096, hidden=16, top_k=1, slices=1), n=8) == -2


CALLS = {
    "monta_rmsnorm": (["x", "residual", "weight", "sum", "out", "out_fp8"], dict(eps=1e-5)),
    "monta_rmsnorm_backward": (["sum", "weight", "dout", "dsum", "dx", "dweight", "scratch"], dict(eps=1e-5)),
    "monta_combine_backward": (["dout", "y", "gates", "dy", "dgates", "ws"], {}),
    "monta_expert_linear_fp8": (["x_rows", "w_codes", "w_scales", "y", "ws"], dict(out_features=16)),
    "monta_expert_linear_backward": (["dy", "x_final", "w_exp", "dx_final", "dw_exp", "ws"], dict(out_features=16)),
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
        bufs[bad] = 3
        with pytest.raises(m.MontaError, match=f"^{name}: ") as e:
            getattr(m, name)(c, **bufs, **kw, stream=0)
        assert e.value.code in (-5, -1)
    bufs = {n: A[i] for i, n in enumerate(names)}
    bufs[names[0]] = None
    with pytest.raises(m.MontaError, match=f"^{name}: ") as e:
        getattr(m, name)(c, **bufs, **kw, stream=0)
    assert e.value.code == -3
    bad_cfg = cfg(top_k=5)
    with pytest.raises(m.MontaError) as e:
        getattr(m, name)(bad_cfg, **{n: A[i] for i, n in enumerate(names)}, **kw, stream=0)
    assert e.value.code == -1
