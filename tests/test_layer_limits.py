"""Host-only: sizes whose tiles are more than one launch has workgroups for are refused before any HIP call.  A launch of 2^32
threads or more would run the low 32 bits' worth of them and report nothing."""
import ctypes

import pytest

import paper_2411_00662_amd as m
from paper_2411_00662_amd import binding as B

A = [(i + 1) << 50 for i in range(8)]                   # addresses far apart; never dereferenced: validation fails first


def cfg(tokens, hidden, dtype, experts=1):
    return ctypes.byref(m.make_cfg(tokens, hidden, dtype, experts, 1, 1, 1, 1))


@pytest.mark.parametrize("dtype,tokens,hidden,n", [
    (m.BF16, 2 ** 24, 256, 2 ** 16),                    # 2^16 x 2^8 tiles of 256 x 256 by 512 threads
    (m.BF16, 2 ** 23, 256, 2 ** 16),
    (m.FP32, 2 ** 24, 256, 2 ** 14),                    # 2^17 x 2^7 tiles of 128 x 128 by 256
    (m.BF16, 2 ** 30, 16, 8192),                        # more tiles than an int32 counts, too
])
def test_experts8(dtype, tokens, hidden, n):
    assert B.lib().monta_expert_linear_fp8(cfg(tokens, hidden, dtype), A[0], A[1], A[2], n, A[3], A[4], -1, 0) == -2


@pytest.mark.parametrize("dtype,tokens,hidden,n", [
    (m.BF16, 2 ** 24, 2 ** 16, 512),                    # dx: 2^16 x 2^8 tiles of 256 x 256
    (m.FP32, 2 ** 20, 2 ** 16, 64),                     # dx: 2^14 x 2^10 tiles of 64 x 64
    (m.BF16, 64, 2 ** 20, 2 ** 20),                     # dw: 2^12 x 2^12 tiles of 256 x 256
    (m.FP32, 64, 2 ** 18, 2 ** 18),                     # dw: 2^12 x 2^12 tiles of 64 x 64
])
@pytest.mark.parametrize("both", [0, 1])
def test_expert_gradients(dtype, tokens, hidden, n, both):
    lib, c = B.lib(), cfg(tokens, hidden, dtype)
    dx_is_large = tokens >= hidden
    args = dict(x=A[1], w=A[2], dx=A[3], dw=A[4]) if both else dict(x=0, w=A[2], dx=A[3], dw=0) if dx_is_large else dict(x=A[1], w=0, dx=0, dw=A[4])
    assert lib.monta_expert_linear_backward(c, A[0], args["x"], args["w"], n, args["dx"], args["dw"], A[5], 0) == -2


@pytest.mark.parametrize("dtype,tokens,hidden,experts", [
    (m.FP32, 2 ** 26, 4, 1),                            # a wave for each token
    (m.FP32, 2 ** 27, 4, 5),                            # 16 tokens by 512 threads
    (m.BF16, 2 ** 29, 8, 1),                            # 32 tokens by 256
    (m.BF16, 2 ** 30, 8, 40),                           # 128 tokens by 512
])
def test_gate(dtype, tokens, hidden, experts):
    assert B.lib().monta_gate(cfg(tokens, hidden, dtype, experts), A[0], A[1], A[2], 0) == -2


@pytest.mark.parametrize("dtype,tokens,hidden,n", [
    (m.BF16, 2 ** 24, 256, 2 ** 16),
    (m.FP32, 2 ** 22, 256, 2 ** 14),
    (m.FP32, 2 ** 20, 2 ** 20 + 4, 2 ** 18),
])
def test_experts(dtype, tokens, hidden, n):
    assert B.lib().monta_expert_linear(cfg(tokens, hidden, dtype), A[0], A[1], n, A[2], A[3], -1, 0) == -2


def test_route():
    """A workgroup, at least, for each unit: 2^24 units of one token."""
    c = ctypes.byref(m.make_cfg(2 ** 24, 8, m.BF16, 1, 1, 1, 1, 2 ** 24))
    assert B.lib().monta_route(c, A[0], A[1], A[2], A[3], 0) == -2
