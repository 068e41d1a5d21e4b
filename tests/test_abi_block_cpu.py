"""CPU checks of the block operators' C ABI: bad arguments are refused with the documented status before the GPU is
touched (placeholder pointers; calls that pass validation are made only where no device is visible)."""
import ctypes

import pytest
import torch

from paper_2606_09200_amd import binding as occ
from test_abi_cpu import P, expect_accepted

EINVAL, EALIAS = occ.OCC_EINVAL, occ.OCC_EALIAS
X, Q, S, QT, ST, C = (P(0x10000000 * i) for i in range(1, 7))


@pytest.fixture(scope="module")
def L():
    return occ.lib()


def test_quantize_argument_errors(L):
    f = L.occ_mx4_quantize
    assert f(X, 2, 4, 64, 64, Q, S, None, None, None) == EINVAL          # not a float type
    assert f(X, 0, -1, 64, 64, Q, S, None, None, None) == EINVAL
    assert f(X, 0, 4, (1 << 23) + 1, 1 << 24, Q, S, None, None, None) == EINVAL
    assert f(X, 0, 4, 64, 63, Q, S, None, None, None) == EINVAL          # rows would overlap
    assert f(None, 0, 4, 64, 64, Q, S, None, None, None) == EINVAL
    assert f(X, 0, 4, 64, 64, None, None, None, None, None) == EINVAL    # nothing asked for
    assert f(X, 0, 4, 64, 64, Q, None, None, None, None) == EINVAL       # half a pair
    assert f(X, 0, 4, 64, 64, Q, S, None, ST, None) == EINVAL
    assert f(P(0x10000001), 0, 4, 64, 64, Q, S, None, None, None) == EINVAL
    assert f(P(0x10000002), 1, 4, 64, 64, Q, S, None, None, None) == EINVAL
    assert f(X, 0, 4, 64, 64, P(0x20000008), S, None, None, None) == EINVAL
    assert f(X, 0, 4, 64, 64, P(0x10000010), S, None, None, None) == EALIAS
    assert f(X, 0, 4, 64, 64, Q, P(0x20000010), None, None, None) == EALIAS
    assert f(X, 0, 4, 64, 64, Q, S, Q, ST, None) == EALIAS
    assert f(X, 0, 1 << 23, 1 << 21, 1 << 21, Q, S, None, None, None) == EINVAL   # beyond a grid
    expect_accepted(L, f, P(0x10000002), 0, 4, 65, 65, Q, S, QT, ST, None)


def test_dequantize_argument_errors(L):
    f = L.occ_mx4_dequantize
    assert f(Q, S, 4, 64, C, 2, 64, None) == EINVAL
    assert f(Q, S, 4, 64, C, 0, 63, None) == EINVAL
    assert f(Q, None, 4, 64, C, 0, 64, None) == EINVAL
    assert f(Q, S, 4, 64, None, 0, 64, None) == EINVAL
    assert f(Q, S, 4, 64, P(0x20000000), 0, 64, None) == EALIAS
    expect_accepted(L, f, Q, S, 4, 65, C, 1, 70, None)


def test_gemm_mx4_argument_errors(L):
    f = L.occ_gemm_mx4
    assert f(X, S, Q, ST, C, 2, 4, 4, 64, 0, None) == EINVAL
    assert f(X, S, Q, ST, C, 0, 4, -1, 64, 0, None) == EINVAL
    assert f(X, S, Q, ST, C, 0, 4, 4, (1 << 23) + 1, 0, None) == EINVAL
    assert f(None, S, Q, ST, C, 0, 4, 4, 64, 0, None) == EINVAL
    assert f(X, S, Q, P(0x30000008), C, 0, 4, 4, 64, 0, None) == EINVAL
    assert f(X, S, Q, ST, P(0x60000002), 1, 4, 4, 64, 0, None) == EINVAL
    assert f(X, S, Q, ST, P(0x20000010), 0, 4, 4, 64, 0, None) == EALIAS
    assert f(X, S, Q, ST, C, 0, 1 << 23, 1 << 23, 64, 0, None) == EINVAL
    expect_accepted(L, f, X, S, Q, ST, P(0x60000002), 0, 4, 5, 65, 0, None)


def test_binding_refuses_wrong_tensors():
    q = occ.mx4_empty(20, 700, device="cpu")
    assert tuple(q.codes.shape) == (20, 512) and tuple(q.scales.shape) == (2, 512)
    with pytest.raises(ValueError):
        occ.Mx4(q.codes, q.scales, 20, 1025)
    with pytest.raises(ValueError):
        occ.Mx4(q.codes.float(), q.scales, 20, 700)
    with pytest.raises(ValueError):
        occ.occ_mx4_quantize(torch.zeros(20, 700), q)                      # not on the GPU
    b = occ.mx4_empty(16, 64, batch=3, device="cpu")
    assert tuple(b[1].codes.shape) == (16, 256)
    with pytest.raises(IndexError):
        q[0]
