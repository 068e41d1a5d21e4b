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


def norm_args(**kw):
    a = occ.occ_norm_args()
    a.rows, a.D, a.act, a.res, a.post, a.groups, a.alpha, a.eps = 6, 40, 0, 1, 1, 1, 1.0, 1e-6
    for i, n in enumerate(("f", "x", "y", "h", "dy", "dh", "df", "dx", "rstd", "w_post", "w_pre", "gate", "dw_post", "dw_pre",
                           "dgate", "workspace")):
        setattr(a, n, 0x10000000 * (i + 1))
    for n in ("f", "x", "y", "h", "dy", "dh", "df", "dx"):
        setattr(a, "ld_" + n, 40)
    a.workspace_bytes = occ.occ_norm_gate_bwd_workspace_bytes(6, 40, 1)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


def test_norm_argument_errors(L):
    for f in (L.occ_norm_gate, L.occ_norm_gate_bwd):
        assert f(None, None) == EINVAL
        for bad in (dict(rows=-1), dict(D=0), dict(D=16385), dict(act=2), dict(act=1, res=0), dict(groups=0), dict(groups=4),
                    dict(groups=7), dict(f=None), dict(y=None), dict(ld_f=39), dict(ld_y=39), dict(y=0x30000002),
                    dict(f=0x10000001), dict(w_post=0xA0000001), dict(post=0)):
            assert f(norm_args(**bad), None) == EINVAL, bad
        expect_accepted(L, f, norm_args(), None)
        expect_accepted(L, f, norm_args(groups=6, f=0x10000002,
                                        workspace_bytes=occ.occ_norm_gate_bwd_workspace_bytes(6, 40, 6)), None)
    f = L.occ_norm_gate
    for bad in (dict(x=None), dict(ld_x=39), dict(ld_h=39), dict(h=0x40000001)):
        assert f(norm_args(**bad), None) == EINVAL, bad
    for bad in (dict(y=0x10000000), dict(y=0x20000004), dict(h=0x20000000), dict(h=0x10000002), dict(h=0x10000000, ld_h=41),
                dict(rstd=0x30000000), dict(h=0xA0000000)):
        assert f(norm_args(**bad), None) == EALIAS, bad
    expect_accepted(L, f, norm_args(y=0x20000000, h=0x10000000, rstd=None), None)      # in place
    f = L.occ_norm_gate_bwd
    for bad in (dict(dy=None, dh=None), dict(rstd=None), dict(ld_dy=39), dict(ld_df=39), dict(dx=0x80000002),
                dict(gate=None), dict(post=0, w_post=None), dict(workspace=None), dict(workspace_bytes=479),
                dict(workspace=0x100000008), dict(dw_pre=0xE0000002)):
        assert f(norm_args(**bad), None) == EINVAL, bad
    for bad in (dict(dx=0x30000000), dict(df=0x50000000), dict(dx=0x50000004), dict(dgate=0x10000000), dict(dw_pre=0xD0000000),
                dict(workspace=0x30000000)):
        assert f(norm_args(**bad), None) == EALIAS, bad
    expect_accepted(L, f, norm_args(dx=0x50000000, df=0x60000000, dw_post=None, dw_pre=None, dgate=None), None)
    assert L.occ_norm_gate_bwd_workspace_bytes(6, 0, 1) == 0 and L.occ_norm_gate_bwd_workspace_bytes(-1, 8, 1) == 0


def moe_args(**kw):
    a = occ.occ_moe_args()
    a.tokens, a.H, a.I, a.experts, a.top_k, a.weight_type, a.renorm = 4, 64, 32, 8, 2, 0, 1
    for i, n in enumerate(("x", "router", "w_gate", "w_up", "w_down", "s_gate", "s_up", "s_down", "mask", "y", "ids", "weights",
                           "workspace")):
        setattr(a, n, 0x10000000 * (i + 1))
    a.ld_x, a.ld_y = 64, 64
    a.workspace_bytes = occ.occ_moe_workspace_bytes(4, 64, 32, 8, 2)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


def test_moe_argument_errors(L):
    f = L.occ_moe
    assert f(None, None) == EINVAL
    for bad in (dict(tokens=-1), dict(tokens=65), dict(H=60), dict(H=0), dict(H=65544), dict(I=12), dict(experts=0), dict(experts=513),
                dict(top_k=0), dict(top_k=9), dict(weight_type=1), dict(x=None), dict(router=None), dict(y=None), dict(w_up=None),
                dict(x=0x10000008), dict(w_down=0x50000008), dict(ld_x=63), dict(ld_x=68), dict(ld_x=(1 << 23) + 8), dict(ld_y=63),
                dict(stride_gate=2040), dict(stride_up=2052), dict(workspace=None), dict(workspace_bytes=64),
                dict(workspace=0xD0000008), dict(weight_type=2, s_up=None), dict(weight_type=2, stride_up=4096),
                dict(weight_type=2, s_down=0x80000008), dict(ids=0xB0000002), dict(y=0xA0000001)):
        assert f(moe_args(**bad), None) == EINVAL, bad
    for bad in (dict(y=0x10000000), dict(ids=0x90000000), dict(weights=0xA0000000), dict(workspace=0x40000010)):
        assert f(moe_args(**bad), None) == EALIAS, bad
    expect_accepted(L, f, moe_args(mask=None, ids=None, weights=None), None)
    expect_accepted(L, f, moe_args(weight_type=2), None)
    assert L.occ_moe_workspace_bytes(65, 64, 32, 8, 2) == 0 and L.occ_moe_workspace_bytes(0, 64, 32, 8, 2) == 0
