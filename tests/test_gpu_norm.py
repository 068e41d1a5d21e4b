"""occ_norm_gate and occ_norm_gate_bwd against plain 64-bit implementations.

Tolerances.  Forward: a row's sums of squares are trees and chains of at most a few
hundred additions whose terms are positive, so r1 and r2 are good to 2^-17 and each
product adds 2^-24: 2^-16 of the magnitudes an output is made of.  Backward: the same
with dot products, 2^-16 of the sums of magnitudes; sums over rows have
chains of under 200 additions (2^-16 of the magnitudes again).  bf16 outputs add one
rounding, 2^-8."""
import numpy as np
import pytest
import torch

import block_reference as ref
from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS, ALPHA = 1e-5, 0.75


def rand(shape, dtype, seed, scale=1.0, ld=None):
    """Normal values on the GPU, rows `ld` apart (NaN between them)."""
    g = torch.Generator().manual_seed(seed)
    t = (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype).to(DEV)
    if ld is None:
        return t
    wide = torch.full((shape[0], ld), float("nan"), dtype=dtype, device=DEV)
    wide[:, :shape[1]] = t
    return wide[:, :shape[1]]


def blank(shape, dtype, ld=None):
    wide = torch.full((shape[0], ld or shape[1]), 77.0, dtype=dtype, device=DEV)
    return wide[:, :shape[1]], wide


def close(name, got, want, mag):
    got = ref.f64(got)
    tol = 2.0 ** -16 * mag + 1e-30
    if name in ("y16", "h16", "df16", "dx16"):
        tol = tol + 2.0 ** -8 * np.abs(want)
    err = np.abs(got - want)
    assert (err <= tol).all(), (name, float(err.max()), np.argwhere(~(err <= tol))[:4].tolist())


def problem(rows, D, act, res, groups, seed=0, ld=None):
    p = dict(f=rand((rows, D), act, seed, 2.0, ld), x=rand((rows, D), res, seed + 1, 1.0, ld),
             w_post=rand((D,), act, seed + 2), w_pre=rand((D,), act, seed + 3),
             gate=None if groups == 0 else rand((groups, D), act, seed + 4))
    return p


def host(t):
    return None if t is None else ref.f64(t)


def check_forward(p, act, res, y, h, rstd, post=True):
    f, x, w1, w2, gate = (host(p[k]) for k in ("f", "x", "w_post", "w_pre", "gate"))
    wy, wh, wr = ref.norm_gate(f, x, w1, w2, gate, ALPHA, EPS, post)
    D = f.shape[1]
    n = wy - ALPHA * x
    y_mag = np.abs(ALPHA * x) + np.abs(n)
    close("y16" if res == BF16 else "y", y, wy, y_mag)
    if h is not None:
        w = np.ones(D) if w2 is None else np.abs(w2)
        close("h16" if act == BF16 else "h", h, wh, 2 * (y_mag * wr[:, 1:] * w + np.abs(wh)))
    if rstd is not None:
        if h is None:
            wr[:, 1] = 1
        close("rstd", rstd, wr, np.abs(wr))


TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]
# one column to the widest row: a wave a row, then 4 and 16 waves, with few rows and many; ragged ends
SHAPES = [(1, 1), (3, 7), (5, 512), (600, 40), (300, 520), (7, 1000), (400, 2047), (2, 4099), (300, 4096), (3, 8192),
          (300, 5003), (2, 16384), (290, 8200), (257, 16383)]


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("rows,D", SHAPES)
def test_forward(rows, D, act, res):
    groups = {0: 0, 1: 1, 2: rows}[(rows + D) % 3]
    p = problem(rows, D, act, res, groups, seed=rows + D)
    (y, _), (h, _) = blank((rows, D), res), blank((rows, D), act)
    rstd = torch.empty((rows, 2), device=DEV)
    occ.occ_norm_gate(p["f"], p["x"], y, h, w_post=p["w_post"], w_pre=p["w_pre"], gate=p["gate"], alpha=ALPHA, eps=EPS,
                      rstd=rstd)
    check_forward(p, act, res, y, h, rstd)


@pytest.mark.parametrize("act,res", TYPES)
def test_forward_options(act, res):
    """No weights, no gate, no norm after, no norm before; groups of rows; strided rows and what lies between them."""
    rows, D, ld = 12, 701, 733
    p = problem(rows, D, act, res, 3, ld=ld)
    for post in (True, False):
        for keep in ((), ("w_pre",), ("gate",), ("w_post", "w_pre", "gate")):
            q = {k: v if k in ("f", "x") or (k in keep and (post or k != "w_post")) else None for k, v in p.items()}
            for with_h in (True, False):
                (y, yw), (h, hw) = blank((rows, D), res, ld), blank((rows, D), act, ld)
                rstd = torch.empty((rows, 2), device=DEV)
                occ.occ_norm_gate(q["f"], q["x"], y, h if with_h else None, w_post=q["w_post"], w_pre=q["w_pre"],
                                  gate=q["gate"], alpha=ALPHA, eps=EPS, post=post, rstd=rstd)
                check_forward(q, act, res, y, h if with_h else None, rstd, post)
                assert (yw[:, D:] == 77).all() and (hw[:, D:] == 77).all() and (with_h or (h == 77).all())


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("rows,D", [(1, 5), (700, 333), (300, 8190), (40, 16381)])
def test_forward_in_place(rows, D, act, res):
    """y over x and h over f: the same bits as in buffers of their own."""
    p = problem(rows, D, act, res, 1, seed=D)
    args = dict(w_post=p["w_post"], w_pre=p["w_pre"], gate=p["gate"], alpha=ALPHA, eps=EPS)
    (y, _), (h, _) = blank((rows, D), res), blank((rows, D), act)
    occ.occ_norm_gate(p["f"], p["x"], y, h, **args)
    f, x = p["f"].clone(), p["x"].clone()
    occ.occ_norm_gate(f, x, x, f, **args)
    assert torch.equal(x, y) and torch.equal(f, h)


@pytest.mark.parametrize("D", [96, 3001, 9000])
def test_zero_and_nonfinite_rows_stay_their_own(D):
    p = problem(6, D, BF16, F32, 1, seed=5)
    p["f"][1] = 0
    p["x"][1] = 0
    p["f"][3, D - 1] = float("nan")
    p["x"][4, 0] = float("inf")
    y, h = torch.empty((6, D), device=DEV), torch.empty((6, D), dtype=BF16, device=DEV)
    occ.occ_norm_gate(p["f"], p["x"], y, h, w_post=p["w_post"], w_pre=p["w_pre"], gate=p["gate"], alpha=ALPHA, eps=EPS)
    assert (y[1] == 0).all() and (h[1] == 0).all()
    assert torch.isnan(y[3]).all() and torch.isnan(h[3]).all() and torch.isinf(y[4, 0])
    for r in (0, 2, 5):
        assert torch.isfinite(y[r]).all() and torch.isfinite(h[r]).all()


def backward(p, act, res, y, rstd, dy, dh, groups, post=True, skip=(), ld=None):
    rows, D = p["f"].shape
    out = {"df": blank((rows, D), act, ld)[0], "dx": blank((rows, D), res, ld)[0],
           "dw_post": torch.full((D,), 77.0, device=DEV), "dw_pre": torch.full((D,), 77.0, device=DEV),
           "dgate": torch.full((groups, D), 77.0, device=DEV) if groups else None}
    if not post:
        out["dw_post"] = None
    out = {k: None if k in skip else v for k, v in out.items()}
    ws = torch.full((occ.occ_norm_gate_bwd_workspace_bytes(rows, D, max(1, groups)),), 0xFF, dtype=torch.uint8, device=DEV)
    occ.occ_norm_gate_bwd(dy, dh, p["f"], y, rstd, out["df"], out["dx"], w_post=p["w_post"], w_pre=p["w_pre"],
                          gate=p["gate"], alpha=ALPHA, post=post, dw_post=out["dw_post"], dw_pre=out["dw_pre"],
                          dgate=out["dgate"], workspace=ws)
    return out


def check_backward(p, act, res, y, rstd, dy, dh, out, post=True):
    want, mag = ref.norm_gate_bwd(host(dy), host(dh), host(p["f"]), host(y), host(rstd), host(p["w_post"]),
                                  host(p["w_pre"]), host(p["gate"]), ALPHA, post)
    for k, t in out.items():
        if t is not None:
            name = k + "16" if (k == "df" and act == BF16) or (k == "dx" and res == BF16) else k
            close(name, t, want[k], mag[k])


def forward_state(p, act, res, post=True):
    rows, D = p["f"].shape
    y, h, rstd = torch.empty((rows, D), dtype=res, device=DEV), torch.empty((rows, D), dtype=act, device=DEV), \
        torch.empty((rows, 2), device=DEV)
    occ.occ_norm_gate(p["f"], p["x"], y, h, w_post=p["w_post"] if post else None, w_pre=p["w_pre"], gate=p["gate"],
                      alpha=ALPHA, eps=EPS, post=post, rstd=rstd)
    return y, rstd


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("rows,D", SHAPES)
def test_backward(rows, D, act, res):
    groups = {0: 0, 1: 1, 2: rows}[(rows + D) % 3]
    p = problem(rows, D, act, res, groups, seed=rows + D)
    y, rstd = forward_state(p, act, res)
    dy, dh = rand((rows, D), res, 11), rand((rows, D), act, 12)
    out = backward(p, act, res, y, rstd, dy, dh, groups)
    check_backward(p, act, res, y, rstd, dy, dh, out)
    again = backward(p, act, res, y, rstd, dy, dh, groups)
    for k, t in out.items():
        assert t is None or torch.equal(t, again[k]), k


# gates shared by one row to many: runs of whole gates, several runs a gate, and the edges between
@pytest.mark.parametrize("act,res", [(BF16, F32), (F32, F32)])
@pytest.mark.parametrize("rows,D,groups", [(24, 300, 8), (5000, 64, 2500), (9000, 48, 10), (9000, 48, 100), (1200, 4100, 3),
                                           (1200, 4100, 300), (1200, 4100, 600), (1040, 8200, 4), (1040, 8200, 520), (7, 9000, 7)])
def test_backward_groups(rows, D, groups, act, res):
    p = problem(rows, D, act, res, groups, seed=rows)
    y, rstd = forward_state(p, act, res)
    dy, dh = rand((rows, D), res, 21), rand((rows, D), act, 22)
    check_backward(p, act, res, y, rstd, dy, dh, backward(p, act, res, y, rstd, dy, dh, groups))


@pytest.mark.parametrize("act,res", TYPES)
@pytest.mark.parametrize("D", [333, 8300])
def test_backward_options(act, res, D):
    rows, ld = 12, D + 31
    base = problem(rows, D, act, res, 4, ld=ld)
    dy, dh = rand((rows, D), res, 31, ld=ld), rand((rows, D), act, 32, ld=ld)
    for post in (True, False):
        for groups in (0, 4):
            for weights in (True, False):
                p = dict(base, gate=base["gate"] if groups else None, w_post=base["w_post"] if weights and post else None,
                         w_pre=base["w_pre"] if weights else None)
                y, rstd = forward_state(p, act, res, post)
                for a, b, skip in ((dy, dh, ()), (None, dh, ("dw_pre",)), (dy, None, ("dgate", "dx")), (dy, dh, ("df", "dw_post"))):
                    out = backward(p, act, res, y, rstd, a, b, groups, post, skip, ld)
                    check_backward(p, act, res, y, rstd, a, b, out, post)


def test_backward_in_place_and_without_rows():
    p = problem(40, 500, BF16, F32, 1)
    y, rstd = forward_state(p, BF16, F32)
    dy, dh = rand((40, 500), F32, 41), rand((40, 500), BF16, 42)
    want = backward(p, BF16, F32, y, rstd, dy, dh, 1)
    ws = torch.empty(occ.occ_norm_gate_bwd_workspace_bytes(40, 500), dtype=torch.uint8, device=DEV)
    a, b = dy.clone(), dh.clone()
    occ.occ_norm_gate_bwd(a, b, p["f"], y, rstd, b, a, w_post=p["w_post"], w_pre=p["w_pre"], gate=p["gate"], alpha=ALPHA,
                          workspace=ws)
    assert torch.equal(a, want["dx"]) and torch.equal(b, want["df"])
    x, f = p["x"].clone(), p["f"].clone()
    y2, h2 = torch.empty_like(y), torch.empty_like(f)
    kw = dict(w_post=p["w_post"], w_pre=p["w_pre"], gate=p["gate"], alpha=ALPHA, eps=EPS)
    occ.occ_norm_gate(f, x, y2, h2, **kw)
    occ.occ_norm_gate(f, x, x, f, **kw)
    assert torch.equal(x, y2) and torch.equal(f, h2)
    for groups in (1, 3):
        e = problem(0, 60, F32, F32, groups)
        none = torch.empty((0, 60), device=DEV)
        assert occ.occ_norm_gate(none, none, none.clone())[0].numel() == 0
        out = {k: torch.full(s, 7.0, device=DEV) for k, s in (("dw_post", (60,)), ("dw_pre", (60,)), ("dgate", (groups, 60)))}
        occ.occ_norm_gate_bwd(none, None, none, none, torch.empty((0, 2), device=DEV), gate=e["gate"], **out)
        assert all((t == 0).all() for t in out.values())


def test_backward_against_differences():
    """<gradient, direction> against the central difference of the 64-bit loss <c, y> + <e, h>."""
    rows, D, groups = 6, 130, 3
    p = problem(rows, D, F32, F32, groups, seed=3)
    dy, dh = rand((rows, D), F32, 51), rand((rows, D), F32, 52)
    y, rstd = forward_state(p, F32, F32)
    out = backward(p, F32, F32, y, rstd, dy, dh, groups)
    at = {k: host(p[k]) for k in ("f", "x", "w_post", "w_pre", "gate")}
    c, e = host(dy), host(dh)

    def loss(q):
        yy, hh, _ = ref.norm_gate(q["f"], q["x"], q["w_post"], q["w_pre"], q["gate"], ALPHA, EPS)
        return (c * yy).sum() + (e * hh).sum()

    rng = np.random.default_rng(0)
    for k, g in (("f", "df"), ("x", "dx"), ("w_post", "dw_post"), ("w_pre", "dw_pre"), ("gate", "dgate")):
        v = rng.standard_normal(at[k].shape)
        step = 1e-5
        slope = (loss(dict(at, **{k: at[k] + step * v})) - loss(dict(at, **{k: at[k] - step * v}))) / (2 * step)
        got, scale = (host(out[g]) * v).sum(), np.abs(host(out[g]) * v).sum()
        # differences are good to step^2 and 2^-53 / step, the kernel to 2^-16 of its magnitudes
        assert abs(got - slope) <= 1e-4 * scale, (k, got, slope)


def test_refusals():
    p = problem(6, 40, BF16, F32, 1)
    y = torch.empty((6, 40), device=DEV)
    for kw in (dict(w_post=p["w_post"].float()), dict(gate=p["gate"][0]), dict(rstd=torch.empty((6, 1), device=DEV))):
        with pytest.raises(ValueError):
            occ.occ_norm_gate(p["f"], p["x"], y, **kw)
    with pytest.raises(ValueError):
        occ.occ_norm_gate(p["f"], p["x"], y.to(BF16))
    for kw in (dict(gate=rand((4, 40), BF16, 1)), dict(w_post=p["w_post"], post=False)):
        with pytest.raises(occ.OccError) as e:
            occ.occ_norm_gate(p["f"], p["x"], y, **kw)
        assert e.value.status == occ.OCC_EINVAL
    with pytest.raises(occ.OccError) as e:
        occ.occ_norm_gate_bwd(y, None, p["f"], y.clone(), torch.empty((6, 2), device=DEV), dx=torch.empty_like(y),
                              workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == occ.OCC_EINVAL


def test_forward_of_more_rows_than_one_grid_dimension():
    """2^26 + 3 rows of 2: a wave a row is past 2^32 work-items; every row's formula is checked on the GPU."""
    rows, D = 2 ** 26 + 3, 2
    base = torch.arange(rows, dtype=torch.int32, device=DEV)
    f = torch.stack((base % 7 - 3, base % 5 + 1), 1).to(BF16)
    x = torch.stack((base % 11 - 5, base % 3), 1).to(BF16)
    y = torch.full((rows, D), float("nan"), dtype=BF16, device=DEV)
    occ.occ_norm_gate(f, x, y, alpha=ALPHA, eps=EPS)
    for lo in range(0, rows, 2 ** 24):
        part = f[lo:lo + 2 ** 24].double()
        n = part / (part.square().mean(1, keepdim=True) + EPS).sqrt()
        ax = ALPHA * x[lo:lo + 2 ** 24].double()
        tol = 2.0 ** -16 * (ax.abs() + n.abs()) + 2.0 ** -8 * (ax + n).abs() + 1e-30
        assert ((y[lo:lo + 2 ** 24].double() - (ax + n)).abs() <= tol).all(), lo
