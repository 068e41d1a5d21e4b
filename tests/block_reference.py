"""Plain 64-bit implementations of the operators of a block, for the tests.

Written from the definitions in include/occ.h, in numpy, sharing nothing with
the library."""
import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def f64(t):
    """A torch tensor as float64 on the host."""
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- MX4

def mx4_kp(cols):
    return (cols + 511) // 512 * 512


def mx4_scale_exponent(block):
    """e of a block's scale 2^e, or None where the block is not finite."""
    top = np.max(np.abs(block)) if len(block) else 0.0
    if not np.isfinite(top):
        return None
    return -127 if top == 0 else max(-127, min(127, math.frexp(top)[1] - 1 - 2))


def mx4_code(a):
    """Code (without sign) of a magnitude in units of the scale: nearest value, ties to the even code, at most 6."""
    d = np.abs(GRID - a)
    best = np.flatnonzero(d == d.min())
    return 7 if a >= 6 else int(best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])


def mx4_quantize(x):
    """(codes as (rows, cols) values 0 .. 15, scale bytes as (rows, ceil(cols / 32))) of a float64 matrix."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    codes = np.zeros((rows, cols), np.uint8)
    scales = np.zeros((rows, nb), np.uint8)
    for r in range(rows):
        for b in range(nb):
            blk = x[r, 32 * b:32 * b + 32]
            e = mx4_scale_exponent(blk)
            scales[r, b] = 255 if e is None else e + 127
            if e is not None:
                for i, v in enumerate(blk):
                    codes[r, 32 * b + i] = mx4_code(abs(v) * 2.0 ** -e) + (8 if np.signbit(v) else 0)
    return codes, scales


def mx4_values(codes, scales):
    """Values of codes (rows, cols) and scale bytes (rows, blocks)."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def mx4_unpack(code_bytes, scale_bytes, rows, cols):
    """(codes, scales, what the padding holds) of the library's layout."""
    kp = mx4_kp(cols)
    assert code_bytes.shape == (rows, kp // 2) and scale_bytes.shape == ((rows + 15) // 16, kp // 2)
    codes = np.empty((rows, kp), np.uint8)
    codes[:, 0::2], codes[:, 1::2] = code_bytes & 15, code_bytes >> 4
    rp, nb = (rows + 15) // 16 * 16, (cols + 31) // 32
    scales = np.empty((rp, kp // 32), np.uint8)
    for r in range(rp):
        for b in range(kp // 32):
            s, j, g = b // 16, b % 16 // 4, b % 4
            scales[r, b] = scale_bytes[r // 16, 256 * s + 4 * (16 * g + r % 16) + j]
    pads = [codes[:, cols:], scales[rows:], scales[:, nb:]]
    return codes[:, :cols], scales[:rows, :nb], pads


def mx4_pack(codes, scales):
    """The library's layout of codes (rows, cols) and scale bytes (rows, blocks)."""
    rows, cols = codes.shape
    kp = mx4_kp(cols)
    full = np.zeros((rows, kp), np.uint8)
    full[:, :cols] = codes
    out = np.zeros(((rows + 15) // 16, kp // 2), np.uint8)
    for r in range(rows):
        for b in range(scales.shape[1]):
            s, j, g = b // 16, b % 16 // 4, b % 4
            out[r // 16, 256 * s + 4 * (16 * g + r % 16) + j] = scales[r, b]
    return full[:, 0::2] | (full[:, 1::2] << 4), out


# ---------------------------------------------------------------- norms around a block

def gate_rows(gate, rows, D):
    """One gate row per row (ones without a gate)."""
    return np.ones((rows, D)) if gate is None else np.repeat(gate, rows // gate.shape[0], axis=0) if rows else np.ones((0, D))


def norm_gate(f, x, w_post, w_pre, gate, alpha, eps, post=True):
    """y, h, rstd (rows, 2) in 64 bits."""
    rows, D = f.shape
    one = np.ones(D)
    r1 = 1 / np.sqrt((f * f).mean(1) + eps) if post else np.ones(rows)
    n = f * r1[:, None] * (one if w_post is None else w_post)
    y = alpha * x + gate_rows(gate, rows, D) * n
    r2 = 1 / np.sqrt((y * y).mean(1) + eps)
    return y, y * r2[:, None] * (one if w_pre is None else w_pre), np.stack([r1, r2], 1)


def norm_gate_bwd(dy, dh, f, y, rstd, w_post, w_pre, gate, alpha, post=True):
    """Gradients and, for each, the sum of the magnitudes it is made of."""
    rows, D = f.shape
    w1, w2 = (np.ones(D) if w is None else w for w in (w_post, w_pre))
    g = gate_rows(gate, rows, D)
    r1, r2 = rstd[:, :1], rstd[:, 1:]
    dy, dh = (np.zeros((rows, D)) if t is None else t for t in (dy, dh))
    u, yn, fn = dh * w2, y * r2, f * r1
    mean = lambda t: t.mean(1, keepdims=True)
    d = dy + r2 * (u - yn * mean(u * yn))
    d_mag = abs(dy) + r2 * (abs(u) + abs(yn) * mean(abs(u * yn)))
    v, v_mag = d * g * w1, d_mag * abs(g * w1)
    out = {"dx": alpha * d, "df": r1 * (v - fn * mean(v * fn)) if post else v,
           "dw_post": (d * g * fn).sum(0), "dw_pre": (dh * yn).sum(0)}
    mag = {"dx": abs(alpha) * d_mag, "df": r1 * (v_mag + (abs(fn) * mean(v_mag * abs(fn)) if post else 0)),
           "dw_post": (d_mag * abs(g * fn)).sum(0), "dw_pre": abs(dh * yn).sum(0)}
    if gate is not None:
        k = gate.shape[0]
        out["dgate"] = (d * fn).reshape(k, -1, D).sum(1) * w1
        mag["dgate"] = (d_mag * abs(fn)).reshape(k, -1, D).sum(1) * abs(w1)
    return out, mag


# ---------------------------------------------------------------- expert layer

def route(logits, top_k, renorm, mask):
    """ids (-1 for masked tokens) and weights: the largest logits, a tie to the lower index, a NaN last."""
    T, E = logits.shape
    ids, w = np.full((T, top_k), -1), np.zeros((T, top_k))
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        l = logits[t]
        pick = sorted(range(E), key=lambda e: (-l[e] if l[e] == l[e] else np.inf, l[e] != l[e], e))[:top_k]
        with np.errstate(all="ignore"):
            p = np.exp(l - l[pick[0]])
            p = p / p.sum()
            ids[t], w[t] = pick, p[pick] / p[pick].sum() if renorm else p[pick]
    return ids, w


def moe(x, ids, w, gate, up, down):
    """y, and how far rounding may take it: the sums of magnitudes of its binary32 sums and of the
    hidden activations' bf16 rounding.  gate, up, down: lists of matrices."""
    T, H = x.shape
    y, tol = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for j, e in enumerate(ids[t]):
            if e < 0:
                continue
            g, u = gate[e] @ x[t], up[e] @ x[t]
            eg, eu = (H * 2.0 ** -23 * (abs(m[e]) @ abs(x[t])) for m in (gate, up))
            s = g / (1 + np.exp(-g))
            h = s * u
            # |silu'| < 1.1; a few roundings of the epilogue; one to bf16
            eh = 1.1 * abs(u) * eg + abs(s) * eu + (2.0 ** -8 + 2.0 ** -20) * abs(h)
            y[t] += w[t, j] * (down[e] @ h)
            tol[t] += w[t, j] * (abs(down[e]) @ (eh + (len(h) * 2.0 ** -23 + 2.0 ** -16) * abs(h)))
    return y, tol + 2.0 ** -8 * abs(y)
