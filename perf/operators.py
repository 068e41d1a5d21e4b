"""The block operators this library is measured on: what sits between the GEMMs of an overlapped step.

``mx4``: microscaled 4-bit floating point (blocks of 32 E2M1 values with an E8M0
scale): quantisation, and a linear layer's products forward and backward.
``moe``: a whole mixture-of-experts layer for a few tokens.  ``norm``: the norms
after and before a block fused with its gate and the residual's scale, forward
and backward.

``listed`` names fixed cases, ``draw`` gives others of the same ranges;
``prepare`` makes what a program holds before the call, ``run`` is one pass: in
elementary torch operations in 32 bits where ``own`` is false, through the
library's entry points where it is true.  ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6
BF16, F32 = torch.bfloat16, torch.float32
DTYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # a decode step's activations on their way into a 4-bit product: launch and latency
        dict(name="quant_decode", op="quant", rows=16, cols=8192, dtype="bf16", both=False),
        # a training step's activations, row blocks for the forward product and column blocks for the weight gradient
        dict(name="quant_train", op="quant", rows=8192, cols=8192, dtype="bf16", both=True),
        # a decode step of 16 sequences through a linear layer with a 4-bit weight (read once)
        dict(name="linear_decode", op="linear", M=16, N=28672, K=8192),
        # the compute-bound layer of the overlap measurements with 4-bit operands
        dict(name="linear_8k", op="linear", M=8192, N=8192, K=8192),
        # the backward of a linear layer on a ragged number of tokens: dX and dW from dY in both orientations
        dict(name="linear_bwd", op="linear_bwd", M=3001, N=5003, K=2504),
        # one token through an expert layer with 4-bit weights
        dict(name="moe_one", op="moe", T=1, H=4096, I=2048, E=64, k=8, weights="mx4", renorm=True, masked=False),
        # a ragged decode batch with empty slots through an expert layer of odd sizes, weights not renormalised
        dict(name="moe_ragged", op="moe", T=37, H=2504, I=1400, E=60, k=4, weights="bf16", renorm=False, masked=True),
        # a decode batch that reaches most of the experts
        dict(name="moe_batch", op="moe", T=64, H=4096, I=2048, E=32, k=4, weights="bf16", renorm=True, masked=False),
        # a decode step's residual update between two blocks: launch and latency
        dict(name="norm_decode", op="norm", rows=16, D=8192, act="bf16", res="bf16", gate="channel", groups=1),
        # a long batch of sequences, each with its own gate, on a 32-bit residual of odd width
        dict(name="norm_ragged", op="norm", rows=12004, D=5003, act="bf16", res="f32", gate="group", groups=4),
        # the backward of the residual update of a training step
        dict(name="norm_bwd", op="norm_bwd", rows=8192, D=8192, act="bf16", res="bf16", gate="channel", groups=1),
        # the same with a gate for each token of a small step
        dict(name="norm_bwd_token", op="norm_bwd", rows=512, D=4096, act="bf16", res="f32", gate="token", groups=512),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, mult=1):
    """A size of [lo, hi] spread over its logarithm: half of them round, half any multiple of `mult`."""
    x = _log(rng, lo, hi)
    step = max(mult, 128) if x >= 256 and rng.random() < 0.5 else mult
    return _other(max(lo, min(hi, (x + step // 2) // step * step)))


def _other(x):
    return x + 128 if x == 3072 else x  # 3072 is no size of this repository


def draw(rng):
    op = rng.choice(("quant", "linear", "linear", "linear_bwd", "moe", "moe", "norm", "norm_bwd"))
    if op == "quant":
        cols, dtype = _size(rng, 40, 16384), rng.choice(("bf16", "bf16", "f32"))
        return dict(op=op, rows=_size(rng, 1, min(16384, (1 << (26 if dtype == "bf16" else 25)) // cols)), cols=cols,
                    dtype=dtype, both=rng.random() < 0.5)
    if op == "linear":
        M = rng.choice((rng.randint(1, 16), _size(rng, 17, 512), _size(rng, 512, 8192)))
        return dict(op=op, M=M, N=_size(rng, 256, 28672 if M <= 512 else 8192), K=_size(rng, 256, 8192))
    if op == "linear_bwd":
        return dict(op=op, M=_size(rng, 64, 4096), N=_size(rng, 256, 8192), K=_size(rng, 256, 8192))
    if op == "moe":
        E = rng.choice((4, 8, 16, 32, 60, 64, 128))
        H, I = _size(rng, 512, 8192, 8), _size(rng, 256, 8192, 8)
        I = _other(max(256, min(I, (1 << 28) // (E * H) // 8 * 8)))
        T = rng.choice((1, rng.randint(2, 16), rng.randint(17, 64)))
        return dict(op=op, T=T, H=H, I=I, E=E, k=rng.randint(1, min(8, E)), weights=rng.choice(("bf16", "mx4")),
                    renorm=rng.random() < 0.5, masked=T > 1 and rng.random() < 0.3)
    act, res = rng.choice((("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")))
    D = _size(rng, 256, 16384)
    rows = _size(rng, 1, min(32768, (1 << (26 if res == "bf16" else 25)) // D))
    gate = rng.choice(("none", "channel", "group", "token"))
    groups = {"none": 1, "channel": 1, "token": rows}.get(gate)
    if groups is None:
        groups = rng.randint(1, 8)
        rows = max(1, rows // groups) * groups
    return dict(op=op, rows=rows, D=D, act=act, res=res, gate=gate, groups=groups)


# ------------------------------------------------------------------ the 4-bit format
#
# rows x cols in blocks of 32 along a row.  Codes: two per byte (the even
# column in the low nibble), rows padded with zeros to a multiple of 512 columns
# (Kp).  Scales: tiles of 16 rows x 512 columns, 256 bytes each; the scale of
# row 16 t + r and block b = (4 s + j) * 4 + g is byte j of word 16 g + r of
# tile (t, s).

def _kp(cols):
    return -(-cols // 512) * 512


def _pow2(e):
    """2^e in 32 bits, e in [-127, 127], from its bits."""
    e = e.int()
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).view(F32)


def _round_e2m1(a):
    """|values| below 8 to the E2M1 grid, ties to even, saturated at 6."""
    r = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2))
    return torch.clamp(r, max=6.0)


def _quantize(x):
    """(codes, scales) of a 2-D tensor in the layout above, by elementary operations."""
    rows, cols = x.shape
    kp, rp = _kp(cols), -(-rows // 16) * 16
    b = torch.zeros((rp, kp), device=x.device, dtype=F32)
    b[:rows, :cols] = x
    b = b.view(rp, kp // 32, 32)
    e = torch.clamp(torch.frexp(b.abs().amax(-1)).exponent - 3, -127, 127)
    e = torch.where(b.abs().amax(-1) > 0, e, torch.full_like(e, -127))
    v = b * _pow2(-e)[..., None]
    r = _round_e2m1(v.abs())
    code = torch.where(r < 2, r * 2, torch.where(r < 4, r + 2, r / 2 + 4)).to(torch.uint8)
    code = (code + 8 * torch.signbit(v).to(torch.uint8)).view(rp, kp)[:rows]
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    s = (e + 127).to(torch.uint8)
    scales = s.view(rp // 16, 16, kp // 512, 4, 4).permute(0, 2, 4, 1, 3).contiguous()
    return codes.contiguous(), scales.view(rp // 16, kp // 2)


_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _dequantize(codes, scales, cols):
    """The values codes and scales stand for, 32 bits."""
    rows, kp = codes.shape[0], codes.shape[1] * 2
    grid = torch.tensor(_GRID + tuple(-v for v in _GRID), device=codes.device)
    v = torch.stack((grid[(codes & 15).long()], grid[(codes >> 4).long()]), -1).view(rows, kp // 32, 32)
    s = scales.view(-1, kp // 512, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(-1, kp // 32)[:rows]
    return (v * _pow2(s.int() - 127)[..., None]).view(rows, kp)[:, :cols]


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=F32)


def _activations(g, rows, cols):
    """Normal values with a few channels an order of magnitude larger, as a block's activations have them."""
    x = _randn(g, rows, cols)
    x *= torch.exp(0.5 * _randn(g, 1, cols))
    return x


def _mx4_weight(g, rows, cols, std):
    """A weight as a program keeps it: laid out once, from its bf16 values."""
    return _mx4(*_quantize((_randn(g, rows, cols) * std).to(BF16)), rows, cols)


def _mx4(codes, scales, rows, cols):
    if own:
        from paper_2606_09200_amd import binding as occ
        return occ.Mx4(codes, scales, rows, cols)
    return codes, scales, cols


def _parts(q):
    """(codes, scales, cols) of a kept 4-bit tensor."""
    return q if isinstance(q, tuple) else (q.codes, q.scales, q.cols)


def _empty_mx4(rows, cols):
    from paper_2606_09200_amd import binding as occ
    return occ.mx4_empty(rows, cols, device=DEV)


def _prepare_quant(c, s, g):
    s["x"] = _activations(g, c["rows"], c["cols"]).to(DTYPES[c["dtype"]])
    if own:
        s["q"] = _empty_mx4(c["rows"], c["cols"])
        s["qt"] = _empty_mx4(c["cols"], c["rows"]) if c["both"] else None
        s["v"] = torch.empty((c["rows"], c["cols"]), device=DEV, dtype=BF16)
        s["vt"] = torch.empty((c["cols"], c["rows"]), device=DEV, dtype=BF16) if c["both"] else None


def _prepare_linear(c, s, g):
    M, N, K = c["M"], c["N"], c["K"]
    std = K ** -0.5
    if c["op"] == "linear":
        s["x"] = _activations(g, M, K).to(BF16)
        s["W"] = _mx4_weight(g, N, K, std)
        if own:
            s["xq"] = _empty_mx4(M, K)
            s["y"] = torch.empty((M, N), device=DEV, dtype=BF16)
        return
    # the forward pass left x in column blocks; the weight is kept in column blocks too
    s["dy"] = _activations(g, M, N).mul_(1e-3).to(BF16)
    s["Wt"] = _mx4_weight(g, K, N, std)
    s["xt"] = _mx4(*_quantize(_activations(g, M, K).to(BF16).t()), K, M)
    if own:
        s["dyq"], s["dyt"] = _empty_mx4(M, N), _empty_mx4(N, M)
        s["dx"] = torch.empty((M, K), device=DEV, dtype=BF16)
        s["dw"] = torch.empty((N, K), device=DEV, dtype=F32)


def _prepare_moe(c, s, g):
    T, H, I, E, k = (c[n] for n in ("T", "H", "I", "E", "k"))
    s["router"] = (_randn(g, E, H) * (1.5 * H ** -0.5)).to(BF16)
    x = _randn(g, T, H).to(BF16)
    if k < E:
        # a token whose k-th and next logit all but tie is drawn again: the order of a
        # sum in 32 bits would decide which expert it goes to
        for _ in range(4):
            top = torch.topk(x.double() @ s["router"].double().t(), k + 1, dim=1).values
            close = (top[:, k - 1] - top[:, k]) < 2e-5
            x = torch.where(close[:, None], _randn(g, T, H).to(BF16), x)
    s["x"] = x
    s["mask"] = torch.rand(T, generator=g, device=DEV) < 0.75 if c["masked"] else None
    for name, rows, cols in (("gate", I, H), ("up", I, H), ("down", H, I)):
        if c["weights"] == "bf16":
            w = torch.empty((E, rows, cols), device=DEV, dtype=BF16)
            for e in range(E):
                w[e] = _randn(g, rows, cols) * cols ** -0.5
            s[name] = w
        else:
            parts = [_quantize((_randn(g, rows, cols) * cols ** -0.5).to(BF16)) for _ in range(E)]
            s[name] = _mx4(torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts]), rows, cols)
    if own:
        from paper_2606_09200_amd import binding as occ
        s["workspace"] = torch.zeros(occ.occ_moe_workspace_bytes(T, H, I, E, k), dtype=torch.uint8, device=DEV)
        s["y"] = torch.empty((T, H), device=DEV, dtype=BF16)
        s["ids"] = torch.empty((T, k), device=DEV, dtype=torch.int32)
        s["w"] = torch.empty((T, k), device=DEV, dtype=F32)


def _prepare_norm(c, s, g):
    rows, D = c["rows"], c["D"]
    act, res = DTYPES[c["act"]], DTYPES[c["res"]]
    s["alpha"] = 0.75
    s["f"] = (_activations(g, rows, D) * 0.5).to(act)
    s["x"] = _activations(g, rows, D).mul_(2.0).to(res)
    s["w_post"] = (1.0 + 0.2 * _randn(g, D)).to(act)
    s["w_pre"] = (1.0 + 0.2 * _randn(g, D)).to(act)
    s["gate"] = None if c["gate"] == "none" else (0.5 + 0.3 * _randn(g, c["groups"], D)).to(act)
    like = dict(device=DEV)
    if c["op"] == "norm":
        if own:
            s["y"] = torch.empty((rows, D), dtype=res, **like)
            s["h"] = torch.empty((rows, D), dtype=act, **like)
            s["rstd"] = torch.empty((rows, 2), dtype=F32, **like)
        return
    s["y"], _, s["rstd"] = _norm_plain(s)   # what the forward pass left
    s["dy"] = _activations(g, rows, D).mul_(1e-2).to(res)
    s["dh"] = _activations(g, rows, D).mul_(1e-2).to(act)
    del s["x"]
    if own:
        from paper_2606_09200_amd import binding as occ
        s["df"] = torch.empty((rows, D), dtype=act, **like)
        s["dx"] = torch.empty((rows, D), dtype=res, **like)
        s["dw_post"], s["dw_pre"] = torch.empty(D, **like), torch.empty(D, **like)
        s["dgate"] = None if s["gate"] is None else torch.empty((c["groups"], D), **like)
        s["workspace"] = torch.empty(occ.occ_norm_gate_bwd_workspace_bytes(rows, D, c["groups"]), dtype=torch.uint8,
                                     **like)


def prepare(case, seed):
    s = dict(case)
    op = case["op"]
    g = _gen(seed)
    if op == "quant":
        _prepare_quant(case, s, g)
    elif op in ("linear", "linear_bwd"):
        _prepare_linear(case, s, g)
    elif op == "moe":
        _prepare_moe(case, s, g)
    else:
        _prepare_norm(case, s, g)
    return s


# ------------------------------------------------------------------ one pass

def _run_plain(s):
    op = s["op"]
    if op == "quant":
        q = _quantize(s["x"])
        out = {"v": _dequantize(*q, s["cols"]).to(BF16)}
        if s["both"]:
            q = _quantize(s["x"].t())
            out["vt"] = _dequantize(*q, s["rows"]).to(BF16)
        return out
    if op == "linear":
        x = _dequantize(*_quantize(s["x"]), s["K"])
        return (x @ _dequantize(*_parts(s["W"])).t()).to(BF16)
    if op == "linear_bwd":
        dy = _dequantize(*_quantize(s["dy"]), s["N"])
        dx = (dy @ _dequantize(*_parts(s["Wt"])).t()).to(BF16)
        dyt = _dequantize(*_quantize(s["dy"].t()), s["M"])
        return {"dx": dx, "dw": dyt @ _dequantize(*_parts(s["xt"])).t()}
    if op == "moe":
        return _moe_plain(s)
    if op == "norm":
        y, h, rstd = _norm_plain(s)
        return {"y": y, "h": h, "rstd": rstd}
    return _norm_bwd_plain(s)


def _expert(q, e):
    """Expert e's matrix in 32 bits."""
    if isinstance(q, torch.Tensor):
        return q[e].float()
    codes, scales, cols = _parts(q)
    return _dequantize(codes[e], scales[e], cols)


def _moe_plain(s):
    x = s["x"].float()
    logits = x @ s["router"].float().t()
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    order = torch.sort(p, dim=1, descending=True, stable=True)  # ties to the lowest index
    w, ids = order.values[:, :s["k"]], order.indices[:, :s["k"]]
    if s["renorm"]:
        w = w / w.sum(1, keepdim=True)
    if s["mask"] is not None:
        live = s["mask"][:, None]
        w, ids = torch.where(live, w, torch.zeros_like(w)), torch.where(live, ids, torch.full_like(ids, -1))
    y = torch.zeros_like(x)
    for e in range(s["E"]):
        at = ids == e
        a = x @ _expert(s["gate"], e).t()
        a = a / (1 + torch.exp(-a)) * (x @ _expert(s["up"], e).t())
        out = a @ _expert(s["down"], e).t()
        y = y + torch.where(at.any(1)[:, None], (w * at).sum(1)[:, None] * out, torch.zeros_like(out))
    return {"y": y.to(BF16), "ids": ids.to(torch.int32), "w": w}


def _gate_rows(s, t):
    """A tensor of one row per group as one row per token."""
    return t.repeat_interleave(s["rows"] // s["groups"], 0) if s["groups"] > 1 else t


def _norm_plain(s):
    f, x = s["f"].float(), s["x"].float()
    r1 = torch.rsqrt((f * f).mean(1, keepdim=True) + EPS)
    n = f * r1 * s["w_post"].float()
    if s["gate"] is not None:
        n = n * _gate_rows(s, s["gate"].float())
    y = s["alpha"] * x + n
    r2 = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    h = y * r2 * s["w_pre"].float()
    return y.to(s["x"].dtype), h.to(s["f"].dtype), torch.cat((r1, r2), 1)


def _norm_bwd_plain(s):
    f, y, dy, dh = (s[n].float() for n in ("f", "y", "dy", "dh"))
    w1, w2 = s["w_post"].float(), s["w_pre"].float()
    r1, r2 = s["rstd"][:, :1], s["rstd"][:, 1:]
    u = dh * w2
    d = dy + r2 * u - y * r2 ** 3 * (u * y).mean(1, keepdim=True)
    g = torch.ones(1, s["D"], device=DEV) if s["gate"] is None else _gate_rows(s, s["gate"].float())
    dn = d * g
    v = dn * w1
    df = r1 * v - f * r1 ** 3 * (v * f).mean(1, keepdim=True)
    out = {"df": df.to(s["f"].dtype), "dx": (s["alpha"] * d).to(s["y"].dtype),
           "dw_post": (dn * f * r1).sum(0), "dw_pre": (dh * y * r2).sum(0)}
    if s["gate"] is not None:
        out["dgate"] = (d * f * r1 * w1).view(s["groups"], -1, s["D"]).sum(1)
    return out


def _run_own(s):
    from paper_2606_09200_amd import binding as occ
    op = s["op"]
    if op == "quant":
        occ.occ_mx4_quantize(s["x"], s["q"], s["qt"])
        out = {"v": occ.occ_mx4_dequantize(s["q"], s["v"])}
        if s["both"]:
            out["vt"] = occ.occ_mx4_dequantize(s["qt"], s["vt"])
        return out
    if op == "linear":
        occ.occ_mx4_quantize(s["x"], s["xq"])
        return occ.occ_gemm_mx4(s["xq"], s["W"], s["y"])
    if op == "linear_bwd":
        occ.occ_mx4_quantize(s["dy"], s["dyq"], s["dyt"])
        return {"dx": occ.occ_gemm_mx4(s["dyq"], s["Wt"], s["dx"]),
                "dw": occ.occ_gemm_mx4(s["dyt"], s["xt"], s["dw"])}
    if op == "moe":
        occ.occ_moe(s["x"], s["router"], s["gate"], s["up"], s["down"], s["y"], top_k=s["k"], ids=s["ids"],
                    weights=s["w"], workspace=s["workspace"], renorm=s["renorm"], mask=s["mask"])
        return {"y": s["y"], "ids": s["ids"], "w": s["w"]}
    if op == "norm":
        occ.occ_norm_gate(s["f"], s["x"], s["y"], s["h"], w_post=s["w_post"], w_pre=s["w_pre"], gate=s["gate"],
                          alpha=s["alpha"], eps=EPS, rstd=s["rstd"])
        return {"y": s["y"], "h": s["h"], "rstd": s["rstd"]}
    occ.occ_norm_gate_bwd(s["dy"], s["dh"], s["f"], s["y"], s["rstd"], s["df"], s["dx"], w_post=s["w_post"],
                          w_pre=s["w_pre"], gate=s["gate"], alpha=s["alpha"], dw_post=s["dw_post"],
                          dw_pre=s["dw_pre"], dgate=s["dgate"], workspace=s["workspace"])
    out = {"df": s["df"], "dx": s["dx"], "dw_post": s["dw_post"], "dw_pre": s["dw_pre"]}
    if s["gate"] is not None:
        out["dgate"] = s["dgate"]
    return out


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------ what a pass cannot do without

def _q_bytes(rows, cols):
    return rows * cols * 17.0 / 32.0


def work(case):
    op = case["op"]
    size = {"bf16": 2.0, "f32": 4.0}
    if op == "quant":
        n, o = case["rows"] * case["cols"], 2 if case["both"] else 1
        # x in; codes, scales and the values they stand for out, for each orientation
        return {"bytes": n * size[case["dtype"]] + o * (_q_bytes(case["rows"], case["cols"]) + 2.0 * n), "flops": 4.0 * n * o}
    if op in ("linear", "linear_bwd"):
        M, N, K = case["M"], case["N"], case["K"]
        if op == "linear":
            return {"bytes": 2.0 * M * K + _q_bytes(N, K) + 2.0 * M * N, "flops": 2.0 * M * N * K}
        return {"bytes": 2.0 * M * N + _q_bytes(K, N) + _q_bytes(K, M) + 2.0 * M * K + 4.0 * N * K, "flops": 4.0 * M * N * K}
    if op == "moe":
        T, H, I, E, k = (case[n] for n in ("T", "H", "I", "E", "k"))
        live = T * 0.75 if case["masked"] else T
        reached = E * (1.0 - (1.0 - k / E) ** live)  # distinct experts that `live` tokens pick, on average
        w = 2.0 if case["weights"] == "bf16" else 17.0 / 32.0
        return {"bytes": 2.0 * E * H + reached * 3 * H * I * w + 4.0 * T * H + 8.0 * T * k,
                "flops": 2.0 * T * E * H + 6.0 * live * k * H * I}
    n = float(case["rows"]) * case["D"]
    a, r = size[case["act"]], size[case["res"]]
    gates = 0.0 if case["gate"] == "none" else float(case["groups"]) * case["D"]
    if op == "norm":
        return {"bytes": n * (2 * a + 2 * r) + (gates + 2 * case["D"]) * a + 8.0 * case["rows"], "flops": 10.0 * n}
    return {"bytes": n * (3 * a + 3 * r) + gates * (a + 4.0) + 2 * case["D"] * (a + 4.0) + 8.0 * case["rows"], "flops": 25.0 * n}


# ------------------------------------------------------------------ the definitions in 64 bits

_EDGES = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def _exact_quantized(x):
    """The values of x's row blocks: the block's power of two, then the nearest grid value, a tie to the even code."""
    rows, cols = x.shape
    x = x.double()
    out = torch.zeros_like(x)
    grid = torch.tensor(_GRID, device=x.device, dtype=torch.float64)
    for at in range(0, cols, 8192):   # whole blocks at a time
        b = x[:, at:at + 8192]
        n = b.shape[1]
        b = torch.nn.functional.pad(b, (0, -n % 32)).view(rows, -1, 32)
        top = b.abs().amax(-1, keepdim=True)
        unit = torch.exp2(torch.clamp(torch.floor(torch.log2(top)), -125, 129) - 2)
        a = (b / unit).abs()
        code = torch.zeros_like(a, dtype=torch.long)
        for edge, even_above in _EDGES:
            code += (a >= edge) if even_above else (a > edge)
        v = torch.where(top > 0, torch.copysign(grid[code] * unit, b), torch.zeros_like(b))
        out[:, at:at + n] = v.reshape(rows, -1)[:, :n]
    return out


def _exact_values(q, e=None):
    """A kept 4-bit tensor's values from the bits of its codes: sign, two exponent bits, one of fraction."""
    codes, scales, cols = _parts(q)
    if e is not None:
        codes, scales = codes[e], scales[e]
    rows, half = codes.shape
    c = torch.empty((rows, half * 2), device=codes.device, dtype=torch.uint8)
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    ex, m = ((c >> 1) & 3).double(), (c & 1).double()
    v = torch.where(ex > 0, (1 + m / 2) * torch.exp2(ex - 1), m / 2) * (1 - 2 * (c >> 3).double())
    r = torch.arange(rows, device=codes.device)[:, None]
    b = torch.arange(half // 16, device=codes.device)[None, :]
    at = (b // 16) * 256 + ((b % 4) * 16 + r % 16) * 4 + (b // 4) % 4
    s = scales[(r // 16).expand(rows, half // 16), at].double()
    v = v.view(rows, half // 16, 32) * torch.exp2(s - 127)[..., None]
    return v.view(rows, half * 2)[:, :cols]


def _exact_moe(s):
    x = s["x"].double()
    T, k = s["T"], s["k"]
    logits = x @ s["router"].double().t()
    p = torch.softmax(logits, 1)
    y = torch.zeros_like(x)
    ids = torch.full((T, k), -1, dtype=torch.int32)
    w = torch.zeros((T, k), dtype=torch.float64)
    host = p.cpu()
    for t in range(T):
        if s["mask"] is not None and not bool(s["mask"][t]):
            continue
        pick = sorted(range(s["E"]), key=lambda e: (-float(host[t, e]), e))[:k]
        total = sum(float(host[t, e]) for e in pick) if s["renorm"] else 1.0
        for j, e in enumerate(pick):
            ids[t, j], w[t, j] = e, float(host[t, e]) / total
    for e in range(s["E"]):
        hit = (ids == e).nonzero()
        if not len(hit):
            continue
        t, j = hit[:, 0].to(DEV), hit[:, 1]
        wg, wu, wd = ((s[n][e].double() if isinstance(s[n], torch.Tensor) else _exact_values(s[n], e))
                      for n in ("gate", "up", "down"))
        a = x[t] @ wg.t()
        a = a * torch.sigmoid(a) * (x[t] @ wu.t())
        y.index_add_(0, t, w[hit[:, 0], j].to(DEV)[:, None] * (a @ wd.t()))
    return {"y": y, "ids": None, "w": w}


def _exact_norm(s):
    f, x = s["f"].double(), s["x"].double()
    r1 = (f.square().mean(1) + EPS).rsqrt()
    y = s["w_post"].double() * (f / (f.square().mean(1) + EPS).sqrt()[:, None])
    if s["gate"] is not None:
        y = (y.view(s["groups"], -1, s["D"]) * s["gate"].double()[:, None]).view(f.shape)
    y = y + s["alpha"] * x
    r2 = (y.square().mean(1) + EPS).rsqrt()
    return {"y": y, "h": y * r2[:, None] * s["w_pre"].double(), "rstd": torch.stack((r1, r2), 1)}


def _exact_norm_bwd(s):
    f, y, dy, dh = (s[n].double() for n in ("f", "y", "dy", "dh"))
    r1, r2 = s["rstd"].double().unbind(1)
    w1, w2 = s["w_post"].double(), s["w_pre"].double()
    yn = y * r2[:, None]
    u = dh * w2
    d = dy + r2[:, None] * (u - yn * (u * yn).mean(1, keepdim=True))
    fn = f * r1[:, None]
    gate = torch.ones((1, s["D"]), device=DEV, dtype=torch.float64) if s["gate"] is None else s["gate"].double()
    dn = (d.view(gate.shape[0], -1, s["D"]) * gate[:, None]).view(d.shape)
    v = dn * w1
    out = {"df": r1[:, None] * (v - fn * (v * fn).mean(1, keepdim=True)), "dx": s["alpha"] * d,
           "dw_post": (dn * fn).sum(0), "dw_pre": (dh * yn).sum(0)}
    if s["gate"] is not None:
        out["dgate"] = (d * fn).view(s["groups"], -1, s["D"]).sum(1) * w1
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        out = {"v": _exact_quantized(s["x"])}
        if case["both"]:
            out["vt"] = _exact_quantized(s["x"].t())
        return out
    if op == "linear":
        return _exact_quantized(s["x"]) @ _exact_values(s["W"]).t()
    if op == "linear_bwd":
        return {"dx": _exact_quantized(s["dy"]) @ _exact_values(s["Wt"]).t(),
                "dw": _exact_quantized(s["dy"].t()) @ _exact_values(s["xt"]).t()}
    if op == "moe":
        return _exact_moe(s)
    return _exact_norm(s) if op == "norm" else _exact_norm_bwd(s)
