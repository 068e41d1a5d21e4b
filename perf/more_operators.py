"""What a decoder keeps and reads between its norms and its experts: a cache in pages, rotary positions, attention.

``tables``: block tables, slots and positions of a step's tokens from the lengths of its requests.
``rope``: rotary positions of queries and keys, forward with keys and values put into their slots
of the cache, and backward.  ``attn``: attention of each request's new tokens (one, or a chunk)
over its pages.

``listed`` names fixed cases, ``draw`` gives others of the same ranges; ``prepare`` makes what a
program holds before the call, ``run`` is one pass: in elementary torch operations in 32 bits
where ``own`` is false, through the library's entry points where it is true.  ``exact`` is the
definition in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
DTYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # a decode step of 64 requests, a few of them over: launch and latency
        dict(name="tables_decode", op="tables", n=64, cached_lo=1, cached_hi=8192, chunks=0, chunk_lo=1, chunk_hi=1, over=3,
             page=16, short=False),
        # a large batch whose prompts come in chunks, with more asked for than there are pages
        dict(name="tables_chunks", op="tables", n=1500, cached_lo=0, cached_hi=20000, chunks=700, chunk_lo=1, chunk_hi=1024,
             over=50, page=48, short=True),
        # a decode step of 16 sequences at hidden size 8192
        dict(name="rope_decode", op="rope", T=16, Hq=64, Hkv=8, D=128, rot=128, interleaved=False, dtype="bf16", page=16, far=131072),
        # the chunk of a long prompt
        dict(name="rope_chunk", op="rope", T=8192, Hq=64, Hkv=8, D=128, rot=128, interleaved=False, dtype="bf16", page=64,
             far=1000000),
        # gradients of a training batch, interleaved pairs in half of heads of odd size, 32 bits
        dict(name="rope_bwd", op="rope_bwd", T=3001, Hq=20, Hkv=4, D=80, rot=40, interleaved=True, dtype="f32", page=1, far=8192),
        # a few short conversations: latency
        dict(name="attn_short", op="attn", n=4, cached_lo=100, cached_hi=900, chunks=0, chunk_lo=1, chunk_hi=1, Hq=32, Hkv=8,
             D=128, page=16, window=0),
        # one long document: the work has to be split along its keys
        dict(name="attn_long", op="attn", n=1, cached_lo=130000, cached_hi=130000, chunks=0, chunk_lo=1, chunk_hi=1, Hq=64, Hkv=8,
             D=128, page=64, window=0),
        # a decode step of a ragged batch
        dict(name="attn_batch", op="attn", n=64, cached_lo=1, cached_hi=8191, chunks=0, chunk_lo=1, chunk_hi=1, Hq=64, Hkv=8,
             D=128, page=16, window=0),
        # a step of decoding requests beside the chunk of a prompt
        dict(name="attn_mixed", op="attn", n=17, cached_lo=500, cached_hi=4000, chunks=1, chunk_lo=512, chunk_hi=512, Hq=32,
             Hkv=8, D=128, page=32, window=0),
        # prompts of odd sizes, heads of 64 that are shared by seven, a window, pages that end inside any tile
        dict(name="attn_window", op="attn", n=7, cached_lo=0, cached_hi=2500, chunks=7, chunk_lo=17, chunk_hi=700, Hq=28, Hkv=4,
             D=64, page=48, window=1000),
        # a whole prompt: the compute-bound end
        dict(name="attn_prompt", op="attn", n=1, cached_lo=0, cached_hi=0, chunks=1, chunk_lo=8192, chunk_hi=8192, Hq=32, Hkv=8,
             D=128, page=64, window=0),
        # the chunk of a prompt over what is cached of it, each head with its own keys
        dict(name="attn_chunk", op="attn", n=2, cached_lo=2000, cached_hi=6000, chunks=2, chunk_lo=1000, chunk_hi=1500, Hq=16,
             Hkv=16, D=128, page=16, window=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("tables", "rope", "rope", "rope_bwd", "attn", "attn", "attn", "attn"))
    if op == "tables":
        n = _log(rng, 1, 2048)
        chunks = rng.choice((0, rng.randint(0, n // 2)))
        return dict(op=op, n=n, cached_lo=rng.choice((0, 1, 100)), cached_hi=_log(rng, 100, 30000), chunks=chunks, chunk_lo=1,
                    chunk_hi=_log(rng, 1, 1024), over=rng.randint(0, (n - chunks) // 2), page=rng.choice((1, 16, 32, 48, 64, 256)),
                    short=rng.random() < 0.3)
    dims = ((32, 8), (64, 8), (28, 4), (16, 16), (24, 1), (8, 2), (40, 40), (64, 4))
    if op in ("rope", "rope_bwd"):
        Hq, Hkv = rng.choice(dims)
        D = rng.choice((64, 80, 96, 128, 256))
        return dict(op=op, T=_log(rng, 1, min(16384, (1 << 26) // ((Hq + 2 * Hkv) * D))), Hq=Hq, Hkv=Hkv, D=D,
                    rot=rng.choice((D, D, D // 2)), interleaved=rng.random() < 0.4, dtype=rng.choice(("bf16", "bf16", "f32")),
                    page=rng.choice((16, 24, 64)), far=_log(rng, 1000, 1000000))
    kind = rng.choice(("decode", "decode", "chunk", "mixed"))
    Hq, Hkv = rng.choice(dims)
    D = rng.choice((64, 128, 128, 80, 256))
    window = rng.choice((0, 0, 0, _log(rng, 16, 4096)))
    n = _log(rng, 1, 128) if kind != "chunk" else rng.randint(1, 8)
    # what the largest listed cases have: keys and values of the batch, pairs of a query and a key
    most = min(130000, (1 << 29) // (n * Hkv * D))
    chunk = 1
    if kind != "decode":
        pairs = (1 << 30) * 128 // (max(D, 128) * n * Hq)
        chunk = _log(rng, 2, min(4096 if kind == "chunk" else 512, math.isqrt(pairs) // 2))
        most = min(most, 32768, pairs // chunk - chunk)
    hi = _log(rng, min(most, 16), most)
    return dict(op=op, n=n, cached_lo=rng.choice((0, hi // 2, hi)), cached_hi=hi,
                chunks={"decode": 0, "chunk": n, "mixed": rng.randint(1, min(n, 3))}[kind], chunk_lo=max(1, chunk // 2),
                chunk_hi=chunk, Hq=Hq, Hkv=Hkv, D=D, page=rng.choice((1, 16, 32, 48, 64, 256)), window=window)


# ------------------------------------------------------------------ lengths

def _spread(i, lo, hi):
    """The i-th of values that fill [lo, hi] evenly, in no order."""
    return lo + int((i * 0.6180339887498949 + 0.37) % 1.0 * (hi - lo + 1))


def _lengths(c):
    """(cached, fresh) of a case's requests: the first `chunks` bring a chunk, the others one token; the last `over`
    of `tables` are over (-1)."""
    n, over = c["n"], c.get("over", 0)
    cached = [_spread(i, c["cached_lo"], c["cached_hi"]) for i in range(n)]
    fresh = [_spread(i, c["chunk_lo"], c["chunk_hi"]) if i < c["chunks"] else 1 for i in range(n)]
    for i in range(n - over, n):
        fresh[i] = -1
    # requests of one kind do not stand together
    order = sorted(range(n), key=lambda i: (i * 0.7548776662466927) % 1.0)
    return [cached[i] for i in order], [fresh[i] for i in order]


def _pages(n, page):
    return -(-n // page)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=F32).to(dtype)


def _ints(values):
    return torch.tensor(values, device=DEV, dtype=torch.int32)


def _tables_of(cached, page, width, perm):
    """A table of each request's pages, taken from `perm` in turn, -1 behind them; and how many were taken."""
    have = (torch.tensor(cached) + page - 1) // page
    end = torch.cumsum(have, 0)
    at = torch.arange(width)[None, :]
    index = ((end - have)[:, None] + at).to(DEV)
    table = torch.where((at < have[:, None]).to(DEV), perm[index.clamp(max=perm.numel() - 1)], -1)
    return table.to(torch.int32), int(end[-1])


def _prepare_tables(c, s, g):
    cached, fresh = _lengths(c)
    page = c["page"]
    T = sum(max(f, 0) for f in fresh)
    total = [x + max(f, 0) for x, f in zip(cached, fresh)]
    width = max(_pages(t, page) for t in total) + 2
    need = sum(_pages(t, page) - _pages(x, page) for x, t in zip(cached, total))
    used = sum(_pages(x, page) for x in cached)
    free = need * 3 // 4 if c["short"] else need + 37  # short: the last requests get none
    pages = used + free
    perm = torch.randperm(pages, generator=g, device=DEV)
    s["table"], taken = _tables_of(cached, page, width, perm)
    ring = torch.full((pages,), -1, device=DEV, dtype=torch.int32)
    head = pages // 3   # the ring's free pages run over its end
    ring[(head + torch.arange(free, device=DEV)) % pages] = perm[taken:].to(torch.int32)
    s["ring"], s["free"] = ring, _ints([head, free])
    s["cached"], s["fresh"], s["pages"] = _ints(cached), _ints(fresh), pages
    s["T"] = T + 7   # a program's buffers hold its largest step
    if own:
        for name, n in (("lens", c["n"]), ("starts", c["n"] + 1), ("slots", s["T"]), ("positions", s["T"]), ("free_after", 2)):
            s[name] = torch.empty(n, device=DEV, dtype=torch.int32)


def _prepare_rope(c, s, g):
    T, Hq, Hkv, D, page = c["T"], c["Hq"], c["Hkv"], c["D"], c["page"]
    dtype = DTYPES[c["dtype"]]
    # the joint projection's output holds q, k and v of a token side by side
    qkv = _randn(g, (T, Hq + 2 * Hkv, D), dtype)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    s["positions"] = torch.randint(0, c["far"], (T,), generator=g, device=DEV).to(torch.int32)
    half = c["rot"] // 2
    s["turns"] = _turns(half)
    s["m"] = 1.25   # an attention factor, as scaled frequencies come with
    s["q_out"] = torch.empty((T, Hq, D), device=DEV, dtype=dtype)
    if c["op"] == "rope_bwd":
        s["k_out"] = torch.empty((T, Hkv, D), device=DEV, dtype=dtype)
        return
    pages = _pages(T, page) + 2
    s["k_cache"], s["v_cache"] = (torch.zeros((pages, page, Hkv, D), device=DEV, dtype=dtype) for _ in range(2))
    perm = torch.randperm(pages - 1, generator=g, device=DEV)  # the last page stays empty
    t = torch.arange(T, device=DEV)
    slots = perm[t // page] * page + t % page
    s["slots"] = torch.where(t % 97 == 96, -1, slots).to(torch.int32)  # tokens of a padded batch have none


def _turns(half):
    """Turns per position of each pair, as 64-bit fractions of one turn."""
    values = [int(500000.0 ** (-i / half) / (2 * math.pi) * 2.0 ** 64) for i in range(half)]
    return torch.tensor([v - (1 << 64) if v >= 1 << 63 else v for v in values], device=DEV, dtype=torch.int64)


def _prepare_attn(c, s, g):
    cached, fresh = _lengths(c)
    page, Hq, Hkv, D = c["page"], c["Hq"], c["Hkv"], c["D"]
    lens = [x + f for x, f in zip(cached, fresh)]
    starts = [0]
    for f in fresh:
        starts.append(starts[-1] + f)
    pages = sum(_pages(x, page) for x in lens) + 3
    s["table"], _ = _tables_of(lens, page, max(_pages(x, page) for x in lens) + 1,
                               torch.randperm(pages, generator=g, device=DEV))
    s["k_cache"] = _randn(g, (pages, page, Hkv, D), BF16)
    s["v_cache"] = _randn(g, (pages, page, Hkv, D), BF16)
    s["q"] = _randn(g, (starts[-1], Hq, D), BF16)
    s["lens"], s["starts"] = _ints(lens), _ints(starts)
    s["longest"], s["max_fresh"] = max(lens), max(fresh)
    if own:
        from paper_2606_09200_amd import binding as occ
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((starts[-1], Hq), device=DEV)
        s["workspace"] = torch.zeros(occ.occ_attn_paged_workspace_bytes(Hq, Hkv, D), device=DEV, dtype=torch.uint8)


def prepare(case, seed):
    s = dict(case)
    {"tables": _prepare_tables, "rope": _prepare_rope, "rope_bwd": _prepare_rope, "attn": _prepare_attn}[case["op"]](
        case, s, _gen(seed))
    return s


# ------------------------------------------------------------------ one pass

def _tables_plain(s):
    page, T, pages = s["page"], s["T"], s["pages"]
    cached, fresh, table, ring = s["cached"].long(), s["fresh"].long(), s["table"], s["ring"]
    head, count = s["free"][0].long(), s["free"][1].long()
    width, size = table.shape[1], ring.numel()
    goes = fresh >= 0
    f = fresh.clamp(min=0)
    end = torch.cumsum(f, 0)
    start = end - f
    total = cached + f
    have, want = (cached + page - 1) // page, (total + page - 1) // page
    fits = goes & (cached >= 0) & (want <= width) & (end <= T)
    need = torch.where(fits, want - have, 0)
    upto = torch.cumsum(need, 0)
    ok = fits & ((need == 0) | (upto <= count))
    taken = torch.where(ok, upto, 0) * (need > 0)
    taken = taken.amax()
    # pages that requests get, and that go back
    at = torch.arange(width, device=DEV)[None, :]
    new = ok[:, None] & (at >= have[:, None]) & (at < want[:, None])
    table = torch.where(new, ring[(head + (upto - need - have)[:, None] + at) % size], table)
    back = torch.where(goes, 0, have.clamp(min=0, max=width))
    back_end = torch.cumsum(back, 0)
    index = count + (back_end - back)[:, None] + at
    index = torch.where((at < back[:, None]) & (index < size), (head + index) % size, size)
    ring = torch.cat((ring, ring[:1])).scatter(0, index.reshape(-1), table.reshape(-1))[:size]
    left = torch.minimum(count - taken + back_end[-1], size - taken)
    # the tokens
    t = torch.arange(T, device=DEV)
    i = (t[:, None] >= end[None, :]).sum(1) if T * len(end) < (1 << 24) else torch.searchsorted(end, t, right=True)
    there = i < len(end)
    i = i.clamp(max=len(end) - 1)
    there = there & ok[i]
    position = torch.where(there, cached[i] + t - start[i], 0)
    p = table[i, (position // page).clamp(max=width - 1)].long()
    slot = torch.where(there & (p >= 0) & (p < pages), p * page + position % page, -1)
    return {"table": table, "ring": ring, "free_after": torch.stack(((head + taken) % size, left)).to(torch.int32),
            "lens": torch.where(goes, torch.where(ok, total, -1), 0).to(torch.int32),
            "starts": torch.cat((torch.zeros_like(end[:1]), end.clamp(max=T))).to(torch.int32),
            "slots": slot.to(torch.int32), "positions": position.to(torch.int32)}


def _rotate_plain(s, x, sign):
    """Heads of x (T, H, D) turned by their token's angles, in 32 bits; the angles in 64."""
    half = s["rot"] // 2
    phase = s["positions"].long()[:, None] * s["turns"][None, :]   # modulo one turn
    angle = phase.double() * (2 * math.pi * 2.0 ** -64)
    cos = (torch.cos(angle) * s["m"]).float()[:, None, :]
    sin = (torch.sin(angle) * s["m"] * sign).float()[:, None, :]
    y = x.float()
    if s["interleaved"]:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, y[..., 2 * half:]), -1).to(x.dtype)


def _rope_plain(s):
    if s["op"] == "rope_bwd":
        return {"dq": _rotate_plain(s, s["q"], -1.0), "dk": _rotate_plain(s, s["k"], -1.0)}
    slots = s["slots"].long()
    for name, x in (("k_cache", _rotate_plain(s, s["k"], 1.0)), ("v_cache", s["v"])):
        rows = s[name].flatten(0, 1)
        rows[torch.where(slots >= 0, slots, rows.shape[0] - 1)] = torch.where((slots >= 0)[:, None, None], x, 0)
    return {"q": _rotate_plain(s, s["q"], 1.0), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attn_plain(s):
    Hq, Hkv, D, n, page = s["Hq"], s["Hkv"], s["D"], s["n"], s["page"]
    L, U, G = s["longest"], s["max_fresh"], s["Hq"] // s["Hkv"]
    starts, lens = s["starts"].long(), s["lens"].long()
    fresh = starts[1:] - starts[:-1]
    u, j = torch.arange(U, device=DEV), torch.arange(L, device=DEV)
    rows = (starts[:-1, None] + u).clamp(max=len(s["q"]) - 1)
    q = s["q"].float()[rows].view(n, U, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * U, D)
    slots = (s["table"].long()[:, j // page] * page + j % page).clamp(min=0)
    k = s["k_cache"].flatten(0, 1)[slots].float().permute(0, 2, 3, 1)
    at = (lens - fresh)[:, None] + u   # positions of the queries
    seen = (j[None, None, :] <= at[..., None]) & (j < lens[:, None])[:, None, :]
    if s["window"]:
        seen &= j[None, None, :] > at[..., None] - s["window"]
    x = torch.matmul(q, k).view(n, Hkv, G, U, L) * D ** -0.5
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top > -math.inf, top, 0))
    total = x.sum(-1, keepdim=True)
    v = s["v_cache"].flatten(0, 1)[slots].float().permute(0, 2, 1, 3)
    o = torch.matmul(x.view(n, Hkv, G * U, L), v).view(n, Hkv, G, U, D) / torch.where(total > 0, total, 1)
    lse = (top + torch.log(total)).view(n, Hkv, G, U)
    t = torch.arange(len(s["q"]), device=DEV)
    i = (t[:, None] >= starts[None, 1:]).sum(1)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, U, Hq, D)[i, t - starts[i]]
    return {"out": o.to(BF16), "lse": lse.permute(0, 3, 1, 2).reshape(n, U, Hq)[i, t - starts[i]]}


def _run_own(s):
    from paper_2606_09200_amd import binding as occ
    op = s["op"]
    if op == "tables":
        occ.occ_kv_tables(s["cached"], s["fresh"], s["table"], s["ring"], s["free"], page=s["page"], pages=s["pages"],
                          lens=s["lens"], starts=s["starts"], slots=s["slots"], positions=s["positions"],
                          free_after=s["free_after"])
        return {k: s[k] for k in ("table", "ring", "free_after", "lens", "starts", "slots", "positions")}
    if op == "rope":
        occ.occ_rope(s["q"], s["k"], s["positions"], s["turns"], q_out=s["q_out"], interleaved=s["interleaved"], scale=s["m"],
                     v=s["v"], k_cache=s["k_cache"], v_cache=s["v_cache"], slots=s["slots"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "rope_bwd":
        occ.occ_rope(s["q"], s["k"], s["positions"], s["turns"], q_out=s["q_out"], k_out=s["k_out"],
                     interleaved=s["interleaved"], scale=s["m"], inverse=True)
        return {"dq": s["q_out"], "dk": s["k_out"]}
    occ.occ_attn_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["lens"], s["out"],
                       max_fresh=s["max_fresh"], window=s["window"], lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    return _tables_plain(s) if op == "tables" else _attn_plain(s) if op == "attn" else _rope_plain(s)


# ------------------------------------------------------------------ what a pass cannot do without

def _pairs(cached, fresh, window):
    """Pairs of a new token and a key that it sees."""
    def first(m):   # 1 + 2 + .. + m
        return m * (m + 1) // 2
    total = first(cached + fresh) - first(cached)
    if window and cached + fresh > window:
        total -= first(cached + fresh - window) - first(max(0, cached - window))
    return total


def work(case):
    op = case["op"]
    if op == "tables":
        cached, fresh = _lengths(case)
        page, n = case["page"], case["n"]
        T = sum(max(f, 0) for f in fresh)
        new = sum(_pages(x + max(f, 0), page) - _pages(x, page) for x, f in zip(cached, fresh))
        back = sum(_pages(x, page) for x, f in zip(cached, fresh) if f < 0)
        return {"bytes": 20.0 * n + 8.0 * (new + back) + 8.0 * T, "flops": 10.0 * (n + T)}
    size = {"bf16": 2.0, "f32": 4.0}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if op == "rope" or op == "rope_bwd":
        heads = Hq + Hkv * (2 if op == "rope" else 1)
        return {"bytes": case["T"] * (2 * heads * D * size[case["dtype"]] + 8.0), "flops": 3.0 * case["T"] * (Hq + Hkv) * case["rot"]}
    cached, fresh = _lengths(case)
    T = sum(fresh)
    seen = sum(min(x + f, case["window"] + f - 1) if case["window"] else x + f for x, f in zip(cached, fresh))
    return {"bytes": 4.0 * T * Hq * D + 4.0 * T * Hq + 4.0 * seen * Hkv * D,
            "flops": 4.0 * Hq * D * sum(_pairs(x, f, case["window"]) for x, f in zip(cached, fresh))}


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_rope(s, x, sign):
    half = s["rot"] // 2
    # whole turns leave no trace: the fraction of a turn in two parts of 32 bits, each exact
    turns = s["turns"].view(torch.int32).view(half, 2).long()
    low, high = turns[:, 0] & 0xFFFFFFFF, turns[:, 1] & 0xFFFFFFFF
    pos = s["positions"].long()[:, None]
    part = (pos * high) % (1 << 32)
    turn = part.double() * 2.0 ** -32 + (pos * low).double() * 2.0 ** -64
    z = torch.polar(torch.full_like(turn, s["m"]), sign * 2 * math.pi * turn)[:, None, :]
    y = x.double().clone()
    if s["interleaved"]:
        y[..., :2 * half] = torch.view_as_real(torch.view_as_complex(y[..., :2 * half].reshape(*y.shape[:2], half, 2)) * z).flatten(-2)
    else:
        w = torch.complex(y[..., :half], y[..., half:2 * half]) * z
        y[..., :half], y[..., half:2 * half] = w.real, w.imag
    return y


def _exact_attn(s):
    Hq, Hkv, D, page = s["Hq"], s["Hkv"], s["D"], s["page"]
    G = Hq // Hkv
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    out = torch.zeros((starts[-1], Hq, D), device=DEV, dtype=torch.float64)
    lse = torch.zeros((starts[-1], Hq), device=DEV, dtype=torch.float64)
    for i, n in enumerate(lens):
        u0, u1 = starts[i], starts[i + 1]
        pages = s["table"][i, :_pages(n, page)].long()
        j = torch.arange(n, device=DEV)
        at = torch.arange(n - (u1 - u0), n, device=DEV)[:, None]
        hidden = (j > at) | ((j <= at - s["window"]) if s["window"] else torch.zeros_like(j > at))
        for h in range(Hkv):
            k = s["k_cache"][pages, :, h].reshape(-1, D)[:n].double()
            v = s["v_cache"][pages, :, h].reshape(-1, D)[:n].double()
            q = s["q"][u0:u1, h * G:(h + 1) * G].double().transpose(0, 1)
            x = (q @ k.t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
            lse[u0:u1, h * G:(h + 1) * G] = torch.logsumexp(x, -1).t()
            out[u0:u1, h * G:(h + 1) * G] = (torch.softmax(x, -1) @ v).transpose(0, 1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "tables":
        return None
    if op == "attn":
        return _exact_attn(s)
    if op == "rope_bwd":
        return {"dq": _exact_rope(s, s["q"], -1), "dk": _exact_rope(s, s["k"], -1)}
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    there = s["slots"] >= 0
    at = s["slots"][there].long()
    k_cache.flatten(0, 1)[at] = _exact_rope(s, s["k"], 1)[there]
    v_cache.flatten(0, 1)[at] = s["v"][there].double()
    return {"q": _exact_rope(s, s["q"], 1), "k_cache": k_cache, "v_cache": v_cache}
