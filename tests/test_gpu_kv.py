"""occ_kv_tables and occ_rope against plain implementations in whole numbers and 64 bits.

Tolerances of the rotation: the angle's remainder is exact but for its conversion to binary32 (2^-25 of a half turn at most,
which is 2^-23 of an angle below pi) and the sine's own 2 ulp, so cos and sin are off by less than 2^-21; times scale, and two
products and a sum of three roundings: 2^-20 of scale (|x_0| + |x_1|).  bf16 outputs add one rounding, 2^-8."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def run_tables(cached, fresh, table, ring, free, page, pages, rows, ld=None, stream=None):
    n, width = len(cached), len(table[0]) if table else 0
    wide = torch.full((n, ld or width), -77, dtype=torch.int32, device=DEV)
    t = wide[:, :width]
    if width:
        t.copy_(i32(table))
    r = i32(ring)
    lens, starts, slots, positions, after = (torch.full((m,), -99, dtype=torch.int32, device=DEV) for m in (n, n + 1, rows, rows, 2))
    occ.occ_kv_tables(i32(cached), i32(fresh), t, r, i32(free), page=page, pages=pages, lens=lens, starts=starts, slots=slots,
                      positions=positions, free_after=after, stream=stream)
    if ld:
        assert bool((wide[:, width:] == -77).all())
    return [v.tolist() for v in (t, r, lens, starts, slots, positions, after)]


def problem(n, page, seed, most=100, over=0.1, spare=5, chunk=20, holes=False):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, most, n).tolist()
    fresh = [-1 if rng.random() < over else int(rng.integers(0, chunk)) for _ in range(n)]
    used = [-(-c // page) for c in cached]
    width = max(-(-(c + chunk) // page) for c in cached) + 1
    need = sum(-(-(c + max(f, 0)) // page) - u for c, f, u in zip(cached, fresh, used))
    free = max(0, need + spare)
    pages = sum(used) + free
    ids = rng.permutation(pages).tolist()
    table = []
    for u in used:
        table.append([ids.pop() for _ in range(u)] + [-5] * (width - u))
    if holes:
        for row in table:
            for j in range(len(row)):
                if rng.random() < 0.1:
                    row[j] = int(rng.choice([-1, pages, 2 ** 31 - 1]))
    size = max(1, pages)
    head = int(rng.integers(0, size))
    ring = [-3] * size
    for j, p in enumerate(ids):
        ring[(head + j) % size] = p
    return cached, fresh, table, ring, [head, free], page, pages


@pytest.mark.parametrize("n,page,spare,chunk", [(1, 1, 0, 2), (3, 16, 5, 20), (64, 16, 0, 2), (255, 3, -40, 9), (256, 48, 3, 40),
                                                (257, 64, -30, 100), (700, 5, -200, 12), (1500, 16, 9, 30), (2047, 2, -50, 7),
                                                (2048, 8, 0, 3), (2049, 8, 0, 3), (5000, 3, -900, 11)])
def test_tables(n, page, spare, chunk):
    for seed in range(3):
        p = problem(n, page, seed, spare=spare, chunk=chunk, holes=seed == 2)
        rows = sum(max(f, 0) for f in p[1]) + seed * 3
        got = run_tables(*p, rows, ld=len(p[2][0]) + 5 if seed else None)
        assert got == list(map(list, ref.tables(*p, rows)))


def test_tables_edges():
    def check(cached, fresh, table, ring, free, page, pages, rows):
        got = run_tables(cached, fresh, table, ring, free, page, pages, rows)
        assert got == list(map(list, ref.tables(cached, fresh, table, ring, free, page, pages, rows)))
        return got
    # nothing cached, nothing asked; a request that fills its page; one that is full
    check([0, 3, 4], [0, 1, 1], [[-1, -1], [0, -1], [1, -1]], [2, 3, -1, -1], [0, 2], 4, 4, 2)
    # beyond the row of the table, negative lengths, sums past 31 bits: refused, the others served
    big = 2 ** 31 - 1
    got = check([7, -2, 5, big, 0], [2, 1, 1, 1, big], [[0, 1], [-1, -1], [2, 3], [0, 0], [-1, -1]], [4, 5], [1, 2], 4, 6, 8)
    assert got[2] == [-1, -1, 6, -1, -1]
    # more tokens than rows: those that end within them are served, and behind them none (a sum of 9 is past 7)
    got = check([0] * 5, [3, 3, 3, 0, 1], [[-1, -1]] * 5, list(range(6)), [0, 6], 4, 6, 7)
    assert got[2] == [3, 3, -1, -1, -1] and got[3] == [0, 3, 6, 7, 7, 7]
    # no free page at all, and a free list that says nonsense is taken within the ring
    check([4, 3], [1, 1], [[0, -1], [1, -1]], [9, 9], [0, 0], 4, 2, 2)
    # all over: pages go behind the free ones, across the ring's end
    got = check([9, 4, 0], [-1, -7, -1], [[5, 6, 7], [8, -1, -1], [-1, -1, -1]], [-1, -1, -1, 1, 2, -1, -1], [3, 2], 4, 9, 0)
    assert got[6] == [3, 6] and got[1] == [7, 8, -1, 1, 2, 5, 6]
    # a width of nothing
    check([0, 0], [0, 1], [[], []], [0], [0, 1], 4, 1, 1)


def test_tables_without_requests():
    """Nothing is asked: no token has a slot, and the free pages stay."""
    empty = torch.empty((0, 5), dtype=torch.int32, device=DEV)
    ring, free = i32([4, 5, 6, 7]), i32([3, 2])
    for rows in (0, 300):
        starts, slots, positions, after = (torch.full((m,), -99, dtype=torch.int32, device=DEV) for m in (1, rows, rows, 2))
        occ.occ_kv_tables(empty[:, 0].contiguous(), empty[:, 0].contiguous(), empty, ring, free, page=4, pages=8, lens=empty[:, 0].contiguous(),
                          starts=starts, slots=slots, positions=positions, free_after=after)
        assert starts.tolist() == [0] and slots.tolist() == [-1] * rows and positions.tolist() == [0] * rows
        assert after.tolist() == [3, 2] and ring.tolist() == [4, 5, 6, 7]


def test_tables_long_requests():
    # more pages and tokens than a wave or a workgroup has lanes, of one request
    cached, fresh, page = [5000, 100000], [9000, -1], 16
    used = [-(-c // page) for c in cached]
    table = [list(range(u)) + [-1] * (6300 - u) for u in used]
    ring = list(range(20000, 20000 + 8000))
    p = (cached, fresh, table, ring, [7900, 700], page, 30000)
    got = run_tables(*p, 9100)
    assert got == list(map(list, ref.tables(*p, 9100)))


def test_tables_replayed_and_on_streams():
    """A captured step, replayed on new lengths, keeps a program's state: lens become cached, free_after free."""
    page, n, rows = 4, 6, 12
    cached, fresh = [0] * n, [2] * n
    table, ring, free = [[-1] * 8 for _ in range(n)], list(range(40)), [0, 40]
    d = dict(cached=i32(cached), fresh=i32(fresh), table=i32(table), ring=i32(ring), free=i32(free))
    o = {k: i32([0] * m) for k, m in (("lens", n), ("starts", n + 1), ("slots", rows), ("positions", rows), ("free_after", 2))}
    before = {k: v.clone() for k, v in d.items()}

    def step():
        occ.occ_kv_tables(d["cached"], d["fresh"], d["table"], d["ring"], d["free"], page=page, pages=40, **o)
        d["cached"].copy_(torch.where(o["lens"] < 0, d["cached"], o["lens"]))
        d["free"].copy_(o["free_after"])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k, v in before.items():
        d[k].copy_(v)
    for k in range(9):
        fresh = [2, 1, -1 if k == 5 else 2, 0, 3 if k % 2 else 1, 2]
        d["fresh"].copy_(i32(fresh))
        graph.replay()
        torch.cuda.synchronize()
        table, ring, lens, starts, slots, positions, free = map(list, ref.tables(cached, fresh, table, ring, free, page, 40, rows))
        assert [o[x].tolist() for x in ("lens", "starts", "slots", "positions", "free_after")] == [lens, starts, slots, positions, free]
        assert d["table"].tolist() == table and d["ring"].tolist() == ring
        cached = [c if x < 0 else x for c, x in zip(cached, lens)]


# ------------------------------------------------------------------ rotary positions

def rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(dtype).to(DEV)


def f64(t):
    return t.double().cpu().numpy()


def close(got, want, x, pairs, interleaved, scale, dtype):
    a = np.abs(f64(x))
    mag = a.copy()
    if interleaved:
        s = a[..., 0:2 * pairs:2] + a[..., 1:2 * pairs:2]
        mag[..., 0:2 * pairs:2], mag[..., 1:2 * pairs:2] = s, s
    else:
        s = a[..., :pairs] + a[..., pairs:2 * pairs]
        mag[..., :pairs], mag[..., pairs:2 * pairs] = s, s
    tol = 2.0 ** -20 * abs(scale) * mag + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0) + 1e-30
    err = np.abs(f64(got) - want)
    assert (err <= tol).all(), (float(err.max()), np.argwhere(~(err <= tol))[:4].tolist())
    assert np.array_equal(f64(got)[..., 2 * pairs:], f64(x)[..., 2 * pairs:])


SIZES = [(1, 1, 1, 2, 1), (3, 2, 1, 8, 4), (5, 3, 1, 10, 3), (7, 4, 2, 64, 32), (2, 8, 8, 128, 64), (33, 5, 5, 80, 20), (9, 2, 2, 96, 48),
         (4, 1, 1, 256, 64), (6, 3, 1, 128, 0), (3, 1, 1, 1024, 512)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,Hq,Hkv,D,pairs", SIZES)
def test_rope(rows, Hq, Hkv, D, pairs, interleaved, dtype):
    q, k = rand((rows, Hq, D), dtype, 1), rand((rows, Hkv, D), dtype, 2)
    pos = torch.randint(0, 1 << 20, (rows,), generator=torch.Generator().manual_seed(3)).int()
    pos[0], pos[-1] = -5, 2 ** 31 - 1
    turns = occ.rope_turns(pairs, base=1e6, linear=0.9)
    for inverse in (False, True):
        for scale in (1.0, -1.3):
            qo, ko = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
            got = occ.occ_rope(q, k, pos.to(DEV), turns, q_out=qo, k_out=ko, interleaved=interleaved, scale=scale, inverse=inverse)
            assert got[0] is qo and got[1] is ko
            for x, y in ((q, qo), (k, ko)):
                want = ref.rope(f64(x), pos.tolist(), turns.tolist(), interleaved, scale, inverse)
                close(y, want, x, pairs, interleaved, scale, dtype)
    # in place, each alone: the same bits
    q2, k2 = q.clone(), k.clone()
    occ.occ_rope(q2, None, pos.to(DEV), turns, interleaved=interleaved, scale=scale, inverse=inverse)
    occ.occ_rope(None, k2, pos.to(DEV), turns, interleaved=interleaved, scale=scale, inverse=inverse)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


def test_rope_many_rows_is_row_by_row():
    """Several rows to a workgroup: the bits of the same rows a few at a time."""
    rows, Hq, Hkv, D = 9001, 3, 1, 64
    q, k = rand((rows, Hq, D), BF16, 4), rand((rows, Hkv, D), BF16, 5)
    pos, turns = torch.arange(rows, device=DEV, dtype=torch.int32) * 7, occ.rope_turns(32)
    qo, ko = occ.occ_rope(q, k, pos, turns, q_out=torch.empty_like(q), k_out=torch.empty_like(k))
    for a in (0, 4095, 8999):
        b = a + 2
        x, y = occ.occ_rope(q[a:b].clone(), k[a:b].clone(), pos[a:b].clone(), turns)
        assert torch.equal(x, qo[a:b]) and torch.equal(y, ko[a:b])


@pytest.mark.parametrize("rows,Hq,Hkv,D,dtype", [(255, 20, 4, 80, BF16), (256, 20, 4, 80, BF16), (257, 64, 8, 128, BF16), (4500, 32, 8, 128, BF16),
                                                 (3000, 32, 8, 96, torch.float32)])
def test_rope_by_launches(rows, Hq, Hkv, D, dtype):
    """Workgroups of other sizes, and outputs larger than the L2s hold: the bits of the same rows a few at a time, in the cache
    and beside it."""
    page, pages = 16, rows // 16 + 3
    q, k, v = (rand((rows, h, D), dtype, 8 + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    pos, turns = torch.arange(rows, device=DEV, dtype=torch.int32) * 3, occ.rope_turns(D // 2)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(9))[:rows].to(torch.int32).to(DEV)
    slots[5] = -1
    kc, vc = (torch.full((pages, page, Hkv, D), 3.0, dtype=dtype, device=DEV) for _ in range(2))
    qo, ko = occ.occ_rope(q, k, pos, turns, q_out=torch.empty_like(q), k_out=torch.empty_like(k), v=v, k_cache=kc, v_cache=vc, slots=slots)
    here = slots >= 0
    assert torch.equal(kc.flatten(0, 1)[slots[here].long()], ko[here]) and torch.equal(vc.flatten(0, 1)[slots[here].long()], v[here])
    rest = torch.ones(pages * page, dtype=torch.bool, device=DEV)
    rest[slots[here].long()] = False
    assert bool((kc.flatten(0, 1)[rest] == 3).all()) and bool((vc.flatten(0, 1)[rest] == 3).all())
    for a in (0, 100, rows - 3):
        x, y = occ.occ_rope(q[a:a + 3].clone(), k[a:a + 3].clone(), pos[a:a + 3].clone(), turns)
        assert torch.equal(x, qo[a:a + 3]) and torch.equal(y, ko[a:a + 3])


@pytest.mark.parametrize("form", ["rows", "heads", "planes", "odd"])
def test_rope_into_the_cache(form):
    """From a joint projection's rows into caches of several layouts; rows without a slot, or one past the cache, go nowhere."""
    rows, Hq, Hkv, D, page, pages = 21, 6, 2, 64, 5, 8
    joint = rand((rows, Hq + 2 * Hkv, D + (2 if form == "odd" else 0)), BF16, 6)[..., :D]
    q, k, v = joint[:, :Hq], joint[:, Hq:Hq + Hkv], joint[:, Hq + Hkv:]
    before = joint.clone()
    if form == "heads":
        caches = [torch.full((pages, Hkv, page, D), 3.0, dtype=BF16, device=DEV).transpose(1, 2) for _ in range(2)]
    elif form == "planes":
        both = torch.full((pages, 2, page, Hkv, D), 3.0, dtype=BF16, device=DEV)
        caches = [both[:, 0], both[:, 1]]
    else:
        caches = [torch.full((pages, page, Hkv, D), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    g = torch.Generator().manual_seed(8)
    slots = torch.randperm(page * pages, generator=g)[:rows].int()
    slots[3], slots[7], slots[9], slots[20] = -1, page * pages, 2 ** 31 - 1, -2 ** 31
    pos, turns = torch.randint(0, 5000, (rows,), generator=g).int(), occ.rope_turns(32)
    qo = torch.empty((rows, Hq, D), dtype=BF16, device=DEV)
    got = occ.occ_rope(q, k, pos.to(DEV), turns, q_out=qo, v=v, k_cache=caches[0], v_cache=caches[1], slots=slots.to(DEV))
    assert got[1] is None and torch.equal(joint, before)
    plain_q, plain_k = occ.occ_rope(q, k, pos.to(DEV), turns, q_out=torch.empty_like(qo), k_out=torch.empty((rows, Hkv, D), dtype=BF16, device=DEV))
    assert torch.equal(qo, plain_q)
    want = [torch.full((pages * page, Hkv, D), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    for r, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            want[0][s], want[1][s] = plain_k[r], v[r]
    for c, w in zip(caches, want):
        assert torch.equal(c.reshape(pages * page, Hkv, D), w)
    # in place on the joint rows, the cache beside it: the same again
    occ.occ_rope(q, k, pos.to(DEV), turns, k_out=k, v=v, k_cache=caches[0], v_cache=caches[1], slots=slots.to(DEV))
    assert torch.equal(q, plain_q) and torch.equal(k, plain_k) and torch.equal(v, before[:, Hq + Hkv:])


def test_rope_gradient_is_that_of_differences():
    """The inverse call gives the gradient: <dy, d rope(x)> = <rope_inverse(dy), dx>, and central differences agree.
    rope is linear, so a difference over 2 h has the two values' roundings only: 2^-23 / h of their size each."""
    rows, H, D = 3, 2, 16
    x, dy = rand((rows, H, D), F32, 9), rand((rows, H, D), F32, 10)
    pos, turns = i32([3, 70, 1001]), occ.rope_turns(5)
    dx, _ = occ.occ_rope(dy, None, pos, turns, q_out=torch.empty_like(dy), scale=0.8, inverse=True)

    def loss(v):
        y, _ = occ.occ_rope(v, None, pos, turns, q_out=torch.empty_like(v), scale=0.8)
        return (y.double() * dy.double()).sum()
    h = 0.25
    for r, head, d in ((0, 0, 0), (1, 1, 4), (2, 0, 7), (1, 0, 12), (2, 1, 9)):
        step = torch.zeros_like(x)
        step[r, head, d] = h
        diff = (loss(x + step) - loss(x - step)) / (2 * h)
        tol = 2.0 ** -19 / h * float(dy.abs().double().sum())
        assert abs(float(diff) - float(dx[r, head, d])) <= tol


def test_rope_in_a_graph_and_on_a_stream():
    rows, H, D = 5, 4, 64
    q, pos, turns = rand((rows, H, D), BF16, 11), i32(list(range(rows))), occ.rope_turns(32)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        occ.occ_rope(q, None, pos, turns, q_out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        occ.occ_rope(q, None, pos, turns, q_out=out)
    for k in range(3):
        pos.add_(1000)
        q.copy_(rand((rows, H, D), BF16, 12 + k))
        eager = occ.occ_rope(q.clone(), None, pos, turns)[0]
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
