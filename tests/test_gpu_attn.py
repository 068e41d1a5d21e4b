"""occ_attn_paged against a plain 64-bit implementation.

Tolerances.  A logit is a sum of D products in binary32: off by (D + 4) 2^-24 of scale sum |q| |k| (the scale's product,
the fused subtraction of the maximum and the exponential's argument are the 4), by which its weight p is off relatively, and by
2^-22 more for the exponential itself.  o is off by that much of sum p |v| / sum p, once in the sum and once in its
divisor, by the additions of a sum of n keys in binary32 (n 2^-24 at most) twice, by the weights' roundings to bf16 (2^-8; with
two bf16 values 2^-16), and by its own, 2^-8 of |o|.  lse is off by the logit's error, that of the sum (n 2^-24 + 2^-22) and
its own rounding."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


class Problem:
    """Requests (cached, fresh) with pages dealt out at random; what no key of a request is holds NaN."""

    def __init__(self, requests, Hq, Hkv, D, page, seed=0, layout="rows", spare=2, rows_behind=0, width=None, peaky=1.0):
        g = torch.Generator().manual_seed(seed)
        self.requests, self.Hq, self.Hkv, self.D, self.page = requests, Hq, Hkv, D, page
        lens = [c + f for c, f in requests]
        need = [-(-n // page) for n in lens]
        self.pages = sum(need) + spare
        ids = torch.randperm(self.pages, generator=g).tolist()
        width = width or max(need + [1]) + 1
        self.table = [[ids.pop() for _ in range(n)] + [-1] * (width - n) for n in need]
        self.starts = [0]
        for _, f in requests:
            self.starts.append(self.starts[-1] + f)
        self.rows = self.starts[-1] + rows_behind
        self.lens = lens
        nan = float("nan")
        shape = (self.pages, page, Hkv, D)
        self.k, self.v = (torch.full(shape, nan, dtype=torch.float64) for _ in range(2))
        for row, n in zip(self.table, lens):
            for j in range(n):
                self.k[row[j // page], j % page] = torch.randn(Hkv, D, generator=g, dtype=torch.float64)
                self.v[row[j // page], j % page] = torch.randn(Hkv, D, generator=g, dtype=torch.float64)
        self.q = torch.randn(max(self.rows, 1), Hq, D, generator=g, dtype=torch.float64)[:self.rows] * peaky
        self.layout = layout
        self.to_gpu()

    def to_gpu(self):
        q, k, v = (t.to(BF16).to(DEV) for t in (self.q, self.k, self.v))
        if self.layout == "heads":
            k, v = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (k, v))
            q = q.transpose(0, 1).contiguous().transpose(0, 1)
        elif self.layout == "joint":   # q in a joint projection's rows, k and v planes of one cache
            wide = torch.full((self.rows, self.Hq + 2 * self.Hkv, self.D), float("nan"), dtype=BF16, device=DEV)
            wide[:, :self.Hq] = q
            q = wide[:, :self.Hq]
            both = torch.stack((k, v), 1)
            k, v = both[:, 0], both[:, 1]
        self.dq, self.dk, self.dv = q, k, v
        self.dtable, self.dstarts, self.dlens = i32(self.table), i32(self.starts), i32(self.lens)

    def run(self, max_fresh=None, scale=None, causal=True, window=0, workspace=None, stream=None):
        self.out = torch.full((self.rows, self.Hq, self.D), 77.0, dtype=BF16, device=DEV)
        self.lse = torch.full((self.rows, self.Hq), 77.0, device=DEV)
        if workspace is None:
            workspace = workspace_for(self.D)
        if max_fresh is None:
            max_fresh = max([b - a for a, b in zip(self.starts, self.starts[1:])] + [0])
        occ.occ_attn_paged(self.dq, self.dk, self.dv, self.dtable, self.dstarts, self.dlens, self.out, max_fresh=max_fresh,
                           scale=scale, causal=causal, window=window, lse=self.lse, workspace=workspace, stream=stream)
        return self.out, self.lse

    def want(self, scale=None, causal=True, window=0):
        scale = self.D ** -0.5 if scale is None else scale
        k, v, q = (f64(t) for t in (self.dk, self.dv, self.dq))
        return ref.attention(q, k, v, self.table, self.starts, self.lens, scale, causal, window)

    def check(self, weights=2.0 ** -8, **how):
        out, lse = (f64(t) for t in self.run(**how))
        how.pop("max_fresh", None)
        how.pop("workspace", None)
        compare(out, lse, self.want(**how), self.D, weights)


def compare(out, lse, want, D, weights=2.0 ** -8):
    wo, wl, mag, logit, seen = want
    some = np.broadcast_to(seen[:, None] >= 0, wl.shape)
    nan = some & np.isnan(wl)   # a key that is seen holds NaN
    assert np.isnan(out[nan]).all() and np.isnan(lse[nan]).all()
    assert (out[~some] == 77).all() and (lse[~some] == 77).all(), "rows of no request"
    n = seen[:, None] * 2.0 ** -24
    err = (D + 4) * 2.0 ** -24 * logit + 2.0 ** -22
    empty = some & (wl == -np.inf)
    assert (out[empty] == 0).all() and (lse[empty] == -np.inf).all()
    full = some & ~empty & ~nan
    tol = (2 * err + 2 * n + weights)[..., None] * mag + 2.0 ** -8 * np.abs(wo) + 1e-30
    off = np.abs(out - wo)
    bad = full[..., None] & ~(off <= tol)
    assert not bad.any(), ("out", np.argwhere(bad)[:4].tolist(), float(np.nanmax(np.where(bad, off / tol, 0))))
    off = np.abs(np.where(full, lse, 0) - np.where(full, wl, 0))
    tol = err + n + 2.0 ** -22 + 2.0 ** -23 * np.abs(np.where(full, wl, 0))
    assert (off <= tol)[full].all(), ("lse", float((off / tol)[full].max()))


_workspaces = {}


def workspace_for(D, fresh=False):
    """One zeroed workspace for all calls of a size, as a program keeps it."""
    n = occ.occ_attn_paged_workspace_bytes(1, 1, D)
    if fresh:
        return torch.zeros(n, dtype=torch.uint8, device=DEV)
    if n not in _workspaces:
        _workspaces[n] = torch.zeros(n, dtype=torch.uint8, device=DEV)
    return _workspaces[n]


def teardown_module():
    torch.cuda.synchronize()
    for w in _workspaces.values():
        assert int(w[:1024].view(torch.int32).abs().sum()) == 0, "counters are left"
    _workspaces.clear()


DECODE = [(0, 1)], [(30, 1)], [(31, 1), (32, 1), (0, 1)], [(5, 1)] * 9 + [(700, 1)], [(1999, 1), (0, 0), (63, 1)]


@pytest.mark.parametrize("requests", DECODE)
@pytest.mark.parametrize("Hq,Hkv,D,page", [(1, 1, 64, 16), (8, 2, 128, 16), (7, 1, 64, 48), (32, 2, 128, 1), (40, 1, 256, 64), (4, 4, 8, 3),
                                          (6, 2, 80, 16), (12, 6, 136, 5)])
def test_single_tokens(requests, Hq, Hkv, D, page):
    Problem(requests, Hq, Hkv, D, page, seed=len(requests)).check(weights=2.0 ** -16)


CHUNKS = [(0, 1)], [(0, 129)], [(100, 70), (0, 200)], [(3, 64), (0, 65), (300, 1), (0, 0), (5, 2)]


@pytest.mark.parametrize("requests", CHUNKS)
@pytest.mark.parametrize("Hq,Hkv,D,page", [(1, 1, 64, 16), (4, 2, 128, 16), (7, 1, 64, 48), (5, 1, 128, 1), (2, 1, 256, 64), (2, 2, 8, 3),
                                          (3, 1, 80, 16), (2, 2, 136, 5), (20, 1, 64, 16), (130, 1, 64, 16), (4, 2, 96, 48), (2, 1, 72, 16),
                                          (2, 1, 104, 24), (2, 1, 40, 7)])
def test_chunks(requests, Hq, Hkv, D, page):
    Problem(requests, Hq, Hkv, D, page, seed=3).check(max_fresh=500)   # a large bound: the kernels of many rows


@pytest.mark.parametrize("window", [1, 2, 33, 100, 1 << 30])
@pytest.mark.parametrize("requests", [[(400, 1), (20, 1)], [(150, 90), (0, 130)]])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(requests, window, causal):
    p = Problem(requests, 6, 2, 64, 24, seed=5)
    p.check(window=window, causal=causal)
    p.check(window=window, causal=causal, max_fresh=1)   # the other kernel, whatever the bound says


def test_peaked_rows_and_scales():
    p = Problem([(500, 3), (0, 100)], 4, 2, 128, 16, seed=6, peaky=20.0)
    p.check(), p.check(scale=0.01), p.check(max_fresh=1, scale=1.0)


@pytest.mark.parametrize("layout", ["heads", "joint"])
@pytest.mark.parametrize("max_fresh", [1, 200])
def test_layouts(layout, max_fresh):
    Problem([(70, 1), (40, 100), (0, 3)], 8, 2, 64, 16, seed=7, layout=layout).check(max_fresh=max_fresh)


def test_a_table_wider_apart_and_rows_behind():
    p = Problem([(70, 1), (0, 0), (40, 5)], 8, 2, 64, 16, seed=8, rows_behind=9)
    wide = torch.full((3, p.dtable.shape[1] + 3), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    wide[:, :-3] = p.dtable
    p.dtable = wide[:, :-3]
    p.check(), p.check(max_fresh=400)


@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("max_fresh", [1, 400])
def test_unseen_infinities_and_nan(max_fresh, D):
    """Later tokens' keys and values are NaN or infinite: rows before them have the bits they have without."""
    p = Problem([(60, 12), (0, 90)], 4, 2, D, 16, seed=9)
    clean, clean_lse = (t.clone() for t in p.run(max_fresh=max_fresh))
    for bad in (float("nan"), float("inf"), -float("inf")):
        for i, (c, f) in enumerate(p.requests):
            last = c + f - 1
            at = p.table[i][last // p.page], last % p.page
            p.dk[at], p.dv[at] = bad, bad
        out, lse = p.run(max_fresh=max_fresh)
        for i, (c, f) in enumerate(p.requests):
            a, b = p.starts[i], p.starts[i + 1]
            assert torch.equal(out[a:b - 1], clean[a:b - 1]) and torch.equal(lse[a:b - 1], clean_lse[a:b - 1])
            assert bool(out[b - 1].isnan().all())
    # a window that has moved past them
    p = Problem([(60, 90)], 4, 2, D, 16, seed=9)
    p.check(window=8, max_fresh=max_fresh)
    clean = p.out.clone()
    for j in range(20):
        p.dk[p.table[0][j // 16], j % 16] = float("nan")
        p.dv[p.table[0][j // 16], j % 16] = float("inf")
    out, _ = p.run(window=8, max_fresh=max_fresh)
    assert torch.equal(out, clean)


@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("max_fresh", [1, 400])
def test_seen_infinite_values(max_fresh, D):
    """An infinite value that a row sees makes that one output infinite, and NaN a NaN; the others stay."""
    p = Problem([(50, 20)], 2, 1, D, 16, seed=10)
    clean, _ = (t.clone() for t in p.run(max_fresh=max_fresh))
    at = p.table[0][10 // 16], 10
    p.dv[at][0, 3], p.dv[at][0, 17], p.dv[at][0, 40] = float("inf"), -float("inf"), float("nan")
    out, _ = p.run(max_fresh=max_fresh)
    assert bool((out[:, :, 3] == float("inf")).all()) and bool((out[:, :, 17] == -float("inf")).all())
    assert bool(out[:, :, 40].isnan().all())
    keep = [d for d in range(D) if d not in (3, 17, 40)]
    assert torch.equal(out[:, :, keep], clean[:, :, keep])


@pytest.mark.parametrize("max_fresh", [1, 400])
def test_bad_pages_are_not_seen(max_fresh):
    p = Problem([(100, 40), (90, 1)], 4, 2, 64, 16, seed=11)
    p.table[0][2], p.table[0][5], p.table[1][0], p.table[1][5] = -1, p.pages, 2 ** 31 - 1, -2 ** 31
    p.dtable = i32(p.table)
    p.check(max_fresh=max_fresh)
    p.table = [[-1] * len(r) for r in p.table]   # nothing left
    p.dtable = i32(p.table)
    p.check(max_fresh=max_fresh)


@pytest.mark.parametrize("max_fresh", [1, 400])
def test_lengths_of_any_kind(max_fresh):
    """Lengths that no program should hold are taken within the buffers."""
    p = Problem([(40, 3), (20, 30), (10, 2)], 4, 2, 64, 16, seed=12)
    for lens in ([-1, 50, 0], [10 ** 9, -5, 2 ** 31 - 1], [1, 7, 12]):
        p.lens = lens
        p.dlens = i32(lens)
        # a length past a request's pages reads entries of -1: keys that are not seen
        p.check(max_fresh=max_fresh)
    p.lens = [43, 50, 12]
    p.dlens = i32(p.lens)
    for starts in ([0, 3, 33, 999], [-4, 3, 1, 35], [0, 0, 35, 35]):
        p.starts = starts
        p.dstarts = i32(starts)
        out, lse = (f64(t) for t in p.run(max_fresh=max_fresh))
        want = p.want()
        # rows 1 and 2 of the second are the first request's and the last's: either's result may be theirs
        claimed = np.zeros(p.rows, int)
        for a, b in zip(starts, starts[1:]):
            claimed[max(a, 0):max(a, 0, min(b, p.rows))] += 1
        one = claimed <= 1
        compare(out[one], lse[one], [w[one] for w in want], p.D)


def test_long_requests_are_shared_and_joined():
    """Few heads and many keys: every workgroup has a part of an item; the same bits every time, and from a graph."""
    p = Problem([(20000, 1), (9000, 2)], 4, 2, 64, 64, seed=13)
    p.check(weights=2.0 ** -16)
    first, first_lse = p.out.clone(), p.lse.clone()
    for _ in range(3):
        out, lse = p.run()
        assert torch.equal(out, first) and torch.equal(lse, first_lse)
    p = Problem([(9000, 70)], 2, 1, 64, 64, seed=14)
    p.check(max_fresh=70)
    first = p.out.clone()
    for _ in range(3):
        assert torch.equal(p.run(max_fresh=70)[0], first)


@pytest.mark.parametrize("requests,D,window", [([(100, 300)] * 5, 64, 0), ([(40, 513), (0, 260), (900, 255)] * 2, 128, 0),
                                                 ([(300, 700), (5, 90)] * 2, 80, 200), ([(7, 400)] * 3, 256, 0)])
def test_more_items_than_workgroups(requests, D, window):
    """Shares that begin and end within items, of chunks: the same bits every time, and what 64 bits give for the first and
    the last head."""
    heads = 32
    p = Problem(requests, heads, heads, D, 16, seed=30)
    out, lse = (t.clone() for t in p.run(window=window))
    for _ in range(4):
        again = p.run(window=window)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    ends = [0, heads - 1]
    k, v, q = (f64(t)[..., ends, :] for t in (p.dk, p.dv, p.dq))
    want = ref.attention(q, k, v, p.table, p.starts, p.lens, D ** -0.5, True, window)
    compare(f64(out)[:, ends], f64(lse)[:, ends], want, D)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_more_pages_than_are_at_hand(D):
    """Pages of one row: a part of an item has more of them than a wave keeps, some of them none."""
    p = Problem([(1500, 70), (700, 1)], 4, 2, D, 1, seed=31)
    p.check()
    for j in (300, 301, 511, 1040):
        p.table[0][j] = -1 if j % 2 else p.pages
    p.dtable = i32(p.table)
    p.check()


def test_many_requests():
    """More requests than a workgroup has threads, most of them short."""
    rng = np.random.default_rng(15)
    requests = [(int(rng.integers(0, 40)), int(rng.integers(0, 3))) for _ in range(700)]
    Problem(requests, 2, 1, 64, 16, seed=15).check(weights=2.0 ** -16)
    requests = [(int(rng.integers(0, 20)), int(rng.choice([0, 1, 40]))) for _ in range(300)]
    Problem(requests, 4, 1, 64, 16, seed=16).check(max_fresh=40)


def test_mixed_steps_split_between_the_kernels():
    p = Problem([(300, 1), (10, 90), (0, 16), (77, 17), (200, 1)], 8, 2, 128, 16, seed=17)
    p.check(max_fresh=90)


def test_positions_past_32_bits():
    """Caches of more than 2^32 bytes and 2^31 values each, of which only far pages are in use."""
    pages, page, Hkv, D = 70000, 64, 8, 64
    k, v = (torch.empty((pages, page, Hkv, D), dtype=BF16, device=DEV) for _ in range(2))
    assert k.numel() > 2 ** 31
    p = Problem([(150, 1), (20, 80)], 8, Hkv, D, page, seed=18)
    small_k, small_v = p.dk, p.dv
    far = [pages - 1 - 9 * i for i in range(p.pages)]
    for i, f in enumerate(far):
        k[f], v[f] = small_k[i], small_v[i]
    out, lse = (t.clone() for t in p.run())
    p.dk, p.dv = k, v
    p.dtable = i32([[far[x] if x >= 0 else -1 for x in r] for r in p.table])
    for max_fresh in (80, 1):
        o, l = p.run(max_fresh=max_fresh)
        if max_fresh == 80:
            assert torch.equal(o, out) and torch.equal(l, lse)
    # and rotary positions into far slots
    x = torch.randn(3, Hkv, D, device=DEV).to(BF16)
    slots = i32([pages * page - 1, pages * page - 70, 5])
    occ.occ_rope(None, x, i32([0, 0, 0]), occ.rope_turns(32), v=x, k_cache=k, v_cache=v, slots=slots)
    for s, r in zip(slots.tolist(), x):
        assert torch.equal(k[s // page, s % page], r) and torch.equal(v[s // page, s % page], r)


def test_streams_with_their_own_workspaces():
    a, b = Problem([(900, 1), (100, 1)], 8, 2, 64, 16, seed=19), Problem([(50, 100)], 4, 2, 64, 16, seed=20)
    want = a.run()[0].clone(), b.run()[0].clone()
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [workspace_for(64, fresh=True) for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(5):
        for p, s, w in zip((a, b), streams, spaces):
            with torch.cuda.stream(s):
                outs.append(p.run(workspace=w)[0])
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, want[i % 2])


def test_graph_serves_other_lengths():
    p = Problem([(300, 1), (50, 1), (0, 1)], 8, 2, 64, 16, seed=21)
    p.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        occ.occ_attn_paged(p.dq, p.dk, p.dv, p.dtable, p.dstarts, p.dlens, p.out, max_fresh=1, lse=p.lse, workspace=workspace_for(64))
    out, lse = p.out, p.lse
    for lens in ([301, 51, 1], [7, 0, 1], [160, 33, 1], [301, 51, 1]):
        p.lens = lens
        p.dlens.copy_(i32(lens))
        out.fill_(77.0), lse.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        compare(f64(out), f64(lse), p.want(), p.D, 2.0 ** -16)


def test_nothing_to_do():
    w = workspace_for(64)
    e = lambda *s: torch.empty(s, dtype=BF16, device=DEV)  # noqa: E731
    occ.occ_attn_paged(e(0, 2, 64), e(3, 16, 1, 64), e(3, 16, 1, 64), i32([[0, 1]]), i32([0, 0]), i32([5]), e(0, 2, 64), max_fresh=0, workspace=w)
    out = torch.full((2, 2, 64), 7.0, dtype=BF16, device=DEV)
    none = torch.empty((0, 4), dtype=torch.int32, device=DEV)
    occ.occ_attn_paged(e(2, 2, 64), e(3, 16, 1, 64), e(3, 16, 1, 64), none, i32([0]), none[:, 0].contiguous(), out, max_fresh=1, workspace=w)
    assert bool((out == 7).all())
