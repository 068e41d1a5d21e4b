"""CPU checks of the paged cache's C ABI: bad arguments are refused with the documented status before the GPU is touched
(placeholder pointers; calls that pass validation are made only where no device is visible)."""
import ctypes

import pytest
import torch

from paper_2606_09200_amd import binding as occ
from test_abi_cpu import expect_accepted

EINVAL, EALIAS = occ.OCC_EINVAL, occ.OCC_EALIAS


@pytest.fixture(scope="module")
def L():
    return occ.lib()


def place(i):
    return 0x100000000 * i


def tables(**k):
    a = occ.occ_kv_tables_args(requests=4, rows=10, width=8, page=16, pages=40, ring_size=40, ld_table=8)
    for i, n in enumerate(("cached", "fresh", "free", "table", "ring", "lens", "starts", "slots", "positions", "free_after")):
        setattr(a, n, place(i + 1))
    for n, v in k.items():
        setattr(a, n, v)
    return ctypes.byref(a)


def rope(**k):
    a = occ.occ_rope_args(rows=6, Hq=8, Hkv=2, D=64, pairs=32, dtype=0, page=16, pages=10, scale=1.0, q_row=512, q_head=64, k_row=128,
                          k_head=64, v_row=128, v_head=64, qo_row=512, qo_head=64, ko_row=128, ko_head=64, cache_page=2048,
                          cache_row=128, cache_head=64)
    for i, n in enumerate(("q", "k", "v", "q_out", "k_out", "k_cache", "v_cache", "positions", "slots", "turns")):
        setattr(a, n, place(i + 1))
    for n, v in k.items():
        setattr(a, n, v)
    return ctypes.byref(a)


def attn(**k):
    a = occ.occ_attn_args(requests=4, rows=6, Hq=8, Hkv=2, D=64, page=16, pages=10, width=5, max_fresh=2, causal=1, scale=0.125,
                          ld_table=5, q_row=512, q_head=64, out_row=512, out_head=64, cache_page=2048, cache_row=128,
                          cache_head=64, workspace_bytes=occ.occ_attn_paged_workspace_bytes(8, 2, 64))
    for i, n in enumerate(("q", "k_cache", "v_cache", "table", "starts", "lens", "out", "lse", "workspace")):
        setattr(a, n, place(i + 1))
    for n, v in k.items():
        setattr(a, n, v)
    return ctypes.byref(a)


@pytest.mark.parametrize("status,change", [
    (EINVAL, dict(requests=-1)), (EINVAL, dict(requests=65537)), (EINVAL, dict(rows=-1)), (EINVAL, dict(rows=(1 << 24) + 1)),
    (EINVAL, dict(width=-1)), (EINVAL, dict(page=0)), (EINVAL, dict(page=65537)), (EINVAL, dict(pages=-1)), (EINVAL, dict(ring_size=0)),
    (EINVAL, dict(pages=1 << 27)), (EINVAL, dict(ring_size=(1 << 30) + 1)), (EINVAL, dict(ld_table=7)), (EINVAL, dict(cached=None)),
    (EINVAL, dict(fresh=place(2) + 2)), (EINVAL, dict(free=None)), (EINVAL, dict(table=None)), (EINVAL, dict(ring=None)),
    (EINVAL, dict(lens=None)), (EINVAL, dict(starts=None)), (EINVAL, dict(slots=None)), (EINVAL, dict(positions=place(9) + 1)),
    (EINVAL, dict(free_after=None)), (EINVAL, dict(requests=0, free=None)), (EINVAL, dict(requests=0, starts=None)), (EALIAS, dict(lens=place(1))), (EALIAS, dict(free_after=place(3))), (EALIAS, dict(ring=place(4) + 64)),
    (EALIAS, dict(starts=place(6) + 12)), (EALIAS, dict(slots=place(9))), (EALIAS, dict(table=place(2) - 100)),
])
def test_tables_refusals(L, status, change):
    assert L.occ_kv_tables(tables(**change), None) == status


def test_tables_accepts(L):
    assert L.occ_kv_tables(None, None) == EINVAL
    for k in (dict(), dict(requests=0, cached=None, fresh=None, lens=None, table=None), dict(rows=0, slots=None, positions=None), dict(width=0, table=None),
              dict(requests=1, ld_table=0), dict(pages=0)):
        expect_accepted(L, L.occ_kv_tables, tables(**k), None)


@pytest.mark.parametrize("status,change", [
    (EINVAL, dict(dtype=2)), (EINVAL, dict(rows=-1)), (EINVAL, dict(rows=(1 << 24) + 1)), (EINVAL, dict(Hq=-1)), (EINVAL, dict(Hkv=-1)),
    (EINVAL, dict(D=63)), (EINVAL, dict(D=0)), (EINVAL, dict(D=1026)), (EINVAL, dict(pairs=33)), (EINVAL, dict(pairs=-1)),
    (EINVAL, dict(scale=float("inf"))), (EINVAL, dict(scale=float("nan"))), (EINVAL, dict(v_cache=None)), (EINVAL, dict(k_cache=None)),
    (EINVAL, dict(positions=None)), (EINVAL, dict(turns=None)), (EINVAL, dict(turns=place(10) + 4)), (EINVAL, dict(q_out=None)),
    (EINVAL, dict(k_out=None, k_cache=None, v_cache=None)), (EINVAL, dict(k=None)), (EINVAL, dict(v=None)), (EINVAL, dict(slots=None)),
    (EINVAL, dict(q=place(1) + 1)), (EINVAL, dict(slots=place(9) + 2)), (EINVAL, dict(q_row=511)), (EINVAL, dict(k_head=63)),
    (EINVAL, dict(qo_row=64)), (EINVAL, dict(page=0)), (EINVAL, dict(pages=0)), (EINVAL, dict(pages=1 << 27)),
    (EINVAL, dict(cache_page=2047)), (EINVAL, dict(cache_row=127)), (EINVAL, dict(v_row=0)),
    (EALIAS, dict(q_out=place(1) + 128)), (EALIAS, dict(q_out=place(2))), (EALIAS, dict(k_out=place(4))), (EALIAS, dict(k_cache=place(7))),
    (EALIAS, dict(k_cache=place(8))), (EALIAS, dict(v_cache=place(3))), (EALIAS, dict(q_out=place(6))), (EALIAS, dict(q_out=place(9))),
    (EALIAS, dict(q_out=place(1), qo_row=520)),
])
def test_rope_refusals(L, status, change):
    assert L.occ_rope(rope(**change), None) == status


def test_rope_accepts(L):
    assert L.occ_rope(None, None) == EINVAL
    joint = dict(q=place(1), k=place(1) + 1024, v=place(1) + 1280, q_row=768, k_row=768, v_row=768)
    for k in (dict(), dict(rows=0, positions=None), dict(q_out=place(1)), dict(k_out=place(2)), dict(k_out=None), dict(pairs=0, turns=None),
              dict(q=None, q_out=None), dict(k=None, k_out=None, k_cache=None, v_cache=None), dict(v=None, k_cache=None, v_cache=None, slots=None),
              dict(q_out=place(1), qo_row=768, k_out=place(1) + 1024, ko_row=768, **joint), joint,
              # planes of one cache, and heads outermost in a page
              dict(v_cache=place(6) + 4096, cache_page=4096), dict(cache_head=1024, cache_row=64), dict(scale=0.0), dict(dtype=1)):
        expect_accepted(L, L.occ_rope, rope(**k), None)


@pytest.mark.parametrize("status,change", [
    (EINVAL, dict(requests=-1)), (EINVAL, dict(requests=65537)), (EINVAL, dict(rows=-1)), (EINVAL, dict(rows=1 << 28)), (EINVAL, dict(Hq=9)),
    (EINVAL, dict(Hkv=0)), (EINVAL, dict(Hq=1)), (EINVAL, dict(D=60)), (EINVAL, dict(D=264)), (EINVAL, dict(D=0)), (EINVAL, dict(page=0)),
    (EINVAL, dict(pages=0)), (EINVAL, dict(pages=1 << 27)), (EINVAL, dict(width=-1)), (EINVAL, dict(max_fresh=-1)), (EINVAL, dict(window=-1)),
    (EINVAL, dict(scale=0.0)), (EINVAL, dict(scale=-1.0)), (EINVAL, dict(scale=float("inf"))), (EINVAL, dict(scale=float("nan"))),
    (EINVAL, dict(q=None)), (EINVAL, dict(q=place(1) + 8)), (EINVAL, dict(out=place(7) + 2)), (EINVAL, dict(k_cache=None)),
    (EINVAL, dict(v_cache=None)), (EINVAL, dict(table=None)), (EINVAL, dict(starts=None)), (EINVAL, dict(lens=place(6) + 2)),
    (EINVAL, dict(lse=place(8) + 2)), (EINVAL, dict(workspace=None)), (EINVAL, dict(workspace_bytes=4096)), (EINVAL, dict(q_row=516)),
    (EINVAL, dict(q_head=68)), (EINVAL, dict(out_row=64)), (EINVAL, dict(cache_row=64)), (EINVAL, dict(cache_page=1024)),
    (EINVAL, dict(cache_page=1 << 31)), (EINVAL, dict(cache_row=1 << 31, cache_page=1 << 36)), (EINVAL, dict(width=1 << 30, ld_table=1 << 30,
                                                                                                     page=65536, pages=5, cache_page=1 << 23, rows=1 << 10)),
    (EINVAL, dict(ld_table=4)), (EALIAS, dict(out=place(1))), (EALIAS, dict(lse=place(7))), (EALIAS, dict(out=place(2) + 64)),
    (EALIAS, dict(workspace=place(3))), (EALIAS, dict(lse=place(5))), (EALIAS, dict(out=place(9) + 4096)),
])
def test_attention_refusals(L, status, change):
    assert L.occ_attn_paged(attn(**change), None) == status


def test_attention_accepts(L):
    assert L.occ_attn_paged(None, None) == EINVAL
    for k in (dict(), dict(requests=0, starts=None), dict(rows=0, q=None, out=None, pages=0), dict(width=0, table=None), dict(lse=None),
              dict(v_cache=place(2) + 4096, cache_page=4096), dict(cache_head=1024, cache_row=64), dict(max_fresh=0), dict(window=1 << 30),
              dict(causal=0)):
        expect_accepted(L, L.occ_attn_paged, attn(**k), None)


def test_workspace_bytes():
    f = occ.occ_attn_paged_workspace_bytes
    assert f(8, 3, 64) == f(8, 0, 64) == f(2, 8, 64) == f(8, 2, 60) == f(8, 2, 264) == 0
    assert f(8, 2, 8) == f(64, 1, 64) > 0 and f(8, 8, 72) == f(8, 8, 128) > f(8, 8, 64)


def test_binding_refuses_before_the_library():
    i32, i64, bf = (lambda *s: torch.zeros(s, dtype=torch.int32)), (lambda *s: torch.zeros(s, dtype=torch.int64)), (
        lambda *s: torch.zeros(s, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="table"):
        occ.occ_kv_tables(i32(2), i32(2), i32(2, 3), i32(4), i32(2), page=16, pages=4, lens=i32(2), starts=i32(3), slots=i32(5),
                          positions=i32(5), free_after=i32(2))
    with pytest.raises(ValueError, match="q or k"):
        occ.occ_rope(None, None, i32(3), i64(4))
    with pytest.raises(ValueError, match="GPU tensor"):
        occ.occ_rope(bf(3, 2, 16), None, i32(3), i64(4))
    with pytest.raises(ValueError, match="three|rows, heads, D"):
        occ.occ_rope(bf(3, 2), None, i32(3), i64(4))
    with pytest.raises(ValueError, match="GPU tensor"):
        occ.occ_attn_paged(bf(3, 2, 16), bf(2, 4, 1, 16), bf(2, 4, 1, 16), i32(1, 2), i32(2), i32(1), bf(3, 2, 16), max_fresh=1,
                           workspace=i32(4))
    with pytest.raises(ValueError, match="rows, heads, D"):
        occ.occ_attn_paged(bf(3, 16), bf(2, 4, 1, 16), bf(2, 4, 1, 16), i32(1, 2), i32(2), i32(1), bf(3, 16), max_fresh=1, workspace=i32(4))


def test_frequencies():
    """The table against its formulas in Python's whole numbers and 64 bits: an entry is cut to a whole number of 2^-64
    turns, so it is off by less than one of them beside the 64-bit arithmetic's roundings."""
    import math
    t = occ.rope_turns(8, base=500000.0, device="cpu").tolist()
    for i, v in enumerate(t):
        want = 500000.0 ** (-i / 8) / (2 * math.pi)
        assert v >= 0 and abs(v / 2.0 ** 64 - want) <= 2.0 ** -52 * want + 2.0 ** -64
    assert occ.rope_turns(8, linear=4.0, device="cpu").tolist()[3] == occ.rope_turns(8, device="cpu").tolist()[3] // 4  # a power of two
    plain, banded = occ.rope_turns(32, device="cpu").tolist(), occ.rope_turns(32, bands=(8.0, 1.0, 4.0, 8192), device="cpu").tolist()
    for a, b in zip(plain, banded):
        turns = a / 2.0 ** 64 * 8192
        keep = min(1.0, max(0.0, (turns - 1.0) / 3.0))
        assert abs(b - a * (keep + (1 - keep) / 8)) <= 2.0 ** -50 * a + 2
    assert banded[0] == plain[0] and abs(banded[-1] - plain[-1] / 8) <= 2.0 ** -50 * plain[-1] + 2
    assert occ.rope_turns(1, base=1.0, linear=1 / 7.0, device="cpu").tolist()[0] < 2 ** 63   # more than a turn a position: its fraction
    assert occ.rope_turns(0, device="cpu").numel() == 0
