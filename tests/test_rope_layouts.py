"""occ_rope where q, k and v, or the two caches, lie among each other in one buffer: taken where no value is another's, in place too,
and refused where some are."""
import pytest
import torch

from paper_2606_09200_amd import binding as occ
from test_abi_cpu import expect_accepted
from test_abi_paged_cpu import EALIAS, L, place, rope  # noqa: F401

# 4 heads of 64 each of q, k and v, in rows that hold q, k, v of a head side by side, in rows of heads outermost, and of other pitches
JOINT = dict(Hq=4, Hkv=4, q=place(1), q_out=place(1), k_out=None)
A_HEAD = dict(JOINT, k=place(1) + 128, v=place(1) + 256, q_row=768, k_row=768, v_row=768, qo_row=768, q_head=192, k_head=192, v_head=192, qo_head=192,
              cache_page=4096, cache_row=256)
OUTER = dict(JOINT, k=place(1) + 128, v=place(1) + 256, q_row=192, k_row=192, v_row=192, qo_row=192, q_head=1152, k_head=1152, v_head=1152,
             qo_head=1152, cache_page=4096, cache_row=256)
# (keys and values of a row, of a head, of a head's rows side by side)
CACHE = dict(k_cache=place(6))
BY_ROW = dict(CACHE, v_cache=place(6) + 256, cache_row=256, cache_page=4096)
BY_HEAD = dict(CACHE, v_cache=place(6) + 128, cache_head=128, cache_row=256, cache_page=4096)
BY_HEADS_ROWS = dict(CACHE, v_cache=place(6) + 2 * 16 * 64, cache_row=64, cache_head=2048, cache_page=4096)


@pytest.mark.parametrize("change", [
    A_HEAD, OUTER, dict(A_HEAD, rows=1), dict(OUTER, rows=1), dict(A_HEAD, k_out=place(1) + 128, ko_row=768, ko_head=192), BY_ROW, BY_HEAD, BY_HEADS_ROWS,
    dict(BY_ROW, pages=1), dict(BY_HEAD, pages=1), dict(BY_HEADS_ROWS, pages=1), dict(BY_ROW, k_cache=place(6) + 256, v_cache=place(6))])
def test_taken(L, change):  # noqa: F811
    expect_accepted(L, L.occ_rope, rope(**change), None)


@pytest.mark.parametrize("change", [
    # half a head further; a pitch that is no multiple; a row or a head of which some is another's
    dict(A_HEAD, k=place(1) + 64), dict(A_HEAD, q_row=800, qo_row=800), dict(A_HEAD, k=place(1) + 128 * 3), dict(OUTER, k=place(1) + 384), dict(A_HEAD, rows=1, v=place(1) + 64),
    dict(A_HEAD, k_head=256, k_row=1024), dict(BY_ROW, v_cache=place(6) + 128), dict(BY_HEAD, v_cache=place(6) + 64), dict(BY_HEADS_ROWS, v_cache=place(6) + 1024),
    dict(BY_ROW, v_cache=place(6) + 512), dict(BY_HEAD, cache_row=264, cache_page=16 * 264), dict(CACHE, v_cache=place(6))])
def test_refused(L, change):  # noqa: F811
    assert L.occ_rope(rope(**change), None) == EALIAS


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 37])
@pytest.mark.parametrize("form", ["head", "outer"])
@pytest.mark.parametrize("cache", ["row", "head", "heads_rows"])
def test_in_place(rows, form, cache):
    from gpu_common import DEV
    H, D, page = 4, 64, 16
    pages = rows // page + 2
    g = torch.Generator().manual_seed(1)

    def rand(*shape):
        return torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)

    joint = rand(rows, H, 3, D) if form == "head" else rand(H, rows, 3, D).transpose(0, 1)
    q, k, v = joint.unbind(2)
    both = {"row": lambda: rand(pages, page, 2, H, D).unbind(2), "head": lambda: rand(pages, page, H, 2, D).unbind(3),
            "heads_rows": lambda: rand(pages, H, 2, page, D).transpose(2, 3).transpose(1, 2).unbind(3)}[cache]()
    keys, values = both
    assert keys.shape == (pages, page, H, D)
    pos, turns = torch.arange(rows, dtype=torch.int32, device=DEV) * 5, occ.rope_turns(32)
    slots = torch.randperm(pages * page, generator=g)[:rows].to(torch.int32).to(DEV)
    apart = [t.contiguous().clone() for t in (q, k, v, keys, values)]
    occ.occ_rope(apart[0], apart[1], pos, turns, v=apart[2], k_cache=apart[3], v_cache=apart[4], slots=slots)
    occ.occ_rope(q, k, pos, turns, v=v, k_cache=keys, v_cache=values, slots=slots)
    for a, b in zip((q, k, v, keys, values), apart):
        assert torch.equal(a, b)
    occ.occ_rope(q, k, pos, turns)
    occ.occ_rope(apart[0], apart[1], pos, turns)
    for a, b in zip((q, k, v), apart):
        assert torch.equal(a, b)
