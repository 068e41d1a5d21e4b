"""Arguments of the paged cache's C ABI whose checks must not pass 32 bits: refused before the GPU is touched (placeholder
pointers)."""
import pytest

from test_abi_cpu import expect_accepted
from test_abi_paged_cpu import EINVAL, L, attn, rope  # noqa: F401

MOST = 2 ** 31 - 1


# 2 * 2^30 is 0 in the bits of an int that are left
@pytest.mark.parametrize("pairs", [1 << 30, (1 << 30) + 1, (1 << 30) + 32, MOST])
def test_more_pairs_than_half_a_head(L, pairs):  # noqa: F811
    assert L.occ_rope(rope(pairs=pairs), None) == EINVAL


# (rows + requests) * width * page * Hq: 2^51 and more, with a sum of rows and requests past 2^31
@pytest.mark.parametrize("rows,requests", [(1 << 20, 65536), (MOST, 65536), (MOST, 1), (MOST - 65535, 65536)])
def test_more_work_than_units_count(L, rows, requests):  # noqa: F811
    one = dict(Hq=1, Hkv=1, D=64, q_row=64, out_row=64, page=65536, pages=100, cache_row=64, cache_page=64 * 65536, width=1 << 15, ld_table=1 << 15)
    # tensors of as many rows are further apart than the default places
    far = {n: (i + 1) << 44 for i, n in enumerate(("q", "k_cache", "v_cache", "table", "starts", "lens", "out", "lse", "workspace"))}
    assert L.occ_attn_paged(attn(rows=rows, requests=requests, **one, **far), None) == EINVAL


# times log2 e it has to stay a number
@pytest.mark.parametrize("scale,status", [(2.0 ** 127 * 1.5, EINVAL), (3.4028234e38, EINVAL), (2.0 ** 127, None), (2.0 ** -149, None)])
def test_scales(L, scale, status):  # noqa: F811
    if status is None:
        expect_accepted(L, L.occ_attn_paged, attn(scale=scale), None)
    else:
        assert L.occ_attn_paged(attn(scale=scale), None) == status
