"""The choice of occ_gemm_mx4's kernel, on a GPU of 256 compute units (CPU: the choice needs no device)."""
import re

import pytest

import test_gpu_mx4_tiles as tiles
from paper_2606_09200_amd import binding as occ


def plan(M, N, K, num_cus=256):
    return occ.occ_gemm_mx4_plan_query(M, N, K, num_cus)


@pytest.mark.parametrize("tile,M,N,K", tiles.CASES)
def test_tested_shapes_take_the_kernel_they_are_listed_for(tile, M, N, K):
    p = plan(M, N, K)
    assert (p["tile_m"], p["tile_n"]) == tile
    assert p["tiles"] == -(-M // tile[0]) * -(-N // tile[1]) and 0 < p["grid"] <= p["tiles"]


def test_every_kernel_is_tested():
    source = open(occ.__file__.replace("binding.py", "csrc/gemm_mx4.hip")).read()
    table = source[source.index("const Mx4Tile kTiles[]"):source.index("constexpr int kMaxDevices")]
    names = re.findall(r"tile_of<(\w+)>", table)
    known = {"Mx4Pp": (256, 256)}
    known.update({n: tuple(map(int, re.findall(r"\d+", n))) for n in names if n != "Mx4Pp"})
    assert set(tiles.SHAPES) == {known[n] for n in names} | {(16, 16), (16, 32)}
    # both layouts of K a tile knows: an odd number of k-steps of 256 and an even one; whole and half steps of 512
    for tile, shapes in tiles.SHAPES.items():
        steps = {-(-K // 256) % 2 for _, _, K in shapes}
        assert steps == {0, 1} or tile == (16, 32), tile
    assert {plan(*s)["nontemporal"] for s in tiles.SHAPES[16, 16]} == {0, 1}


def test_plan_of_odd_calls():
    assert plan(0, 5, 64) == plan(5, 0, 64) == dict(tile_m=0, tile_n=0, tiles=0, grid=0, nontemporal=0)
    assert plan(16, 40, 0)["tile_m"] == 16 and plan(17, 40, 0)["tile_m"] == 32
    for bad in ((-1, 5, 64), (5, 5, (1 << 23) + 1), (1 << 23, 1 << 23, 64)):
        with pytest.raises(occ.OccError) as e:
            plan(*bad)
        assert e.value.status == occ.OCC_EINVAL
    with pytest.raises(occ.OccError):
        plan(5, 5, 64, -1)


def test_a_workgroup_has_one_tile():
    """The tiled kernels have no loop over tiles."""
    for tile, M, N, K in tiles.CASES:
        p = plan(M, N, K)
        assert p["grid"] == p["tiles"] or tile == (16, 16)


def test_plan_names_the_loads_that_are_made():
    """Short rows are read through the caches, whatever their number."""
    assert plan(16, 40000, 2048)["nontemporal"] == 0 and plan(16, 40000, 2049)["nontemporal"] == 1
    assert plan(16, 40000, 8193)["nontemporal"] == 0
