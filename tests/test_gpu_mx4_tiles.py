"""occ_gemm_mx4's kernels, each by shapes that the choice sends to it, against a 64-bit product.

The shapes end inside tiles in both dimensions, with odd and even numbers of k-steps (of 256 and of 512) and one to
many of them; test_mx4_tiles_cpu.py holds the choice to this table.  Operands are packed here from include/occ.h's
layout, the reference is a matrix product in float64."""
import pytest
import torch

from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu

# tile of C -> (M, N, K)
SHAPES = {
    (256, 256): [(3380, 2485, 519), (2525, 3437, 759), (2459, 3283, 1000), (2459, 3283, 2200), (5367, 1912, 2745),
                 (385, 16714, 727)],
    (128, 128): [(131, 8265, 35), (1235, 1653, 725), (1415, 1437, 1290), (1810, 1109, 2121)],
    (128, 64): [(5513, 131, 35), (69, 8233, 45), (1475, 687, 713), (871, 1252, 2139), (871, 1252, 2500), (795, 1247, 3600), (8323, 77, 1600)],
    (64, 64): [(4425, 69, 33), (4467, 66, 600), (577, 962, 2157), (1037, 468, 3500), (42, 11296, 6372)],
    (32, 64): [(17, 19, 32), (33, 200, 1500), (64, 1000, 1030), (100, 333, 9000)],
    # M <= 16: one to two k-steps a wave, then, beyond K = 8192, as many as there are
    (16, 16): [(1, 40, 600), (16, 300, 1024), (5, 77, 2100), (11, 33, 8192), (16, 8209, 8192), (3, 16401, 4000)],
    (16, 32): [(1, 77, 8193), (5, 77, 20000), (16, 77, 8193), (16, 133, 20000), (9, 1000, 12345)],
}
CASES = [(tile, *s) for tile, shapes in SHAPES.items() for s in shapes]
ONE_EACH = [(tile, *shapes[1]) for tile, shapes in SHAPES.items()]


def operand(rows, cols, seed, low=119, high=134):
    """Random codes and scale bytes of [low, high] in the library's layout, and their values in float64."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    kp, rp = (cols + 511) // 512 * 512, (rows + 15) // 16 * 16
    codes = torch.zeros((rows, kp), dtype=torch.uint8, device=DEV)
    codes[:, :cols] = torch.randint(16, (rows, cols), generator=g, device=DEV, dtype=torch.uint8)
    blocks = (cols + 31) // 32
    scales = torch.zeros((rp, kp // 32), dtype=torch.uint8, device=DEV)
    scales[:rows, :blocks] = torch.randint(low, high + 1, (rows, blocks), generator=g, device=DEV, dtype=torch.uint8)
    return pack(codes, scales, rows, cols), values(codes, scales, rows, cols)


def pack(codes, scales, rows, cols):
    # block (4 s + j) 4 + g of row 16 t + r is byte j of word 16 g + r of tile (t, s)
    t, s = scales.shape[0] // 16, scales.shape[1] // 16
    laid = scales.view(t, 16, s, 4, 4).permute(0, 2, 4, 1, 3).reshape(t, s * 256).contiguous()
    return occ.Mx4((codes[:, 0::2] | codes[:, 1::2] << 4).contiguous(), laid, rows, cols)


def values(codes, scales, rows, cols):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    v = grid[(codes & 7).long()] * torch.where(codes > 7, -1.0, 1.0)
    return (v.view(rows, -1, 32) * torch.exp2(scales[:rows].double() - 127)[:, :, None]).view(rows, -1)[:, :cols].contiguous()


def guarded(M, N, dtype):
    """A NaN-filled (M, N) tensor between 4096 values that nothing may write."""
    flat = torch.full((M * N + 8192,), float("nan"), dtype=dtype, device=DEV)
    flat[:4096] = flat[-4096:] = 7
    return flat[4096:4096 + M * N].view(M, N), flat


def check(C, flat, a, b, dtype):
    """Products of two 4-bit values are exact in binary32; each of the K additions rounds (or truncates) by at most
    2^-23 of the sum of magnitudes, and bf16 outputs by 2^-8 more."""
    want = a @ b.t()
    tol = a.shape[1] * 2.0 ** -23 * (a.abs() @ b.abs().t()) + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0.0)
    err = (C.double() - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), (~(err <= tol)).nonzero()[:4].tolist())
    assert bool((flat[:4096] == 7).all()) and bool((flat[-4096:] == 7).all())


def tile_of(M, N, K):
    p = occ.occ_gemm_mx4_plan_query(M, N, K)
    return p["tile_m"], p["tile_n"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tile,M,N,K", CASES)
def test_product(tile, M, N, K, dtype):
    assert tile_of(M, N, K) == tile
    (A, a), (B, b) = operand(M, K, M + K), operand(N, K, N + K + 1)
    C, flat = guarded(M, N, dtype)
    occ.occ_gemm_mx4(A, B, C)
    check(C, flat, a, b, dtype)


@pytest.mark.parametrize("tile,M,N,K", ONE_EACH)
def test_scales_far_apart(tile, M, N, K):
    """A's near 2^-110 and B's near 2^110: the products are of ordinary size and exact all the same."""
    (A, a), (B, b) = operand(M, K, 1, 7, 27), operand(N, K, 2, 227, 247)
    C, flat = guarded(M, N, torch.float32)
    occ.occ_gemm_mx4(A, B, C)
    check(C, flat, a, b, torch.float32)


@pytest.mark.parametrize("tile,M,N,K", ONE_EACH)
def test_nan_scales_stay_in_their_row_and_column(tile, M, N, K):
    (A, _), (B, _) = operand(M, K, 3), operand(N, K, 4)
    row, col, block = M // 2, N - 1, (K - 1) // 32   # the last block of both
    at = block // 16 * 256 + 4 * (16 * (block % 4)) + block % 16 // 4
    A.scales[row // 16, at + 4 * (row % 16)] = 255
    B.scales[col // 16, at + 4 * (col % 16)] = 255
    C, _ = guarded(M, N, torch.float32)
    C.zero_()
    occ.occ_gemm_mx4(A, B, C)
    bad = torch.isnan(C)
    assert bool(bad[row].all()) and bool(bad[:, col].all())
    bad[row], bad[:, col] = False, False
    assert not bool(bad.any())


@pytest.mark.parametrize("tile,M,N,K", ONE_EACH)
def test_repeat_and_pad_give_the_same_bits(tile, M, N, K):
    (A, _), (B, _) = operand(M, K, 5), operand(N, K, 6)
    C = occ.occ_gemm_mx4(A, B, torch.empty((M, N), device=DEV))
    assert torch.equal(occ.occ_gemm_mx4(A, B, torch.empty((M, N), device=DEV)), C)
    # the 128 x 64 tile leaves 4 KiB of a workgroup's LDS
    assert torch.equal(occ.occ_gemm_mx4(A, B, torch.empty((M, N), device=DEV), lds_bytes=4096), C)
