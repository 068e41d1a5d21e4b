"""occ_mx4_quantize, occ_mx4_dequantize and occ_gemm_mx4 against plain 64-bit implementations."""
import numpy as np
import pytest
import torch

import block_reference as ref
from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu


def draw(rows, cols, dtype, seed, spread=6.0):
    """Normal values whose blocks differ in scale by powers of two, some of them on ties of the grid."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, dtype=torch.float64)
    x *= torch.exp2(torch.round(spread * torch.randn((rows, 1), generator=g, dtype=torch.float64)))
    x[:, ::7] = torch.round(x[:, ::7] * 4) / 4
    return x.to(dtype)


def unpack(q):
    return ref.mx4_unpack(q.codes.cpu().numpy(), q.scales.cpu().numpy(), q.rows, q.cols)


def check_quantized(x, q):
    codes, scales, pads = unpack(q)
    want_c, want_s = ref.mx4_quantize(ref.f64(x))
    assert np.array_equal(scales, want_s)
    assert np.array_equal(codes, want_c)
    assert all((p == 0).all() for p in pads)


def filled(rows, cols):
    q = occ.mx4_empty(rows, cols, device=DEV)
    q.codes.fill_(0xA5)
    q.scales.fill_(0xA5)
    return q


SHAPES = [(1, 1), (1, 32), (3, 31), (16, 512), (17, 513), (33, 40), (130, 129), (5, 1100), (600, 70)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_both_orientations(rows, cols, dtype):
    x = draw(rows, cols, dtype, seed=rows + cols).to(DEV)
    q, qt = filled(rows, cols), filled(cols, rows)
    occ.occ_mx4_quantize(x, q, qt)
    check_quantized(x, q)
    check_quantized(x.t(), qt)
    alone, alone_t = filled(rows, cols), filled(cols, rows)
    occ.occ_mx4_quantize(x, alone)
    occ.occ_mx4_quantize(x, None, alone_t)
    assert torch.equal(alone.codes, q.codes) and torch.equal(alone.scales, q.scales)
    assert torch.equal(alone_t.codes, qt.codes) and torch.equal(alone_t.scales, qt.scales)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_quantize_strided_rows_at_any_alignment(dtype, offset):
    """Rows of a wider buffer, at any element: what lies between them is not read into a block."""
    rows, cols, ld = 37, 200, 331
    wide = torch.full((rows * ld + 8,), float("nan"), dtype=dtype, device=DEV)
    x = wide[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    x.copy_(draw(rows, cols, dtype, seed=9))
    q, qt = filled(rows, cols), filled(cols, rows)
    occ.occ_mx4_quantize(x, q, qt)
    check_quantized(x, q)
    check_quantized(x.t(), qt)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_extremes(dtype):
    """Zeros of both signs, subnormals, the largest values, ties, and blocks that hold an infinity or a NaN."""
    big = float(torch.finfo(dtype).max)
    x = torch.zeros((40, 96), dtype=torch.float64)
    x[0, :] = -0.0
    x[1, 0], x[2, 40] = float(torch.finfo(dtype).tiny), -float(torch.finfo(dtype).tiny) / 2
    x[3, :32] = big
    x[4, 5], x[4, 6] = -big, big / 16
    x[5, :16] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 4.0, 0.2499, 0.7501, 6.0, 7.0, 7.96875, -0.25, -5.0, -7.0])
    x[6, 33], x[7, 64], x[8, 0] = float("inf"), float("-inf"), float("nan")
    x[9, :] = 2.0 ** -130
    x[10, 31] = 2.0 ** -126
    x = x.to(dtype).to(DEV)
    q, qt = filled(40, 96), filled(96, 40)
    occ.occ_mx4_quantize(x, q, qt)
    check_quantized(x, q)
    check_quantized(x.t(), qt)
    for p, y in ((q, x), (qt, x.t())):
        codes, scales, _ = unpack(p)
        for kind in (torch.bfloat16, torch.float32):
            out = torch.empty(tuple(y.shape), dtype=kind, device=DEV)
            assert np.array_equal(ref.f64(occ.occ_mx4_dequantize(p, out)), ref.mx4_values(codes, scales), equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_dequantize_every_code(rows, cols, dtype):
    rng = np.random.default_rng(rows * cols)
    codes = rng.integers(0, 16, (rows, cols), dtype=np.uint8)
    scales = rng.integers(0, 250, (rows, (cols + 31) // 32), dtype=np.uint8)
    c, s = ref.mx4_pack(codes, scales)
    q = occ.Mx4(torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV), rows, cols)
    wide = torch.full((rows, cols + 3), 7.0, dtype=dtype, device=DEV)
    occ.occ_mx4_dequantize(q, wide[:, 1:1 + cols])
    assert np.array_equal(ref.f64(wide[:, 1:1 + cols]), ref.mx4_values(codes, scales))
    assert (wide[:, 0] == 7).all() and (wide[:, 1 + cols:] == 7).all()


def operand(rows, cols, seed):
    """Random codes and scales within 2^-8 .. 2^7, packed, and their values."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (rows, cols), dtype=np.uint8)
    scales = rng.integers(119, 135, (rows, (cols + 31) // 32), dtype=np.uint8)
    c, s = ref.mx4_pack(codes, scales)
    return (occ.Mx4(torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV), rows, cols),
            ref.mx4_values(codes, scales))


def check_product(C, a, b, dtype):
    """Products of two 4-bit values are exact in binary32; each of the K additions rounds (or truncates) by at most
    2^-23 of the sum of magnitudes, and bf16 outputs by 2^-8 more."""
    want, mags = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = a.shape[1] * 2.0 ** -23 * mags + (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0)
    err = np.abs(ref.f64(C) - want)
    assert (err <= tol).all(), (float(err.max()), np.argwhere(err > tol)[:4].tolist())


# one row to many tiles, ragged in each dimension; K of one block to several k-steps (each kernel: test_gpu_mx4_tiles.py)
PRODUCTS = [(1, 1, 1), (1, 40, 600), (3, 17, 32), (16, 33, 5000), (16, 300, 1024), (5, 8200, 2100), (2, 9001, 512),
            (17, 64, 512), (40, 70, 2000), (64, 1000, 1030), (130, 260, 257), (300, 513, 1537), (257, 100, 4100),
            (1025, 2050, 700), (2100, 2310, 300)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_gemm(M, N, K, dtype):
    A, a = operand(M, K, M + K)
    B, b = operand(N, K, N + K + 1)
    C = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    occ.occ_gemm_mx4(A, B, C)
    check_product(C, a, b, dtype)


def test_gemm_empty_and_zero_inner():
    A, B = occ.mx4_empty(5, 0, device=DEV), occ.mx4_empty(7, 0, device=DEV)
    C = torch.full((5, 7), float("nan"), device=DEV)
    assert (occ.occ_gemm_mx4(A, B, C) == 0).all()
    C = torch.full((40, 70), float("nan"), device=DEV)
    assert (occ.occ_gemm_mx4(occ.mx4_empty(40, 0, device=DEV), occ.mx4_empty(70, 0, device=DEV), C) == 0).all()
    assert occ.occ_gemm_mx4(occ.mx4_empty(0, 64, device=DEV), occ.mx4_empty(7, 64, device=DEV),
                            torch.empty((0, 7), device=DEV)).numel() == 0


@pytest.mark.parametrize("M", [3, 70, 300])
def test_gemm_nan_scales_stay_in_their_rows(M):
    """A NaN block makes its row's outputs NaN and no others."""
    N, K = 90, 1200
    A, a = operand(M, K, 3)
    B, b = operand(N, K, 4)
    x = torch.from_numpy(a).float()
    x[M - 2, 700] = float("inf")
    A = occ.mx4_empty(M, K, device=DEV)
    occ.occ_mx4_quantize(x.to(DEV), A)
    C = torch.zeros((M, N), device=DEV)
    occ.occ_gemm_mx4(A, B, C)
    bad = torch.isnan(C).cpu()
    assert bad[M - 2].all() and not bad[:M - 2].any() and not bad[M - 1:].any()


@pytest.mark.parametrize("M,N,K", [(8, 600, 1500), (33, 200, 1500), (300, 700, 900)])
def test_gemm_pad_stream_and_repeat_give_the_same_bits(M, N, K):
    A, _ = operand(M, K, 5)
    B, _ = operand(N, K, 6)
    C = occ.occ_gemm_mx4(A, B, torch.empty((M, N), device=DEV))
    assert torch.equal(occ.occ_gemm_mx4(A, B, torch.empty((M, N), device=DEV)), C)
    assert torch.equal(occ.occ_gemm_mx4(A, B, torch.empty((M, N), device=DEV), lds_bytes=8192), C)
    s = torch.cuda.Stream()
    D = torch.empty((M, N), device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    occ.occ_gemm_mx4(A, B, D, stream=s)
    s.synchronize()
    assert torch.equal(D, C)
    with pytest.raises(occ.OccError) as e:
        occ.occ_gemm_mx4(A, B, C, lds_bytes=160 * 1024)
    assert e.value.status == occ.OCC_ELDS


def test_linear_layer_backward_from_column_blocks():
    """dX = dY W and dW = dY^T X with the operands quantised along the dimension each product sums over."""
    M, N, K = 200, 150, 330
    x, w, dy = draw(M, K, torch.bfloat16, 1, 0.5), draw(N, K, torch.bfloat16, 2, 0.5), draw(M, N, torch.bfloat16, 3, 0.5)
    q = {n: occ.occ_mx4_quantize(t.to(DEV), occ.mx4_empty(*t.shape, device=DEV),
                                 occ.mx4_empty(*t.t().shape, device=DEV)) for n, t in (("x", x), ("w", w), ("dy", dy))}
    val = {n: [ref.mx4_values(*ref.mx4_quantize(ref.f64(y))) for y in (t, t.t())] for n, t in (("x", x), ("w", w), ("dy", dy))}
    dx = occ.occ_gemm_mx4(q["dy"][0], q["w"][1], torch.empty((M, K), dtype=torch.bfloat16, device=DEV))
    dw = occ.occ_gemm_mx4(q["dy"][1], q["x"][1], torch.empty((N, K), device=DEV))
    check_product(dx, val["dy"][0], val["w"][1], torch.bfloat16)
    check_product(dw, val["dy"][1], val["x"][1], torch.float32)
