"""occ_attn_paged at the ends of what occ.h allows.  The plan's numbers are checked on the host (test_attn_plan_limits_cpu.py); here
what the kernels make of them."""
import pytest
import torch

from gpu_common import DEV
from paper_2606_09200_amd import binding as occ
from test_gpu_attn import BF16, i32, workspace_for

pytestmark = pytest.mark.gpu


def expected(q, k, v, scale):
    """64 bits: q (n, D) over all of k, v (keys, D)."""
    p = torch.softmax(q.double() @ k.double().t() * scale, 1)
    return p @ v.double()


def close(out, q, k, v, scale):
    """Weights of one bf16 value and the output's own rounding, 2^-8 each; the logits' part is next to nothing with 8 products."""
    want, mag = expected(q, k, v, scale), expected(q, k, v.abs(), scale)
    assert bool(((out.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -18) * mag + 2.0 ** -8 * want.abs()).all())


@pytest.mark.parametrize("most", [1, 1 << 18])
@pytest.mark.parametrize("window", [2 ** 31 - 65537, 2 ** 31 - 200000])
def test_a_window_that_reaches_back_past_32_bits(window, most):
    """2^18 rows over 3 keys without causality: the window of the first begins 2^31 + 2^18 keys before key 0, and all see all."""
    rows, D = 1 << 18, 8
    g = torch.Generator().manual_seed(1)
    k, v = (torch.full((2, 65536, 1, D), float("nan"), dtype=BF16, device=DEV) for _ in range(2))
    k[1, :3, 0], v[1, :3, 0] = (torch.randn((3, D), generator=g).to(BF16).to(DEV) for _ in range(2))
    q = torch.randn((rows, 1, D), generator=g).to(BF16).to(DEV)
    table = torch.full((1, 32767), -1, dtype=torch.int32, device=DEV)
    table[0, 0] = 1
    out = torch.full_like(q, 7.0)
    occ.occ_attn_paged(q, k, v, table, i32([0, rows]), i32([3]), out, max_fresh=most, causal=False, window=window, workspace=workspace_for(D))
    close(out[:, 0], q[:, 0], k[1, :3, 0], v[1, :3, 0], D ** -0.5)


@pytest.mark.parametrize("causal", [False, True])
def test_all_rows_that_there_can_be(causal):
    """One request of 2^31 - 1 rows, of which causality leaves the last 5 some keys."""
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("80 GB of memory")
    rows, D, n = 2 ** 31 - 1, 8, 5
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((1, 16, 1, D), generator=g).to(BF16).to(DEV) for _ in range(2))
    q, out = (torch.empty((rows, 1, D), dtype=BF16, device=DEV) for _ in range(2))
    some = [0, 1, 255, 256, rows // 2, rows - 300, rows - 257, rows - 256, rows - 255, rows - 6, rows - 5, rows - 4, rows - 3, rows - 2, rows - 1]
    q[some, 0] = torch.randn((len(some), D), generator=g).to(BF16).to(DEV)
    out[some] = 7.0
    occ.occ_attn_paged(q, k, v, i32([[0]]), i32([0, rows]), i32([n]), out, max_fresh=rows, causal=causal, workspace=workspace_for(D))
    for r in some:
        seen = n if not causal else max(0, n - rows + r + 1)
        if seen == 0:
            assert bool((out[r] == 0).all())
        else:
            close(out[r], q[r], k[0, :seen, 0], v[0, :seen, 0], D ** -0.5)
