"""occ_attn_paged: what a row does not see has no influence on its bits, neither later tokens' keys and values, whatever they are,
nor the other rows of its tile, whose running maxima grow at other times."""
import pytest
import torch

from test_gpu_attn import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_fresh", [1, 400])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("peaky", [1.0, 3.0, 10.0])
def test_later_keys(D, max_fresh, peaky):
    p = Problem([(300, 200), (20, 90)], 4, 2, D, 16, seed=40 + D, peaky=peaky)
    clean, clean_lse = (t.clone() for t in p.run(max_fresh=max_fresh))
    for factor in (2.0 ** 4, 2.0 ** 30, float("inf"), float("nan")):
        for i, (cached, fresh) in enumerate(p.requests):
            for new in (fresh - 1, fresh // 2, 5):
                j, at = cached + new, p.starts[i]
                page = p.table[i][j // p.page], j % p.page
                k, v = p.dk[page].clone(), p.dv[page].clone()
                p.dk[page] *= factor
                p.dv[page] *= factor
                out, lse = p.run(max_fresh=max_fresh)
                assert torch.equal(out[at:at + new], clean[at:at + new]), (factor, i, new)
                assert torch.equal(lse[at:at + new], clean_lse[at:at + new]), (factor, i, new)
                p.dk[page], p.dv[page] = k, v


@pytest.mark.parametrize("max_fresh", [1, 400])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("factor", [0.0, 8.0, 2.0 ** 60])
def test_other_rows(D, max_fresh, factor):
    p = Problem([(300, 200), (90, 1)], 4, 2, D, 16, seed=50 + D, peaky=3.0)
    clean, clean_lse = (t.clone() for t in p.run(max_fresh=max_fresh))
    rows = torch.arange(p.rows) % 3 == 0
    p.dq[rows.to(p.dq.device)] *= factor
    out, lse = p.run(max_fresh=max_fresh)
    others = (~rows).to(out.device)
    assert torch.equal(out[others], clean[others]) and torch.equal(lse[others], clean_lse[others])
