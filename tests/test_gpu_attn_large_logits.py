"""occ_attn_paged where logits are so large that one binary32 step of theirs is a power of 2^64 and more: finite values have a finite
answer, the value of the largest logit's key.

A logit is off by (D + 4) 2^-24 of scale sum |q| |k|, as in test_gpu_attn.py.  Rows whose largest logit is ahead of every other by
twice that and 64 more have weights of 1 and below 2^-90: o is that key's value, off by the weight's rounding and by
its own, 2^-8 each, and lse is that logit, off by its error and its own rounding."""
import numpy as np
import pytest
import torch

from test_gpu_attn import Problem, compare, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_fresh", [1, 400])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("power", [20, 28, 32, 33, 40, 70, 110])
def test_the_largest_logit_wins(power, D, max_fresh):
    p = Problem([(150, 30), (0, 40), (200, 1)], 4, 2, D, 16, seed=power + D)
    p.dq *= 2.0 ** (power // 2)
    p.dk *= 2.0 ** (power - power // 2)
    out, lse = (f64(t) for t in p.run(max_fresh=max_fresh))
    q, k, v = f64(p.dq), f64(p.dk), f64(p.dv)
    checked = 0
    for i, (cached, fresh) in enumerate(p.requests):
        ids = np.array([p.table[i][j // p.page] for j in range(cached + fresh)])
        keys, values = (t[ids, np.arange(len(ids)) % p.page] for t in (k, v))
        for r in range(fresh):
            n, row = cached + r + 1, p.starts[i] + r
            for h in range(p.Hq):
                x = keys[:n, h // 2] @ q[row, h] * D ** -0.5
                err = (D + 4) * 2.0 ** -24 * (np.abs(keys[:n, h // 2]) @ np.abs(q[row, h])).max() * D ** -0.5
                assert np.isfinite(out[row, h]).all() and np.isfinite(lse[row, h]), (i, r, h)
                best = int(x.argmax())
                if n > 1 and x[best] - np.partition(x, -2)[-2] < 2 * err + 64:
                    continue
                checked += 1
                want = values[best, h // 2]
                assert (np.abs(out[row, h] - want) <= (2.0 ** -7 + 2.0 ** -16) * np.abs(want)).all(), (i, r, h)
                assert abs(lse[row, h] - x[best]) <= err + 2.0 ** -23 * abs(x[best]) + 2.0 ** -22, (i, r, h)
    assert checked > 200


@pytest.mark.parametrize("max_fresh", [1, 400])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_ordinary_rows_beside_them(D, max_fresh):
    """Rows of ordinary logits in the same tiles are what they are in 64 bits; with few rows, where each has its own maximum at
    all times, they have the bits that they have without such rows."""
    p = Problem([(60, 50), (90, 1)], 4, 2, D, 16, seed=3)
    clean, clean_lse = (t.clone() for t in p.run(max_fresh=max_fresh))
    large = list(range(0, p.rows, 3))
    p.dq[large] *= 2.0 ** 60
    out, lse = p.run(max_fresh=max_fresh)
    others = [r for r in range(p.rows) if r not in large]
    if max_fresh == 1:
        assert torch.equal(out[others], clean[others]) and torch.equal(lse[others], clean_lse[others])
    compare(f64(out)[others], f64(lse)[others], [w[others] for w in p.want()], p.D)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
