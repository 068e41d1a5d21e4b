"""Attention over a paged cache as a decoder uses it: tables, rotary positions, the cache and what is read from it, over steps in
which requests bring chunks and single tokens, end, begin and find no room."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from test_gpu_attn import f64

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

REQUESTS, TOKENS, PAGE, WIDTH, PAGES = 5, 24, 4, 8, 14
HQ, HKV, HEAD = 4, 2, 24
# the third: request 0 takes the last pages, 3 and 4 have no room; the fourth: 2's pages go to 2 and 3, 4 has none; the last: all pages are
# in use until the next step, 1 and 4 need one, 2 does not
STEPS = [[10, 1, 0, 7, 3], [1, 1, 5, 1, 1], [20, 1, -1, 1, 1], [1, 1, 2, 1, 1], [0, 0, 0, 0, 0], [-1, 1, 1, -1, 1]]
UNSERVED = [[], [], [3, 4], [4], [], [1, 4]]


def decoder(layers, window=0):
    from paper_2606_09200_amd.block import Cache, Decoder
    cache = Cache(layers, REQUESTS, TOKENS, WIDTH, PAGES, PAGE, HKV, HEAD)
    return Decoder(layers, TOKENS, hidden=264, inner=136, experts=6, top_k=2, heads=HQ, cache=cache, window=window)


@pytest.mark.parametrize("window", [0, 6])
def test_steps_against_dense_attention(window):
    from paper_2606_09200_amd import binding as occ
    d = decoder(1, window)
    c = d.cache
    raw = torch.empty_like(d.qkv)
    inner = d.attend

    def attend(w, i):
        occ.occ_gemm_bt(d.h, w["qkv"], raw.flatten(1))   # what the projection gives before positions are in it
        inner(w, i)

    d.attend = attend
    turns = [int(t) for t in d.turns.cpu()]
    dense = [np.zeros((REQUESTS, WIDTH * PAGE, HKV, HEAD)) for _ in range(2)]   # keys turned in 64 bits, and values
    cached = [0] * REQUESTS
    for n, (fresh, unserved) in enumerate(zip(STEPS, UNSERVED)):
        d.embedded.copy_(torch.randn(TOKENS, 264, generator=torch.Generator().manual_seed(n)))
        c.fresh.copy_(torch.tensor(fresh, dtype=torch.int32))
        d.step()
        lens = [-1 if i in unserved else 0 if f < 0 else cached[i] + f for i, f in enumerate(fresh)]
        assert c.lens.tolist() == lens
        starts = np.concatenate([[0], np.cumsum(np.maximum(fresh, 0))]).tolist()
        assert c.starts.tolist() == starts
        q, k, v = np.split(f64(raw), [HQ, HQ + HKV], 1)
        positions = np.zeros(TOKENS, dtype=np.int64)
        for i in range(REQUESTS):
            rows = range(starts[i], starts[i + 1])
            positions[rows] = cached[i] + np.arange(len(rows))
        k = ref.rope(k, positions, turns, False, 1.0, False)
        live = np.zeros(TOKENS, dtype=bool)
        for i in range(REQUESTS):
            if lens[i] > 0:
                for r in range(starts[i], starts[i + 1]):
                    dense[0][i, positions[r]], dense[1][i, positions[r]], live[r] = k[r], v[r], True
        assert d.live.tolist() == live.tolist()
        q = ref.rope(q, positions, turns, False, 1.0, False)
        want, lse, mag, logit, seen = ref.attention(q, dense[0], dense[1], [[i] for i in range(REQUESTS)], starts, lens,
                                                    HEAD ** -0.5, True, window)
        of_requests = seen >= 0
        got = f64(d.attended)
        # q and keys are rounded to bf16 after fp32 sums: 2^-8 (1 + 2^-8) each of the logits' terms
        err = 2 * (2.0 ** -8 + 2.0 ** -15) * logit
        tol = (2 * err + 2 * err ** 2 + 2.0 ** -8 + 2.0 ** -16)[..., None] * mag + 2.0 ** -8 * np.abs(want) + 1e-30
        assert (np.abs(got - want) <= tol)[of_requests].all(), n
        assert (got[of_requests & ~live] == 0).all()
        assert torch.isfinite(d.out).all()
        c.advance()
        cached = [cached[i] if x < 0 else x for i, x in enumerate(lens)]
        assert c.cached.tolist() == cached
    assert c.free.tolist()[1] == PAGES - sum(-(-x // PAGE) for x in cached)


def test_steps_from_a_graph():
    d = decoder(2)
    graph = None
    for n, fresh in enumerate(STEPS):
        d.embedded.copy_(torch.randn(TOKENS, 264, generator=torch.Generator().manual_seed(10 + n)))
        d.cache.fresh.copy_(torch.tensor(fresh, dtype=torch.int32))
        eager = d.step().clone()
        state = [t.clone() for t in (d.cache.k, d.cache.v, d.cache.table, d.cache.lens, d.cache.slots, d.cache.free_after)]
        if graph is None:
            graph = d.graph()
        for _ in range(2):
            d.out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(d.out, eager), n
            for a, b in zip((d.cache.k, d.cache.v, d.cache.table, d.cache.lens, d.cache.slots, d.cache.free_after), state):
                assert torch.equal(a, b), n
        d.cache.advance()


def test_a_prompt_is_its_tokens():
    """One request's prompt at once and token by token: the same keys in the cache's pages, but for what the rounding of
    the layers between makes of different kernels; the first layer's are the projection's."""
    from paper_2606_09200_amd.block import Cache, Decoder
    x = torch.randn(20, 264, generator=torch.Generator().manual_seed(3)).cuda()
    outs = []
    for tokens in (20, 1):
        cache = Cache(1, 1, tokens, WIDTH, PAGES, PAGE, HKV, HEAD)
        d = Decoder(1, tokens, hidden=264, inner=136, experts=6, top_k=2, heads=HQ, cache=cache)
        cache.fresh.fill_(tokens)
        for t in range(0, 20, tokens):
            d.embedded.copy_(x[t:t + tokens])
            d.step()
            cache.advance()
        outs.append((f64(cache.k[0, :5]), f64(cache.v[0, :5])))
    for a, b in zip(*outs):
        # bf16 of two fp32 sums of 264 products in different orders: a step, 2^-7, where they fall on both sides of a rounding
        # boundary; a turned key has that of two elements, sqrt(2) 2^-7 of the largest, and a step of its own
        assert (np.abs(a - b) <= 2.0 ** -5 * np.abs(a).max(-1, keepdims=True)).all()


def test_the_command(capsys):
    from paper_2606_09200_amd.block import main
    main(["--layers", "2", "--tokens", "3", "--hidden", "256", "--inner", "128", "--experts", "4", "--top-k", "2", "--rows", "64",
          "--out", "64", "--steps", "1", "--heads", "4", "--kv-heads", "2", "--head", "32", "--context", "40", "--window", "16"])
    assert "attention over 41 keys" in capsys.readouterr().out
