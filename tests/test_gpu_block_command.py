"""The command of block.py: what its decode step with attention has in its cache is what it says."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,context,page,window", [(3, 40, 16, 16), (4, 300, 16, 0), (5, 0, 16, 0), (2, 31, 16, 0), (2, 32, 1, 0)])
def test_the_cache_holds_the_context(monkeypatch, capsys, tokens, context, page, window):
    from paper_2606_09200_amd import block
    made = []

    class Recorded(block.Decoder):
        def __init__(self, *a, **k):
            super().__init__(*a, **k)
            made.append(self)

    monkeypatch.setattr(block, "Decoder", Recorded)
    block.main(["--layers", "2", "--tokens", str(tokens), "--hidden", "256", "--inner", "128", "--experts", "4", "--top-k", "2", "--rows", "64",
                "--out", "64", "--steps", "1", "--heads", "4", "--kv-heads", "2", "--head", "32", "--context", str(context), "--page", str(page),
                "--window", str(window)])
    assert "attention over %d keys" % (context + 1) in capsys.readouterr().out
    d, = [d for d in made if d.cache is not None]
    c = d.cache
    assert c.cached.tolist() == [context] * tokens and c.lens.tolist() == [context + 1] * tokens
    assert c.positions.tolist() == [context] * tokens and d.window == window
    # pages of their own, in which the new tokens' slots are
    used = -(-(context + 1) // page)
    pages = c.table[:, :used].flatten().tolist()
    assert len(set(pages)) == tokens * used and all(0 <= p < c.pages for p in pages)
    assert c.slots.tolist() == [p * page + context % page for p in c.table[:, used - 1].tolist()]
    assert bool(d.live.all())
    # what is cached is read: other values in every row but the new ones change every token's output
    before = d.step().clone()
    new = c.slots.long()
    for t in (c.k, c.v):
        rows = t.flatten(1, 2)
        kept = rows[:, new].clone()
        rows.copy_(rows.flip(1) * 0.5)
        rows[:, new] = kept
    changed = (d.step() != before).any(1)
    assert changed.tolist() == [context > 0] * tokens
