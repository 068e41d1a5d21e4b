"""occ_moe against a plain 64-bit implementation.

Router inputs are small integers over powers of two, so that logits are exact in binary32
whatever the order of their sums: the experts picked are equal to the reference's,
ties included.  Weights are a softmax of exact logits (2^-18: exp and a few hundred
additions); y's tolerance is the reference's sum of magnitudes."""
import numpy as np
import pytest
import torch

import block_reference as ref
from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def integers(shape, top, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-top, top + 1, shape, generator=g).double()


def normal(shape, std, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std).to(BF16)


class Layer:
    def __init__(self, T, H, I, E, k, kind, seed=0, masked=False):
        self.T, self.H, self.I, self.E, self.k = T, H, I, E, k
        self.x = (integers((T, H), 3, seed) / 2).to(BF16).to(DEV)
        self.router = (integers((E, H), 2, seed + 1) / 64).to(BF16).to(DEV)
        self.values, self.w = {}, {}
        for n, (name, rows, cols) in enumerate((("gate", I, H), ("up", I, H), ("down", H, I))):
            w = normal((E, rows, cols), cols ** -0.5, seed + 2 + n)
            if kind == "bf16":
                self.values[name], self.w[name] = [ref.f64(m) for m in w], w.to(DEV)
            else:
                q = occ.mx4_empty(rows, cols, batch=E, device=DEV)
                self.values[name] = []
                for e in range(E):
                    occ.occ_mx4_quantize(w[e].to(DEV), q[e])
                    c, s, _ = ref.mx4_unpack(q[e].codes.cpu().numpy(), q[e].scales.cpu().numpy(), rows, cols)
                    self.values[name].append(ref.mx4_values(c, s))
                self.w[name] = q
        self.mask = None
        if masked:
            self.mask = torch.arange(T) % 3 != 1
        self.workspace = torch.zeros(occ.occ_moe_workspace_bytes(T, H, I, E, k), dtype=torch.uint8, device=DEV)

    def run(self, renorm=True, stream=None, x=None):
        y = torch.full((self.T, self.H), float("nan"), dtype=BF16, device=DEV)
        ids = torch.full((self.T, self.k), -7, dtype=torch.int32, device=DEV)
        w = torch.full((self.T, self.k), float("nan"), device=DEV)
        occ.occ_moe(self.x if x is None else x, self.router, self.w["gate"], self.w["up"], self.w["down"], y, top_k=self.k,
                    workspace=self.workspace, ids=ids, weights=w, renorm=renorm,
                    mask=None if self.mask is None else self.mask.to(DEV), stream=stream)
        return y, ids, w

    def check(self, y, ids, w, renorm=True):
        mask = None if self.mask is None else self.mask.numpy()
        want_ids, want_w = ref.route(ref.f64(self.x) @ ref.f64(self.router).T, self.k, renorm, mask)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        assert (np.abs(ref.f64(w) - want_w) <= 2.0 ** -18 * want_w).all()
        want, tol = ref.moe(ref.f64(self.x), want_ids, want_w, *(self.values[n] for n in ("gate", "up", "down")))
        err = np.abs(ref.f64(y) - want)
        assert (err <= tol).all(), (float(err.max()), np.argwhere(~(err <= tol))[:4].tolist())


# one token to 64; one expert to more than a wave holds; every expert picked; ragged rows of 16 and steps of 128
SHAPES = [(1, 8, 8, 1, 1), (1, 128, 64, 4, 2), (1, 1032, 520, 9, 3), (2, 256, 136, 130, 5), (5, 264, 1048, 6, 6),
          (16, 512, 128, 16, 4), (17, 320, 264, 12, 2), (31, 72, 200, 70, 16), (33, 640, 96, 8, 8), (50, 200, 128, 5, 1),
          (64, 384, 328, 20, 4), (64, 64, 32, 300, 7)]


@pytest.mark.parametrize("kind", ["bf16", "mx4"])
@pytest.mark.parametrize("T,H,I,E,k", SHAPES)
def test_layer(T, H, I, E, k, kind):
    m = Layer(T, H, I, E, k, kind, seed=T + E, masked=T % 2 == 0)
    renorm = (T + k) % 2 == 0
    out = m.run(renorm)
    m.check(*out, renorm)
    again = m.run(renorm)   # the workspace is ready for the next call, and no sum depends on timing
    assert all(torch.equal(a, b) for a, b in zip(out, again))


# the most logits a routing can have; long runs of units in the second product; several units of four row blocks in the
# first; one token to every expert
@pytest.mark.parametrize("kind", ["bf16", "mx4"])
@pytest.mark.parametrize("T,H,I,E,k", [(64, 64, 32, 512, 16), (20, 72, 8200, 6, 3), (24, 1160, 264, 4, 2), (1, 96, 40, 16, 16)])
def test_layer_at_the_ends_of_its_splits(T, H, I, E, k, kind):
    test_layer(T, H, I, E, k, kind)


# the last expert's last task has blocks past its rows, in both products: what follows them reaches no output (that
# nothing of it is read either is test_moe_extent_cpu.py's)
@pytest.mark.parametrize("T,H,I,E,k", [(2, 48, 80, 3, 3), (18, 1072, 208, 2, 2)])
def test_blocks_past_the_last_experts_rows(T, H, I, E, k):
    m = Layer(T, H, I, E, k, "mx4", seed=11)
    own = m.run()
    m.check(*own)
    for name in ("gate", "up", "down"):   # NaN scales follow the last expert's
        q = m.w[name]
        more = occ.mx4_empty(q.rows, q.cols, batch=E + 1, device=DEV)
        more.codes[:E], more.scales[:E] = q.codes, q.scales
        more.codes[E], more.scales[E] = 0, 255
        m.w[name] = occ.Mx4(more.codes[:E], more.scales[:E], q.rows, q.cols)
    assert all(torch.equal(a, b) for a, b in zip(own, m.run()))


def test_equal_logits_go_to_the_lower_index():
    m = Layer(3, 64, 32, 100, 6, "bf16")
    m.router[:] = m.router[7]
    _, ids, w = m.run()
    assert (ids.cpu() == torch.arange(6)).all() and torch.allclose(w, torch.full_like(w, 1 / 6), rtol=1e-6)


def test_all_tokens_masked():
    m = Layer(20, 136, 64, 10, 3, "bf16", masked=True)
    m.mask[:] = False
    y, ids, w = m.run()
    assert (y == 0).all() and (ids == -1).all() and (w == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [6, 40])
def test_nonfinite_values_stay_with_their_tokens(T, kind):
    """A NaN token spoils its own row; an expert whose weights hold a NaN or an infinity, only rows that picked it."""
    m = Layer(T, 256, 128, 8, 2, kind, seed=5)
    clean = m.run()
    bad_expert = int(clean[1][0, 0])
    for name in ("gate", "down"):
        w = normal((m.w[name].shape if kind == "bf16" else (8, m.w[name].rows, m.w[name].cols))[1:], 0.1, 9).to(DEV)
        w[17, 33] = float("nan") if name == "gate" else float("inf")
        w[16, 1] = float("inf")
        if kind == "bf16":
            m.w[name][bad_expert] = w
        else:
            occ.occ_mx4_quantize(w, m.w[name][bad_expert])
    x = m.x.clone()
    x[T - 1, 3] = float("nan")
    y, ids, wts = m.run(x=x)
    assert torch.isnan(y[T - 1]).all() and torch.isnan(wts[T - 1]).all()
    hit = (clean[1] == bad_expert).any(1)
    assert torch.equal(ids[:T - 1], clean[1][:T - 1])
    for t in range(T - 1):
        if hit[t]:
            assert not torch.isfinite(y[t]).all()
        else:
            assert torch.equal(y[t], clean[0][t]), t


def test_strided_tokens_experts_and_outputs():
    T, H, I, E, k = 9, 136, 72, 5, 2
    m = Layer(T, H, I, E, k, "bf16", seed=3)
    want = m.run()
    wide_x = torch.full((T, H + 24), float("nan"), dtype=BF16, device=DEV)
    wide_x[:, :H] = m.x
    both = torch.full((E, 2 * I + 1, H), float("nan"), dtype=BF16, device=DEV)   # gate and up rows of an expert together
    both[:, :I], both[:, I:2 * I] = m.w["gate"], m.w["up"]
    wide_y = torch.full((T, H + 7), 7.0, dtype=BF16, device=DEV)
    y = wide_y[:, 3:3 + H]
    occ.occ_moe(wide_x[:, :H], m.router, both[:, :I], both[:, I:2 * I], m.w["down"], y, top_k=k, workspace=m.workspace)
    assert torch.equal(y, want[0]) and (wide_y[:, :3] == 7).all() and (wide_y[:, 3 + H:] == 7).all()


def test_two_streams_with_a_workspace_each():
    layers = [Layer(7, 1032, 520, 12, 3, "bf16", seed=1), Layer(40, 640, 264, 9, 4, "mx4", seed=2)]
    want = [m.run() for m in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for m, s in zip(layers, streams):
            with torch.cuda.stream(s):
                got.append(m.run())
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(out, want[i % 2])), i


def test_graph_replays():
    """Captured once, replayed with new tokens, with other work on the device between the replays."""
    m = Layer(4, 264, 136, 16, 4, "bf16", seed=8)
    y = torch.empty((4, 264), dtype=BF16, device=DEV)
    x = m.x.clone()
    args = (m.router, m.w["gate"], m.w["up"], m.w["down"], y)
    kw = dict(top_k=4, workspace=m.workspace)
    occ.occ_moe(x, *args, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        occ.occ_moe(x, *args, **kw)
    for i in range(4):
        x.copy_((integers((4, 264), 3, 50 + i) / 2).to(BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, m.run(x=x)[0]), i


def test_refusals():
    m = Layer(4, 64, 32, 8, 2, "bf16")
    y = torch.empty((4, 64), dtype=BF16, device=DEV)
    w = m.w
    small = torch.zeros(64, dtype=torch.uint8, device=DEV)
    for kw, status in ((dict(top_k=9), occ.OCC_EINVAL), (dict(top_k=0), occ.OCC_EINVAL), (dict(workspace=small), occ.OCC_EINVAL)):
        with pytest.raises(occ.OccError) as e:
            occ.occ_moe(m.x, m.router, w["gate"], w["up"], w["down"], y, **dict(dict(top_k=2, workspace=m.workspace), **kw))
        assert e.value.status == status
    with pytest.raises(occ.OccError) as e:
        occ.occ_moe(m.x, m.router, w["gate"], w["up"], w["down"], m.x, top_k=2, workspace=m.workspace)
    assert e.value.status == occ.OCC_EALIAS
    for bad in (dict(x=m.x.float()), dict(w_down=w["gate"]), dict(w_up=w["up"].float()), dict(mask=torch.ones(3, device=DEV).bool())):
        a = dict(x=m.x, router=m.router, w_gate=w["gate"], w_up=w["up"], w_down=w["down"], y=y, top_k=2, workspace=m.workspace)
        with pytest.raises(ValueError):
            occ.occ_moe(**dict(a, **bad))


@pytest.mark.parametrize("kind", ["bf16", "mx4"])
@pytest.mark.parametrize("T,H,I,E,k", [(1, 64, 264, 4, 2), (7, 136, 520, 3, 2), (12, 64, 264, 2, 2), (40, 128, 200, 2, 2),
                                       (64, 64, 1032, 5, 3)])
def test_hidden_activations_keep_their_bits(T, H, I, E, k, kind):
    """y's own rounding (2^-8) is the only one to bf16 in sight: a hidden activation is good to 2^-15 besides what its
    sums cost, so y's tolerance has that of the sums of magnitudes.  8, 16 and 32 tokens of an expert among them."""
    m = Layer(T, H, I, E, k, kind, seed=31 + T)
    y, ids, w = m.run()
    x, want, tol = ref.f64(m.x), np.zeros((T, H)), np.zeros((T, H))
    ids, w = ref.route(x @ ref.f64(m.router).T, k, True, None)
    for t in range(T):
        for e, p in zip(ids[t], w[t]):
            wg, wu, wd = (m.values[n][e] for n in ("gate", "up", "down"))
            g, u = wg @ x[t], wu @ x[t]
            s = g / (1 + np.exp(-g))
            eg, eu = (H * 2.0 ** -23 * (abs(v) @ abs(x[t])) for v in (wg, wu))
            eh = 1.1 * abs(u) * eg + abs(s) * eu + (2.0 ** -15 + 2.0 ** -20) * abs(s * u)
            want[t] += p * (wd @ (s * u))
            tol[t] += p * (abs(wd) @ (eh + (I * 2.0 ** -23 + 2.0 ** -16) * abs(s * u)))
    err = np.abs(ref.f64(y) - want)
    assert (err <= tol + 2.0 ** -8 * np.abs(want)).all(), float((err - tol - 2.0 ** -8 * np.abs(want)).max())


@pytest.mark.parametrize("T", [6, 40])
def test_an_infinite_weight_gives_an_infinity(T):
    """In one place of each expert's last product: its row of y is that infinity, no NaN, and nothing else changes."""
    m = Layer(T, 128, 72, 3, 2, "bf16", seed=4)
    clean, ids, _ = m.run()
    x = ref.f64(m.x)
    for e in range(3):
        m.w["down"][e, 17 + e, 33] = float("inf")
    y = m.run()[0].cpu()
    for t in range(T):
        rows = {}
        for e in ids[t].tolist():
            g, u = m.values["gate"][e] @ x[t], m.values["up"][e] @ x[t]
            rows[17 + e] = float(np.sign((g / (1 + np.exp(-g)) * u)[33]))
        for r in range(128):
            if r in rows:
                assert rows[r] != 0 and float(y[t, r]) == rows[r] * float("inf"), (t, r)
            else:
                assert y[t, r] == clean[t, r].cpu(), (t, r)


def test_refuses_experts_that_share_memory():
    """An expanded weight has one matrix; the call raises before anything is launched."""
    m = Layer(4, 64, 32, 8, 2, "bf16")
    y = torch.full((4, 64), 5.0, dtype=BF16, device=DEV)
    for name in ("gate", "up", "down"):
        w = dict(m.w, **{name: m.w[name][:1].expand(8, -1, -1)})
        with pytest.raises(ValueError):
            occ.occ_moe(m.x, m.router, w["gate"], w["up"], w["down"], y, top_k=2, workspace=m.workspace)
    assert (y == 5).all()


def test_host_threads_with_layers_of_different_sizes():
    """The router's logits of the two are 128 and 36 KiB of LDS: each thread's calls give what they give alone."""
    import threading
    layers = [Layer(64, 64, 32, 512, 2, "bf16", seed=1), Layer(64, 72, 40, 140, 2, "bf16", seed=2)]
    want = [m.run() for m in layers]
    streams, bad = [torch.cuda.Stream() for _ in layers], []
    torch.cuda.synchronize()

    def work(m, s, expected):
        try:
            with torch.cuda.stream(s):
                for _ in range(50):
                    if not all(torch.equal(a, b) for a, b in zip(m.run(stream=s), expected)):
                        bad.append("other results")
        except Exception as e:   # a refused launch among them
            bad.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in zip(layers, streams, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad, bad[:3]
