"""The block operators together: a decode step eagerly and from a graph, and training steps."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_decode_step_and_its_graph():
    from paper_2606_09200_amd.block import Decoder
    d = Decoder(layers=2, tokens=5, hidden=264, inner=136, experts=6, top_k=2)
    inputs = [torch.randn(5, 264, generator=torch.Generator().manual_seed(i)).cuda() for i in range(3)]
    lives = [torch.tensor(m, device="cuda") for m in ([True] * 5, [True, False, True, True, False], [False] * 5)]
    graph = None
    for again in range(2):
        for x, live in zip(inputs, lives):
            d.embedded.copy_(x)
            d.live.copy_(live)
            d.out.zero_()
            eager, ids = d.step().clone(), d.ids.clone()
            assert bool((ids[:, ~live] == -1).all()) and bool((ids[:, live] >= 0).all())
            if graph is None:
                graph = d.graph()
            for _ in range(2):
                d.out.zero_()
                d.ids.fill_(7)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(d.out, eager) and torch.equal(d.ids, ids)
            if not live.any():  # the experts give nothing, its norm is of zeros, the residual stays
                assert torch.equal(d.out, d.embedded)


def test_training_step_is_the_operators_composed():
    """Each gradient against the formulas in 64 bits on the operands the 4-bit products had."""
    from paper_2606_09200_amd import binding as occ
    from paper_2606_09200_amd.block import Trainee
    rows, hidden, out = 70, 136, 96
    t = Trainee(rows, hidden, out)
    g = torch.Generator().manual_seed(5)
    f, x, dz = ((torch.randn(rows, n, generator=g)).to(BF16).cuda() for n in (hidden, hidden, out))
    z = t.forward(f, x)

    def values(q):
        return occ.occ_mx4_dequantize(q, torch.empty(q.rows, q.cols, device="cuda")).double()

    want = values(t.h4) @ values(t.w4).t()
    # a binary32 sum of `hidden` products rounded once to bf16
    tol = want.abs() * 2.0 ** -8 + hidden * 2.0 ** -24 * (values(t.h4).abs() @ values(t.w4).abs().t()) + 1e-30
    assert bool(((z.double() - want).abs() <= tol).all())
    t.backward(dz, f)
    want = values(t.dz4_t) @ values(t.h4_t).t()
    tol = rows * 2.0 ** -23 * (values(t.dz4_t).abs() @ values(t.h4_t).abs().t()) + 1e-30
    assert bool(((t.dW.double() - want).abs() <= tol).all())


def test_training_lowers_the_loss():
    from paper_2606_09200_amd.block import main
    losses = main(["--layers", "1", "--tokens", "2", "--hidden", "256", "--inner", "128", "--experts", "4", "--top-k", "2",
                   "--rows", "512", "--out", "128", "--steps", "12"])
    assert losses[-1] < 0.7 * losses[0]


@pytest.mark.parametrize("rows,hidden,out", [(70, 136, 96), (300, 520, 72)])
def test_training_step_gives_every_gradient(rows, hidden, out):
    """dh against the product of the 4-bit operands it had, and the norms' gradients against the formulas in 64 bits from
    that dh: df, dx and those of the weights and the gate.  Tolerances as in the operators' own tests."""
    import block_reference as ref
    from paper_2606_09200_amd import binding as occ
    from paper_2606_09200_amd.block import Trainee
    t = Trainee(rows, hidden, out)
    g = torch.Generator().manual_seed(6)
    for w in (t.w_post, t.w_pre, t.gate):
        w.copy_(1 + 0.2 * torch.randn(hidden, generator=g))
    f, x, dz = ((torch.randn(rows, n, generator=g)).to(BF16).cuda() for n in (hidden, hidden, out))
    t.forward(f, x)
    t.backward(dz, f)

    def values(q):
        return ref.f64(occ.occ_mx4_dequantize(q, torch.empty(q.rows, q.cols, device="cuda")))

    a, b = values(t.dz4), values(t.w4_t)
    want = a @ b.T
    tol = out * 2.0 ** -23 * (abs(a) @ abs(b).T) + 2.0 ** -8 * abs(want)
    assert (abs(ref.f64(t.dh) - want) <= tol).all()
    # the training step passes the norms' weights in bf16
    w = {n: ref.f64(getattr(t, n).to(BF16)) for n in ("w_post", "w_pre", "gate")}
    y, _, rstd = ref.norm_gate(ref.f64(f), ref.f64(x), w["w_post"], w["w_pre"], w["gate"][None], 1.0, 1e-6)
    assert (abs(ref.f64(t.y) - y) <= 2.0 ** -8 * abs(y) + 2.0 ** -16 * (abs(ref.f64(x)) + abs(y - ref.f64(x)))).all()
    assert (abs(ref.f64(t.rstd) - rstd) <= 2.0 ** -16 * rstd).all()
    want, mag = ref.norm_gate_bwd(None, ref.f64(t.dh), ref.f64(f), ref.f64(t.y), ref.f64(t.rstd), w["w_post"], w["w_pre"],
                                  w["gate"][None], 1.0)
    for n in ("df", "dx", "dw_post", "dw_pre", "dgate"):
        rounding = 2.0 ** -8 * abs(want[n]) if n in ("df", "dx") else 0.0
        assert (abs(ref.f64(getattr(t, n)) - want[n]) <= 2.0 ** -16 * mag[n] + rounding + 1e-30).all(), n
