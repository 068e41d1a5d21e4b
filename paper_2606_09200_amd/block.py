"""The block operators as a model uses them.

``Decoder`` serves: layers of norms and a mixture of experts with 4-bit weights, one
step of a few tokens, which a HIP graph can hold.  ``Trainee`` trains: a block's norms
with their gate and a linear layer whose products, forward and backward, are 4-bit.

    python paper_2606_09200_amd/block.py            # both, with their times
"""
import argparse
import os
import sys
import time

if __package__ in (None, ""):
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2606_09200_amd import binding as occ

BF16 = torch.bfloat16


def quantize_experts(w):
    """(experts, rows, cols) weights as an Mx4 batch."""
    q = occ.mx4_empty(w.shape[1], w.shape[2], batch=w.shape[0], device=w.device)
    for e in range(w.shape[0]):
        occ.occ_mx4_quantize(w[e], out=q[e])
    return q


class Decoder:
    """``layers`` times: the residual takes the last block's output, normed, and what it
    then is goes, normed, through the experts.  Weights are random."""

    def __init__(self, layers, tokens, hidden, inner, experts, top_k, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)

        def rand(*shape, scale):
            return (torch.randn(*shape, generator=g, device=device) * scale).to(BF16)

        self.top_k = top_k
        self.layers = []
        for _ in range(layers):
            up = dict(scale=hidden ** -0.5)
            self.layers.append(dict(
                w_post=1 + rand(hidden, scale=0.1), w_pre=1 + rand(hidden, scale=0.1),
                router=rand(experts, hidden, scale=hidden ** -0.5),
                gate=quantize_experts(rand(experts, inner, hidden, **up)),
                up=quantize_experts(rand(experts, inner, hidden, **up)),
                down=quantize_experts(rand(experts, hidden, inner, scale=inner ** -0.5))))
        # what a step reads, writes and passes on; the experts' workspace is zeroed once
        self.embedded = torch.zeros(tokens, hidden, dtype=BF16, device=device)
        self.live = torch.ones(tokens, dtype=torch.bool, device=device)  # slots that hold a request
        self.x, self.h, self.f = (torch.zeros_like(self.embedded) for _ in range(3))
        self.out = torch.zeros_like(self.embedded)
        self.ids = torch.zeros(layers, tokens, top_k, dtype=torch.int32, device=device)
        self.workspace = torch.zeros(occ.occ_moe_workspace_bytes(tokens, hidden, inner, experts, top_k),
                                     dtype=torch.uint8, device=device)

    def step(self):
        """``out`` from ``embedded`` and ``live``, on the current stream."""
        for i, w in enumerate(self.layers):
            if i == 0:  # nothing to add yet: the embedding is the residual, and only the norm before the block runs
                self.f.zero_()
                occ.occ_norm_gate(self.f, self.embedded, self.x, self.h, w_pre=w["w_pre"], post=False)
            else:
                occ.occ_norm_gate(self.f, self.x, self.x, self.h, w_post=self.layers[i - 1]["w_post"], w_pre=w["w_pre"])
            occ.occ_moe(self.h, w["router"], w["gate"], w["up"], w["down"], self.f, top_k=self.top_k,
                        workspace=self.workspace, ids=self.ids[i], mask=self.live)
        occ.occ_norm_gate(self.f, self.x, self.out, w_post=self.layers[-1]["w_post"])
        return self.out

    def graph(self):
        """The step as a graph: ``replay()`` it after writing ``embedded`` and ``live``."""
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        return graph


class Trainee:
    """z = W norm(x + gate norm(f)), all norms and products by the block operators:
    activations, gradients and weights are rounded to 4 bits for the products, the weights
    themselves and their gradients are binary32."""

    def __init__(self, rows, hidden, out, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.W = torch.randn(out, hidden, generator=g, device=device) * hidden ** -0.5
        self.w_post, self.w_pre, self.gate = (torch.ones(hidden, device=device) for _ in range(3))
        self.w4, self.w4_t = occ.mx4_empty(out, hidden, device=device), occ.mx4_empty(hidden, out, device=device)
        self.h4, self.h4_t = occ.mx4_empty(rows, hidden, device=device), occ.mx4_empty(hidden, rows, device=device)
        self.dz4, self.dz4_t = occ.mx4_empty(rows, out, device=device), occ.mx4_empty(out, rows, device=device)

        def empty(*shape, dtype=BF16):
            return torch.empty(*shape, dtype=dtype, device=device)

        f32 = torch.float32
        self.y, self.h, self.dh = (empty(rows, hidden) for _ in range(3))
        self.df, self.dx = empty(rows, hidden), empty(rows, hidden)
        self.z, self.rstd = empty(rows, out), empty(rows, 2, dtype=f32)
        self.dW = empty(out, hidden, dtype=f32)
        self.dw_post, self.dw_pre, self.dgate = empty(hidden, dtype=f32), empty(hidden, dtype=f32), empty(1, hidden, dtype=f32)
        self.workspace = empty(occ.occ_norm_gate_bwd_workspace_bytes(rows, hidden), dtype=torch.uint8)

    def _norm_weights(self):
        return dict(w_post=self.w_post.to(BF16), w_pre=self.w_pre.to(BF16), gate=self.gate.to(BF16)[None])

    def forward(self, f, x):
        occ.occ_norm_gate(f, x, self.y, self.h, rstd=self.rstd, **self._norm_weights())
        occ.occ_mx4_quantize(self.h, out=self.h4, out_t=self.h4_t)
        occ.occ_mx4_quantize(self.W, out=self.w4, out_t=self.w4_t)
        return occ.occ_gemm_mx4(self.h4, self.w4, self.z)

    def backward(self, dz, f):
        """Gradients of the weights, and df and dx."""
        occ.occ_mx4_quantize(dz, out=self.dz4, out_t=self.dz4_t)
        occ.occ_gemm_mx4(self.dz4, self.w4_t, self.dh)
        occ.occ_gemm_mx4(self.dz4_t, self.h4_t, self.dW)
        return occ.occ_norm_gate_bwd(None, self.dh, f, self.y, self.rstd, self.df, self.dx, dw_post=self.dw_post,
                                     dw_pre=self.dw_pre, dgate=self.dgate, workspace=self.workspace,
                                     **self._norm_weights())

    def step(self, f, x, target, lr):
        """One step of gradient descent on the mean over rows of |z - target|^2 / 2; the loss before it."""
        diff = self.forward(f, x).float() - target
        loss = diff.square().sum() / (2 * len(f))
        self.backward((diff / len(f)).to(BF16), f)
        for w, dw in ((self.W, self.dW), (self.w_post, self.dw_post), (self.w_pre, self.dw_pre),
                      (self.gate, self.dgate[0])):
            w.sub_(dw, alpha=lr)
        return loss


def timed(fn, n):
    """us of ``fn``, n at a time."""
    fn()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(n):
        fn()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / n * 1e6


def main(argv=None):
    p = argparse.ArgumentParser(description="a decode step and a training step of the block operators")
    for name, value in (("layers", 4), ("tokens", 8), ("hidden", 4096), ("inner", 2048), ("experts", 32), ("top-k", 4),
                        ("rows", 4096), ("out", 4096), ("steps", 20)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)
    d = Decoder(a.layers, a.tokens, a.hidden, a.inner, a.experts, a.top_k)
    d.embedded.copy_(torch.randn(a.tokens, a.hidden, generator=g, device="cuda"))
    eager = d.step().clone()
    graph = d.graph()
    graph.replay()
    assert torch.equal(d.out, eager), "the graph's step differs"
    print("decode: %d layers, %d tokens: %.0f us a step, %.0f from a graph"
          % (a.layers, a.tokens, timed(d.step, 50), timed(graph.replay, 50)), flush=True)
    t = Trainee(a.rows, a.hidden, a.out)
    f, x = (torch.randn(a.rows, a.hidden, generator=g, device="cuda").to(BF16) for _ in range(2))
    teacher = torch.randn(a.out, a.hidden, generator=g, device="cuda") * a.hidden ** -0.5
    target = torch.nn.functional.rms_norm(x.float(), (a.hidden,)) @ teacher.t()
    losses = [float(t.step(f, x, target, 0.3)) for _ in range(a.steps)]
    print("train: %d x %d x %d: loss %.2f -> %.2f in %d steps, %.0f us a step"
          % (a.rows, a.hidden, a.out, losses[0], losses[-1], a.steps,
             timed(lambda: t.step(f, x, target, 0.0), 20)), flush=True)
    return losses


if __name__ == "__main__":
    main()
