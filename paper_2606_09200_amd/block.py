"""The block operators as a model uses them.

``Decoder`` serves: layers of norms and a mixture of experts with 4-bit weights, with a
``Cache`` each of them after attention, one step of new tokens, which a HIP graph can hold.
``Trainee`` trains: a block's norms
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


class Cache:
    """Keys and values of ``layers`` layers in pages, and the tables of a step: up to ``requests`` requests that bring up to
    ``tokens`` new tokens, each of ``width`` pages at most.  Write ``fresh`` before a step: a request's new tokens (0: none,
    -1: it is over); their rows follow each other in the requests' order.  ``most``: the new tokens that one request brings at
    most, all of them if not given."""

    def __init__(self, layers, requests, tokens, width, pages, page, kv_heads, head, most=None, device="cuda"):
        def zeros(*shape):
            return torch.zeros(*shape, dtype=torch.int32, device=device)

        self.page, self.pages, self.most = page, pages, tokens if most is None else most
        self.k, self.v = (torch.zeros(layers, pages, page, kv_heads, head, dtype=BF16, device=device) for _ in range(2))
        self.cached, self.fresh, self.lens, self.starts = (zeros(n) for n in (requests, requests, requests, requests + 1))
        self.table, self.ring = zeros(requests, width), torch.arange(pages, dtype=torch.int32, device=device)
        self.free, self.free_after = torch.tensor([0, pages], dtype=torch.int32, device=device), zeros(2)
        self.slots, self.positions = zeros(tokens), zeros(tokens)

    def tables(self):
        """Pages for what ``fresh`` brings; the same again if nothing has moved on."""
        occ.occ_kv_tables(self.cached, self.fresh, self.table, self.ring, self.free, page=self.page, pages=self.pages,
                          lens=self.lens, starts=self.starts, slots=self.slots, positions=self.positions,
                          free_after=self.free_after)

    def advance(self):
        """The step is taken: what it brought is cached.  Requests that had no room (``lens`` -1) are where they were."""
        self.cached.copy_(torch.where(self.lens < 0, self.cached, self.lens))
        self.free.copy_(self.free_after)


class Decoder:
    """``layers`` times: the residual takes the last block's output, normed, and what it
    then is goes, normed, through the experts.  Weights are random.  With ``heads`` query heads over a ``cache``, each layer
    has a block of attention before that of its experts."""

    def __init__(self, layers, tokens, hidden, inner, experts, top_k, device="cuda", seed=0, heads=0, cache=None, window=0):
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
        self.cache, self.window = cache, window
        if cache is not None:
            kv_heads, head = cache.k.shape[3:]
            self.split = (heads, kv_heads, kv_heads)
            for w in self.layers:
                w.update(w_attn_post=1 + rand(hidden, scale=0.1), w_attn_pre=1 + rand(hidden, scale=0.1),
                         qkv=rand((heads + 2 * kv_heads) * head, hidden, scale=hidden ** -0.5),
                         proj=rand(hidden, heads * head, scale=(heads * head) ** -0.5))
            self.turns = occ.rope_turns(head // 2, device=device)
            self.qkv, self.attended = (torch.zeros(tokens, n, head, dtype=BF16, device=device) for n in (heads + 2 * kv_heads, heads))
            self.attn_workspace = torch.zeros(occ.occ_attn_paged_workspace_bytes(heads, kv_heads, head), dtype=torch.uint8,
                                              device=device)
        # what a step reads, writes and passes on; the experts' workspace is zeroed once
        self.embedded = torch.zeros(tokens, hidden, dtype=BF16, device=device)
        self.live = torch.ones(tokens, dtype=torch.bool, device=device)  # slots that hold a request
        self.x, self.h, self.f = (torch.zeros_like(self.embedded) for _ in range(3))
        self.out = torch.zeros_like(self.embedded)
        self.ids = torch.zeros(layers, tokens, top_k, dtype=torch.int32, device=device)
        self.workspace = torch.zeros(occ.occ_moe_workspace_bytes(tokens, hidden, inner, experts, top_k),
                                     dtype=torch.uint8, device=device)

    def attend(self, w, i):
        """Layer i's attention of ``h`` into ``f``; its keys and values go into the cache."""
        occ.occ_gemm_bt(self.h, w["qkv"], self.qkv.flatten(1))
        q, k, v = self.qkv.split(self.split, 1)
        keys, values = self.cache.k[i], self.cache.v[i]
        occ.occ_rope(q, k, self.cache.positions, self.turns, v=v, k_cache=keys, v_cache=values, slots=self.cache.slots)
        occ.occ_attn_paged(q, keys, values, self.cache.table, self.cache.starts, self.cache.lens, self.attended,
                           max_fresh=self.cache.most, window=self.window, workspace=self.attn_workspace)
        occ.occ_gemm_bt(self.attended.flatten(1), w["proj"], self.f)

    def step(self):
        """``out`` from ``embedded`` and ``live``, on the current stream.  With a cache, ``live`` is what its ``fresh``
        brings; the step can be taken again until the cache advances."""
        if self.cache is not None:
            self.cache.tables()
            torch.ge(self.cache.slots, 0, out=self.live)
        post = None  # the norm of what the last block put out
        for i, w in enumerate(self.layers):
            if self.cache is not None:
                self.norm(post, w["w_attn_pre"])
                self.attend(w, i)
                post = w["w_attn_post"]
            self.norm(post, w["w_pre"])
            occ.occ_moe(self.h, w["router"], w["gate"], w["up"], w["down"], self.f, top_k=self.top_k,
                        workspace=self.workspace, ids=self.ids[i], mask=self.live)
            post = w["w_post"]
        occ.occ_norm_gate(self.f, self.x, self.out, w_post=post)
        return self.out

    def norm(self, post, pre):
        """The residual takes ``f``; ``h`` is its norm."""
        if post is None:  # nothing to add yet: the embedding is the residual, and only the norm before the block runs
            self.f.zero_()
            occ.occ_norm_gate(self.f, self.embedded, self.x, self.h, w_pre=pre, post=False)
        else:
            occ.occ_norm_gate(self.f, self.x, self.x, self.h, w_post=post, w_pre=pre)

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
                        ("rows", 4096), ("out", 4096), ("steps", 20), ("heads", 0), ("kv-heads", 8), ("head", 128),
                        ("page", 16), ("context", 1000), ("window", 0)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(1)

    def decode(what, d):
        d.embedded.copy_(torch.randn(a.tokens, a.hidden, generator=g, device="cuda"))
        eager = d.step().clone()
        if d.cache is not None:
            assert bool((d.cache.lens == a.context + 1).all()), "a request has not the keys it should have"
        graph = d.graph()
        graph.replay()
        assert torch.equal(d.out, eager), "the graph's step differs"
        print("%s: %d layers, %d tokens: %.0f us a step, %.0f from a graph"
              % (what, a.layers, a.tokens, timed(d.step, 50), timed(graph.replay, 50)), flush=True)

    decode("decode", Decoder(a.layers, a.tokens, a.hidden, a.inner, a.experts, a.top_k))
    if a.heads:  # each token a request of its own, after `context` others
        width = a.context // a.page + 1
        cache = Cache(a.layers, a.tokens, a.tokens, width, a.tokens * width, a.page, a.kv_heads, a.head, most=1)
        for t in (cache.k, cache.v):
            t.normal_(generator=g)
        cache.fresh.fill_(1)
        for _ in range(a.context):  # a step has room for a token of each
            cache.tables()
            cache.advance()
        decode("decode with attention over %d keys" % (a.context + 1),
               Decoder(a.layers, a.tokens, a.hidden, a.inner, a.experts, a.top_k, heads=a.heads, cache=cache, window=a.window))
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
