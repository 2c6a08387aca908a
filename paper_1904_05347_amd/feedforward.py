"""A feed-forward layer on 8-bit integers: the 8-bit operators as a network uses them.

    h = x + residual
    n = h * norm / sqrt(mean(h^2) + eps)           rmsnorm_i8: to 8 bits, a scale for each token
    p = n [gate; up]^T                             gemm_i8
    y = (act(p_gate) * p_up) down^T                gated_i8, gemm_i8

The weights are taken to 8 bits once, with a scale for each output channel
(``quantize_i8``); the activations at every call, with a scale for each token.
``python -m paper_1904_05347_amd.feedforward`` times the layer for one token and
for prompts, and compares it with the same layer in float64.
"""
from __future__ import annotations

import argparse

from . import binding as pk


class FeedForwardI8:
    """norm: D; gate, up: F x D; down: D x F (float32, bfloat16 or float16, on a HIP device)."""

    def __init__(self, norm, gate, up, down, activation="silu", eps=1e-6):
        import torch
        if gate.shape != up.shape or down.shape != gate.shape[::-1] or norm.shape != gate.shape[1:]:
            raise ValueError("gate and up are F x D, down is D x F, norm is D")
        self.norm, self.activation, self.eps = norm, activation, eps
        self.width = gate.size(0)
        # one product for gate and up
        self.first, self.first_scale = pk.quantize_i8(torch.cat((gate, up)))
        self.second, self.second_scale = pk.quantize_i8(down)

    def __call__(self, x, residual=None):
        """(y, h) for x of tokens x D: y in x's type, h = x + residual the new residual stream."""
        q, scale, h = pk.rmsnorm_i8(x, self.norm, residual=residual, eps=self.eps)
        p = pk.gemm_i8(q, self.first, scale, self.first_scale, dtype=x.dtype)
        q, scale = pk.gated_i8(p[:, :self.width], p[:, self.width:], activation=self.activation)
        return pk.gemm_i8(q, self.second, scale, self.second_scale, dtype=x.dtype), h


def reference(x, residual, norm, gate, up, down, activation="silu", eps=1e-6):
    """The same layer in float64, from weights that are not quantised."""
    import torch
    h = x.double() + (0 if residual is None else residual.double())
    n = h * norm.double() / torch.sqrt(h.square().mean(dim=1, keepdim=True) + eps)
    g, u = n @ gate.double().t().contiguous(), n @ up.double().t().contiguous()
    act = torch.nn.functional.silu(g) if activation == "silu" else torch.nn.functional.gelu(g, approximate="tanh")
    return (act * u) @ down.double().t().contiguous(), h


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description="times a feed-forward layer on 8-bit integers")
    ap.add_argument("--tokens", type=int, nargs="+", default=[1, 32, 512, 4096])
    ap.add_argument("--dim", type=int, default=4096)
    ap.add_argument("--width", type=int, default=8192)
    ap.add_argument("--activation", choices=sorted(pk.ACTIVATIONS), default="silu")
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

    norm = 1 + normal(a.dim, scale=0.1)
    gate, up = normal(a.width, a.dim, scale=a.dim ** -0.5), normal(a.width, a.dim, scale=a.dim ** -0.5)
    down = normal(a.dim, a.width, scale=a.width ** -0.5)
    layer = FeedForwardI8(norm, gate, up, down, a.activation)
    for tokens in a.tokens:
        x, r = normal(tokens, a.dim, scale=0.5), normal(tokens, a.dim)
        y, _ = layer(x, r)
        want, _ = reference(x[:64], r[:64], norm, gate, up, down, a.activation)
        off = float((y[:64].double() - want).norm() / want.norm())
        # the layer's launches as a graph, as a serving loop replays them
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(x, r)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        # until times are steady: the first of a run would come out a fifth too long
        for _ in range(500):
            graph.replay()
        start.record()
        for _ in range(100):
            graph.replay()
        end.record()
        torch.cuda.synchronize()
        us = start.elapsed_time(end) / 100 * 1e3
        print("%5d tokens, %d -> 2 x %d -> %d: %8.1f us, %7.1f TOP/s, %.3g off float64"
              % (tokens, a.dim, a.width, a.dim, us, 6e-6 * tokens * a.dim * a.width / us, off), flush=True)


if __name__ == "__main__":
    main()
