"""An attention layer on 8-bit integers over a paged cache: the attention operators as a
network uses them, between the same products as the feed-forward layer's.

    h = x + residual
    n = h * norm / sqrt(mean(h^2) + eps)           rmsnorm_i8: to 8 bits, a scale for each token
    q, k, v = n [wq; wk; wv]^T                     gemm_i8
    q, k normed by head and rotated, k and v to their places in the cache
                                                   cache_append
    o = attention of each sequence's new tokens over its cache
                                                   attention_tree
    y = o wo^T                                     quantize_i8, gemm_i8

New tokens are one, a chain or a tree of drafted ones for each sequence.
``python -m paper_1904_05347_amd.attention`` times the layer for sequences that generate
together, and compares it with the same layer in float64.
"""
from __future__ import annotations

import argparse

from . import binding as pk


class AttentionI8:
    """norm: D; wq: Hq d x D; wk, wv: Hk d x D; wo: D x Hq d (float32, bfloat16 or float16, on a
    HIP device); q_norm, k_norm: d, the heads' norms, or None; frequencies: as
    ``rope_frequencies`` gives them, or None."""

    def __init__(self, norm, wq, wk, wv, wo, heads, kv_heads, q_norm=None, k_norm=None, frequencies=None, layout="half",
                 amplitude=1.0, scale=None, cap=0.0, eps=1e-6):
        import torch
        self.size = wq.size(0) // heads if heads else 0
        rows = tuple((h * self.size, norm.size(0)) for h in (heads, kv_heads, kv_heads))
        if norm.dim() != 1 or heads < 1 or kv_heads < 1 or heads % kv_heads or \
                tuple(tuple(w.shape) for w in (wq, wk, wv)) != rows or tuple(wo.shape) != rows[0][::-1]:
            raise ValueError("wq is heads * size x D, wk and wv are kv_heads * size x D, wo is D x heads * size, norm is D")
        self.norm, self.heads, self.kv_heads, self.q_norm, self.k_norm = norm, heads, kv_heads, q_norm, k_norm
        self.frequencies, self.layout, self.amplitude = frequencies, layout, amplitude
        self.scale, self.cap, self.eps = scale, cap, eps
        # one product for queries, keys and values
        self.first, self.first_scale = pk.quantize_i8(torch.cat((wq, wk, wv)))
        self.second, self.second_scale = pk.quantize_i8(wo)

    def __call__(self, x, key_cache, value_cache, slots, positions, page_table, lengths, starts, most, mask=None, residual=None):
        """(y, h) for x of tokens x D: y in x's type, h = x + residual the new residual stream.
        The tokens' keys and values are in the cache afterwards; the arguments of the cache are
        those of ``cache_append`` and ``attention_tree``."""
        M, a, b = x.size(0), self.heads * self.size, (self.heads + self.kv_heads) * self.size
        q8, scale, h = pk.rmsnorm_i8(x, self.norm, residual=residual, eps=self.eps)
        p = pk.gemm_i8(q8, self.first, scale, self.first_scale, dtype=x.dtype)
        q, k, v = (t.view(M, -1, self.size) for t in (p[:, :a], p[:, a:b], p[:, b:]))
        turned = self.frequencies is not None
        pk.cache_append(k, v, key_cache, value_cache, slots, positions if turned else None, self.frequencies, self.k_norm, q=q,
                        q_weight=self.q_norm, eps=self.eps, layout=self.layout, amplitude=self.amplitude, q_out=q)
        o = pk.attention_tree(q, key_cache, value_cache, page_table, lengths, starts, most, mask=mask, scale=self.scale, cap=self.cap)
        q8, scale = pk.quantize_i8(o.view(M, a))
        return pk.gemm_i8(q8, self.second, scale, self.second_scale, dtype=x.dtype), h


def reference(layer, weights, x, key_cache, value_cache, positions, page_table, lengths, starts, mask=None, residual=None):
    """The same layer in float64, from weights (norm, wq, wk, wv, wo) that are not quantised and the
    cache as it was before the call."""
    import torch
    norm, wq, wk, wv, wo = (w.double() for w in weights)
    H, K, d = layer.heads, layer.kv_heads, layer.size
    h = x.double() + (0 if residual is None else residual.double())
    n = h * norm / torch.sqrt(h.square().mean(dim=1, keepdim=True) + layer.eps)
    q, k, v = ((n @ w.t().contiguous()).view(x.size(0), -1, d) for w in (wq, wk, wv))

    def turned(t, weight):
        if weight is not None:
            t = t * weight.double() / torch.sqrt(t.square().mean(dim=-1, keepdim=True) + layer.eps)
        if layer.frequencies is None:
            return t
        r = layer.frequencies.numel()
        angle = (positions.double()[:, None] * layer.frequencies)[:, None]
        i = torch.arange(r, device=t.device)
        a, b = (i, i + r) if layer.layout == "half" else (2 * i, 2 * i + 1)
        out = t.clone()
        out[..., a] = layer.amplitude * (t[..., a] * angle.cos() - t[..., b] * angle.sin())
        out[..., b] = layer.amplitude * (t[..., b] * angle.cos() + t[..., a] * angle.sin())
        return out

    q, k = turned(q, layer.q_norm), turned(k, layer.k_norm)
    o = torch.zeros_like(q)
    page = key_cache.size(1)
    for b, (n_past, m0, m1) in enumerate(zip(lengths.tolist(), starts.tolist(), starts.tolist()[1:])):
        pages = page_table[b, :-(-n_past // page)].long()
        keys = torch.cat((key_cache[pages].reshape(-1, K, d)[:n_past].double(), k[m0:m1])).repeat_interleave(H // K, dim=1)
        values = torch.cat((value_cache[pages].reshape(-1, K, d)[:n_past].double(), v[m0:m1])).repeat_interleave(H // K, dim=1)
        for i in range(m1 - m0):
            word = (2 << i) - 1 if mask is None else int(mask[m0 + i])
            seen = torch.tensor([True] * n_past + [bool(word >> e & 1) for e in range(m1 - m0)], device=x.device)
            score = (keys[seen] * q[m0 + i]).sum(-1) * (d ** -0.5 if layer.scale is None else layer.scale)
            if layer.cap:
                score = layer.cap * torch.tanh(score / layer.cap)
            o[m0 + i] = (torch.softmax(score, dim=0)[..., None] * values[seen]).sum(0)
    return o.reshape(x.size(0), H * d) @ wo.t().contiguous(), h


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description="times an attention layer on 8-bit integers over a paged cache")
    ap.add_argument("--sequences", type=int, nargs="+", default=[1, 32])
    ap.add_argument("--tokens", type=int, nargs="+", default=[1, 8], help="new tokens of each sequence, a chain")
    ap.add_argument("--length", type=int, default=4096, help="positions in the cache before them")
    ap.add_argument("--dim", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--size", type=int, default=128, help="channels of a head")
    ap.add_argument("--page", type=int, default=16, help="positions of a page")
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

    rows = (a.heads * a.size, a.kv_heads * a.size, a.kv_heads * a.size)
    weights = [1 + normal(a.dim, scale=0.1)] + [normal(r, a.dim, scale=a.dim ** -0.5) for r in rows]
    weights.append(normal(a.dim, rows[0], scale=rows[0] ** -0.5))
    layer = AttentionI8(*weights, a.heads, a.kv_heads, 1 + normal(a.size, scale=0.1), 1 + normal(a.size, scale=0.1),
                        pk.rope_frequencies(a.size // 2))
    for B in a.sequences:
        for T in a.tokens:
            P = -(-(a.length + T) // a.page)
            key, value = (normal(B * P, a.page, a.kv_heads, a.size) for _ in range(2))
            table = torch.randperm(B * P, generator=g, device="cuda").int().view(B, P)
            at = (a.length + torch.arange(T, device="cuda")).repeat(B, 1)
            slots = (torch.gather(table.long(), 1, at // a.page) * a.page + at % a.page).view(-1)
            x, r = normal(B * T, a.dim, scale=0.5), normal(B * T, a.dim)
            lengths = torch.full((B,), a.length, dtype=torch.int32, device="cuda")
            starts = T * torch.arange(B + 1, dtype=torch.int32, device="cuda")
            args = (x, key, value, slots, at.view(-1), table, lengths, starts, T)
            n = min(B, 2)
            want, _ = reference(layer, weights, x[:n * T], key, value, at.view(-1)[:n * T], table[:n], lengths[:n], starts[:n + 1],
                                residual=r[:n * T])
            y, _ = layer(*args, residual=r)
            off = float((y[:n * T].double() - want).norm() / want.norm())
            # the layer's launches as a graph, as a serving loop replays them
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                layer(*args, residual=r)
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
            print("%3d sequences of %d tokens over %d positions, %d heads of %d over %d: %8.1f us, %.3g off float64"
                  % (B, T, a.length, a.heads, a.size, a.kv_heads, us, off), flush=True)


if __name__ == "__main__":
    main()
