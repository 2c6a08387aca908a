"""The attention layer that runs the attention operators between the 8-bit products."""
import pytest

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _case(torch, pk, kind, D, H, K, d, lengths, tokens, page, turned, normed, layout="half", cap=0.0):
    from paper_1904_05347_amd.attention import AttentionI8
    g = torch.Generator(device="cuda").manual_seed(D + H)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(kind)

    weights = [1 + normal(D, scale=0.1)] + [normal(h * d, D, scale=D ** -0.5) for h in (H, K, K)] + [normal(D, H * d, scale=(H * d) ** -0.5)]
    norms = [1 + normal(d, scale=0.1) for _ in range(2)] if normed else [None, None]
    layer = AttentionI8(*weights, H, K, *norms, pk.rope_frequencies(d // 4) if turned else None, layout=layout, cap=cap)
    need = [-(-(n + t) // page) for n, t in zip(lengths, tokens)]
    pages = sum(need) + 1
    key, value = normal(pages, page, K, d), normal(pages, page, K, d)
    order, table, at = torch.randperm(pages, generator=g, device="cuda").int(), torch.zeros((len(lengths), max(need)), dtype=torch.int32, device="cuda"), 0
    slots, positions, starts = [], [], [0]
    for b, (n, t) in enumerate(zip(lengths, tokens)):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        starts.append(starts[-1] + t)
        for i in range(t):
            positions.append(n + i)
            slots.append(int(table[b, (n + i) // page]) * page + (n + i) % page)
    i64 = dict(dtype=torch.int64, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    M = starts[-1]
    return (layer, weights, normal(M, D, scale=0.5), normal(M, D), key, value, torch.tensor(slots, **i64), torch.tensor(positions, **i64), table,
            torch.tensor(lengths, **i32), torch.tensor(starts, **i32), max(tokens))


@pytest.mark.parametrize("kind,D,H,K,d,lengths,tokens,page,turned,normed,layout,cap", [
    ("bfloat16", 512, 8, 2, 64, [70, 300], [1, 1], 16, True, True, "half", 0.0),
    ("float16", 333, 6, 3, 80, [5, 0, 129], [4, 2, 7], 24, True, False, "interleaved", 30.0),
    ("float32", 256, 4, 4, 36, [33], [9], 5, False, True, "half", 0.0)])
def test_layer(kind, D, H, K, d, lengths, tokens, page, turned, normed, layout, cap):
    """Against float64 with the weights as they were.  Each 8-bit product is 1.7 % off (1.2 % for either
    operand's rounding of normal rows).  Of queries and keys that moves a score by 0.024 (|q| = |k| =
    sqrt(d), scale d^-1/2; 1.7 % of either, in any direction), so a weight by 2.4 %; the values are 1.7 %
    off: 2.9 % of o.  Its own product adds 1.7 %: 3.4 %, and storage in 16 bits 0.4 % for each of three
    steps: 3.5 %."""
    torch, pk = require_gpu()
    from paper_1904_05347_amd.attention import reference
    layer, weights, x, r, key, value, slots, positions, table, n, starts, most = _case(
        torch, pk, getattr(torch, kind), D, H, K, d, lengths, tokens, page, turned, normed, layout, cap)
    for residual in (r, None):
        want, want_h = reference(layer, weights, x, key, value, positions, table, n, starts, residual=residual)
        key2, value2 = key.clone(), value.clone()
        y, h = layer(x, key2, value2, slots, positions, table, n, starts, most, residual=residual)
        assert y.dtype == x.dtype and y.shape == x.shape
        assert float((y.double() - want).norm() / want.norm()) < 0.05
        assert torch.equal(h, x if residual is None else (x.float() + r.float()).to(x.dtype))
        # what the cache got, and nothing else
        kept = torch.ones(key.size(0) * page, dtype=torch.bool, device="cuda")
        kept[slots] = False
        assert torch.equal(key2.flatten(0, 1)[kept], key.flatten(0, 1)[kept]) and torch.equal(value2.flatten(0, 1)[kept], value.flatten(0, 1)[kept])
        # bit for bit the operators one by one, on tensors of their own
        q8, s, _ = pk.rmsnorm_i8(x, layer.norm, residual=residual)
        p = pk.gemm_i8(q8, layer.first, s, layer.first_scale, dtype=x.dtype)
        q, k, v = (t.contiguous().view(len(x), -1, d) for t in p.split([H * d, K * d, K * d], dim=1))
        qr, kr = pk.rope_qk(q, k, positions if turned else None, layer.frequencies, layer.q_norm, layer.k_norm, layout=layout)
        assert torch.equal(key2.flatten(0, 1)[slots], kr) and torch.equal(value2.flatten(0, 1)[slots], v)
        o = pk.attention_tree(qr, key2, value2, table, n, starts, most, cap=cap)
        q8, s = pk.quantize_i8(o.view(len(x), -1))
        assert torch.equal(y, pk.gemm_i8(q8, layer.second, s, layer.second_scale, dtype=x.dtype))


def test_graph_of_the_layer():
    """Captured once, replayed while sequences grow."""
    torch, pk = require_gpu()
    layer, _, x, _, key, value, slots, positions, table, n, starts, most = _case(
        torch, pk, torch.bfloat16, 256, 4, 2, 64, [100, 40], [1, 1], 16, True, True)
    layer(x, key, value, slots, positions, table, n, starts, most)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = layer(x, key, value, slots, positions, table, n, starts, most)
    for step in range(4):
        x.copy_(torch.randn_like(x))
        before = key.clone(), value.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        key2, value2 = before
        want, _ = layer(x, key2, value2, slots, positions, table, n, starts, most)
        assert torch.equal(got, want) and torch.equal(key, key2) and torch.equal(value, value2), step
        n.add_(1), positions.add_(1)
        slots.copy_(torch.gather(table.long(), 1, (n.long() // 16)[:, None])[:, 0] * 16 + n.long() % 16)


def test_shapes_are_checked():
    torch, pk = require_gpu()
    from paper_1904_05347_amd.attention import AttentionI8
    one = torch.ones
    for norm, wq, wk, wv, wo, H, K in (((8,), (32, 8), (16, 8), (16, 8), (8, 16), 4, 2), ((8,), (32, 8), (16, 8), (8, 8), (8, 32), 4, 2),
                                       ((7,), (32, 8), (16, 8), (16, 8), (8, 32), 4, 2), ((8,), (32, 8), (24, 8), (24, 8), (8, 32), 4, 3)):
        with pytest.raises(ValueError):
            AttentionI8(*(one(s, device="cuda") for s in (norm, wq, wk, wv, wo)), H, K)


def test_command(capsys):
    require_gpu()
    from paper_1904_05347_amd import attention
    attention.main(["--sequences", "1", "3", "--tokens", "1", "5", "--length", "100", "--dim", "256", "--heads", "4", "--kv-heads", "2", "--size", "64"])
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 4 and all("off float64" in line for line in lines)
