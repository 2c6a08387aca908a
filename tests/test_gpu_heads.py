"""rope_qk, rope_qk_backward and cache_append on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

KINDS = ("f32", "bf16", "f16")


def _type(torch, kind):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]


def _f64(t):
    return t.detach().double().cpu().numpy()


def _normal(torch, g, shape, kind, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(_type(torch, kind))


def _inputs(torch, seed, M, Hq, Hk, d, kind, fused=True):
    """Queries, keys and values as views of one projection's output, with a few spare columns."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if not fused:
        return (g,) + tuple(_normal(torch, g, (M, h, d), kind) for h in (Hq, Hk, Hk))
    p = _normal(torch, g, (M, (Hq + 2 * Hk) * d + 3), kind)
    cut = [0, Hq * d, (Hq + Hk) * d, (Hq + 2 * Hk) * d]
    return (g,) + tuple(p[:, a:b].unflatten(1, (-1, d)) for a, b in zip(cut, cut[1:]))


# tokens, query heads, key heads, channels, pairs: one lane to a head, whole waves of lanes, odd channels,
# part of a head rotated, tokens that share a work-group, heads that need several rounds
SHAPES = [(1, 1, 1, 1, 0), (3, 1, 1, 2, 1), (5, 2, 1, 7, 3), (2, 3, 1, 16, 8), (130, 1, 1, 8, 2), (4, 32, 8, 128, 64),
          (7, 12, 3, 80, 20), (3, 5, 5, 50, 25), (2, 70, 10, 128, 32), (3, 8, 2, 256, 128), (2, 9, 3, 255, 127),
          (5, 4, 2, 96, 0), (2, 200, 1, 64, 32), (1, 130, 2, 200, 33)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rope(shape, layout, kind):
    torch, pk = require_gpu()
    M, Hq, Hk, d, pairs = shape
    g, q, k, _ = _inputs(torch, M + d, M, Hq, Hk, d, kind)
    f = pk.rope_frequencies(pairs)
    positions = torch.randint(-50, 1 << 20, (M,), generator=g, device="cuda")
    for wkind in (None, kind, "f32"):
        qw = None if wkind is None else _normal(torch, g, (d,), wkind) + 1
        for kw, amplitude in ((qw, 1.0), (None, -0.75)):
            oq, ok = pk.rope_qk(q, k, positions, f, qw, kw, eps=1e-5, layout=layout, amplitude=amplitude)
            for x, w, y, what in ((q, qw, oq, "q"), (k, kw, ok, "k")):
                want, bound = plain.rope(_f64(x), positions.cpu().numpy(), _f64(f), None if w is None else _f64(w), 1e-5, layout,
                                         amplitude, kind)
                assert y.dtype == x.dtype and y.shape == x.shape
                plain.check(_f64(y), want, bound, "%s %s" % (what, wkind))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shape", SHAPES)
def test_rope_backward(shape, layout, kind):
    torch, pk = require_gpu()
    M, Hq, Hk, d, pairs = shape
    g, q, k, _ = _inputs(torch, M + d, M, Hq, Hk, d, kind)
    dq, dk = _normal(torch, g, (M, Hq, d), kind), _normal(torch, g, (M, Hk, d), kind)
    f = pk.rope_frequencies(pairs)
    positions = torch.randint(0, 5000, (M,), generator=g, device="cuda")
    for wkind in (None, kind, "f32"):
        w = None if wkind is None else _normal(torch, g, (d,), wkind) + 1
        for qw, kw, amplitude in ((w, w, 1.0), (w, None, 1.25), (None, w, 1.0)):
            gq, gk, gqw, gkw = pk.rope_qk_backward(dq, dk, q, k, positions, f, qw, kw, eps=1e-5, layout=layout, amplitude=amplitude)
            for dy, x, v, gx, gw, what in ((dq, q, qw, gq, gqw, "q"), (dk, k, kw, gk, gkw, "k")):
                want, bound, wdw, wbound = plain.rope_backward(_f64(dy), _f64(x), positions.cpu().numpy(), _f64(f),
                                                               None if v is None else _f64(v), 1e-5, layout, amplitude, kind, wkind)
                assert gx.dtype == dy.dtype and gx.shape == dy.shape
                plain.check(_f64(gx), want, bound, what)
                if v is None:
                    assert gw is None
                else:
                    assert gw.dtype == v.dtype
                    plain.check(_f64(gw), wdw, wbound, what + " weight")


def test_backward_of_many_tokens():
    """More tokens than work-groups.  A lane adds 5 rows of 8 tokens more than a sum of 1024 tokens has steps."""
    torch, pk = require_gpu()
    M, d = 9001, 32
    g, q, k, _ = _inputs(torch, 9, M, 3, 2, d, "f32")
    dq, dk = _normal(torch, g, (M, 3, d), "f32"), _normal(torch, g, (M, 2, d), "f32")
    w, f = _normal(torch, g, (d,), "f32"), pk.rope_frequencies(16)
    positions = torch.arange(M, device="cuda")
    first = pk.rope_qk_backward(dq, dk, q, k, positions, f, w, w)
    again = pk.rope_qk_backward(dq, dk, q, k, positions, f, w, w)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    for dy, x, gx, gw in ((dq, q, first[0], first[2]), (dk, k, first[1], first[3])):
        want, bound, wdw, wbound = plain.rope_backward(_f64(dy), _f64(x), positions.cpu().numpy(), _f64(f), _f64(w), 1e-6, "half",
                                                       1.0, "f32", "f32")
        plain.check(_f64(gx), want, bound, "x")
        plain.check(_f64(gw), wdw, wbound * (160 + 33 + 40) / (160 + 33), "weight")


def test_gradient_against_differences():
    """Of the operator itself: (L(x + h e) - L(x - h e)) / 2h for L = sum of y times dy, in fp32.  With
    |y| of about 1, 2 heads of 12 channels and h = 2^-5, the sum's rounding (24 terms off by 32 u each, over 2h: 1e-3) and
    the third derivative's share (h^2 / 6 times at most 30 for |x| near 1: 5e-3) stay below 1e-2."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.rand((1, 2, 12), generator=g, device="cuda") + 0.5
    dq, w = torch.rand(q.shape, generator=g, device="cuda") - 0.5, torch.rand(12, generator=g, device="cuda") + 0.5
    f, positions, h = pk.rope_frequencies(4), torch.tensor([5], device="cuda"), 2.0 ** -5

    def loss(x, weight):
        return float((pk.rope_qk(x, None, positions, f, weight)[0].double() * dq.double()).sum())

    gq, _, gw, _ = pk.rope_qk_backward(dq, None, q, None, positions, f, w)
    for i in range(24):
        e = torch.zeros(24, device="cuda")
        e[i] = h
        e = e.view(q.shape)
        assert abs((loss(q + e, w) - loss(q - e, w)) / (2 * h) - float(gq.view(-1)[i])) < 1e-2
    for i in range(12):
        e = torch.zeros(12, device="cuda")
        e[i] = h
        assert abs((loss(q, w + e) - loss(q, w - e)) / (2 * h) - float(gw[i])) < 1e-2


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-21, 1e18, 1e30, 1e37])
def test_rows_at_the_ends_of_the_range(scale):
    """The mean neither overflows nor underflows, whatever the others in a wave are."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((6, 4, 32), generator=g, device="cuda")
    q[1::2] *= scale
    q[2, 1] = 0
    w = torch.ones(32, device="cuda")
    for eps in (0.0, 1e-6):
        y, _ = pk.rope_qk(q, None, None, None, w, eps=eps)
        x = _f64(q)
        with np.errstate(invalid="ignore"):
            want, bound = plain.rope(x, None, np.zeros(0), _f64(w), eps, "half", 1.0, "f32")
        # an eps is held in 32 bits; subnormal inputs are what they are
        plain.check(_f64(y), want, bound + 2 * plain.U * np.abs(want), "scale %g" % scale)


def test_infinities_and_nan_stay_in_their_rows():
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((4, 8, 64), generator=g, device="cuda").bfloat16()
    w, f, positions = torch.ones(64, device="cuda").bfloat16(), pk.rope_frequencies(32), torch.arange(4, device="cuda")
    clean, _ = pk.rope_qk(q, None, positions, f, w)
    q[1, 3, 5], q[2, 0, 7] = float("nan"), float("inf")
    y, _ = pk.rope_qk(q, None, positions, f, w)
    hit = torch.zeros((4, 8), dtype=torch.bool, device="cuda")
    hit[1, 3] = hit[2, 0] = True
    assert torch.equal(y[~hit], clean[~hit])
    assert y[1, 3].isnan().all() and y[2, 0, 7].isnan()


def test_positions_far_and_before():
    torch, pk = require_gpu()
    positions = torch.tensor([0, 1, -1, 4096, (1 << 31) + 5, 1 << 40, -(1 << 40) + 3], device="cuda")
    g, q, k, _ = _inputs(torch, 3, len(positions), 2, 1, 64, "f32")
    f = pk.rope_frequencies(32)
    oq, ok = pk.rope_qk(q, k, positions, f)
    for x, y in ((q, oq), (k, ok)):
        # the angle's own 64 bits: two roundings of 2^-53 of up to 2^40 radians
        want, bound = plain.rope(_f64(x), positions.cpu().numpy(), _f64(f), None, 0, "half", 1.0, "f32")
        _, size = plain.rotate(_f64(x), positions.cpu().numpy(), _f64(f), "half", 1.0)
        angle = np.abs(positions.cpu().numpy().astype(np.float64))[:, None, None] * 2.0 ** -51
        plain.check(_f64(y), want, bound + size * angle, "far")


def test_in_place_strided_and_one_side():
    torch, pk = require_gpu()
    for kind in KINDS:
        g, q, k, _ = _inputs(torch, 5, 9, 6, 2, 48, kind)
        f, positions = pk.rope_frequencies(24), torch.arange(9, device="cuda") * 7
        w = _normal(torch, g, (48,), kind)
        want = pk.rope_qk(q, k, positions, f, w, w)
        alone, none = pk.rope_qk(k, None, positions, f, w)
        assert none is None and torch.equal(alone, want[1])
        # heads before tokens, a spare channel between heads
        wide = torch.zeros((6, 9, 49), dtype=q.dtype, device="cuda")
        turned = wide[:, :, :48].transpose(0, 1)
        out = pk.rope_qk(q, None, positions, f, w, q_out=turned)[0]
        assert out is turned and torch.equal(turned, want[0]) and not wide[:, :, 48].any()
        # one row for all tokens, without copying it
        same = pk.rope_qk(q[:1].expand(9, 6, 48), None, positions, f, w)[0]
        assert torch.equal(same, pk.rope_qk(q[:1].repeat(9, 1, 1), None, positions, f, w)[0])
        got = pk.rope_qk(q, k, positions, f, w, w, q_out=q, k_out=k)
        assert got[0] is q and got[1] is k and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_no_tokens():
    torch, pk = require_gpu()
    f, positions = pk.rope_frequencies(4), torch.zeros(0, dtype=torch.int64, device="cuda")
    q, k, w = torch.ones((0, 4, 8), device="cuda"), torch.ones((0, 2, 8), device="cuda"), torch.ones(8, device="cuda")
    assert pk.rope_qk(q, k, positions, f, w, w)[1].shape == (0, 2, 8)
    grads = pk.rope_qk_backward(q, k, q, k, positions, f, w, w)
    assert not grads[2].any() and not grads[3].any() and grads[2].shape == (8,)
    kc, vc = torch.ones((2, 4, 2, 8), device="cuda"), torch.ones((2, 4, 2, 8), device="cuda")
    assert pk.cache_append(k, k, kc, vc, positions) is None


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_append(shape, kind):
    torch, pk = require_gpu()
    M, Hq, Hk, d, pairs = shape
    g, q, k, v = _inputs(torch, M + d + 1, M, Hq, Hk, d, kind)
    f = pk.rope_frequencies(pairs)
    positions = torch.randint(0, 1 << 17, (M,), generator=g, device="cuda")
    page, pages = 5, M // 5 + 3
    w = _normal(torch, g, (d,), kind)
    for kw, layout in ((w, "half"), (None, "interleaved")):
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:M].contiguous()
        if M > 2:
            slots[1], slots[M // 2] = -1, pages * page + (1 << 40)
        stores = [torch.full((pages, page, Hk, d), 3.0, dtype=q.dtype, device="cuda"),
                  torch.full((pages, Hk, page, d + 1), 3.0, dtype=q.dtype, device="cuda")[..., :d].transpose(1, 2)]
        for kc, vc in (stores, stores[::-1], (torch.full((pages, page, 2, Hk, d), 3.0, dtype=q.dtype, device="cuda").unbind(2))):
            kc.fill_(3.0), vc.fill_(3.0)
            oq = pk.cache_append(k, v, kc, vc, slots, positions, f, kw, q=q, q_weight=kw, layout=layout)
            want_q, want_k = pk.rope_qk(q, k, positions, f, kw, kw, layout=layout)
            assert torch.equal(oq, want_q)
            wk, wv = torch.full_like(kc, 3.0), torch.full_like(vc, 3.0)
            for m, s in enumerate(slots.tolist()):
                if 0 <= s < pages * page:
                    wk[s // page, s % page], wv[s // page, s % page] = want_k[m], v[m]
            assert torch.equal(kc, wk) and torch.equal(vc, wv)
            kc.fill_(3.0), vc.fill_(3.0)
            assert pk.cache_append(k, v, kc, vc, slots, positions, f, kw, layout=layout) is None
            assert torch.equal(kc, wk) and torch.equal(vc, wv)


def test_append_copies_values_bit_for_bit_beyond_4_gib():
    """A cache whose last pages lie past 2^32 elements, and NaN and infinities among the values."""
    torch, pk = require_gpu()
    pages, page, d = (1 << 32) // (16 * 64) + 8, 16, 64
    kc = torch.empty((pages, page, 1, d), dtype=torch.float16, device="cuda")
    vc = torch.empty_like(kc)
    k = torch.randn((3, 1, d), device="cuda").half()
    v = torch.randint(-(1 << 15), 1 << 15, (3, 1, d), device="cuda", dtype=torch.int16).view(torch.float16)
    slots = torch.tensor([pages * page - 1, 3, pages * page - 40], device="cuda")
    around = (slots[0] - 1, slots[2] + 1)
    flat_k, flat_v = kc.view(-1, 1, d), vc.view(-1, 1, d)
    for s in around:
        flat_k[s] = 1
        flat_v[s] = 2
    pk.cache_append(k, v, kc, vc, slots)
    assert torch.equal(flat_k[slots], k) and torch.equal(flat_v[slots].view(torch.int16), v.view(torch.int16))
    assert all(bool((flat_k[s] == 1).all()) and bool((flat_v[s] == 2).all()) for s in around)


def test_frequencies():
    torch, pk = require_gpu()
    f = pk.rope_frequencies(8, base=500.0)
    assert f.dtype == torch.float64 and f.is_cuda
    assert np.allclose(_f64(f), 500.0 ** (-np.arange(8) / 8), rtol=1e-14)
    assert np.allclose(_f64(pk.rope_frequencies(8, base=500.0, factor=4.0)), _f64(f) / 4, rtol=1e-14)


def test_streams_and_graph():
    """On a stream of their own, and captured and replayed with other inputs between."""
    torch, pk = require_gpu()
    g, q, k, v = _inputs(torch, 8, 33, 8, 2, 64, "bf16", fused=False)
    f, positions = pk.rope_frequencies(32), torch.arange(33, device="cuda")
    w = _normal(torch, g, (64,), "bf16")
    kc = torch.zeros((9, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    vc, slots = torch.zeros_like(kc), torch.randperm(36, generator=g, device="cuda")[:33].contiguous()
    dq, dk = torch.randn_like(q), torch.randn_like(k)

    def step():
        out = pk.cache_append(k, v, kc, vc, slots, positions, f, w, q=q, q_weight=w)
        return (out, kc, vc) + pk.rope_qk_backward(dq, dk, q, k, positions, f, w, w)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = [t.clone() for t in step()]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        for t in (q, k, v, dq, dk):
            t.copy_(torch.randn_like(t))
        positions.add_(i)
        kc.zero_(), vc.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        kc.zero_(), vc.zero_()
        assert all(torch.equal(a, b) for a, b in zip(got, step())), i
