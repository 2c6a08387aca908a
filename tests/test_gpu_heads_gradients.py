"""rope_qk_backward where its forms change: rows at the ends of the range beside ordinary ones, and tokens of many
heads, several rounds of a work-group each, more of them than work-groups."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu
from tests.test_gpu_heads import KINDS, _f64, _inputs, _normal

pytestmark = pytest.mark.gpu


def _compare(dys, xs, ws, grads, weight_grads, positions, f, eps, layout, amplitude, kind, wkind, what):
    eps = float(np.float32(eps))
    for dy, x, w, gx, gw, side in zip(dys, xs, ws, grads, weight_grads, "qk"):
        want, bound, wdw, wbound = plain.rope_backward(_f64(dy), _f64(x), positions, f, None if w is None else _f64(w), eps, layout,
                                                       amplitude, kind, wkind)
        plain.check(_f64(gx), want, bound, "%s %s" % (what, side))
        if w is None:
            assert gw is None
        else:
            plain.check(_f64(gw), wdw, wbound, "%s %s weight" % (what, side))


# of the odd rows, and of their gradients, such that all results are numbers of the type
@pytest.mark.parametrize("scale,of_gradient", [(1e-38, 1e-8), (1e-30, 1e-5), (1e-21, 1.0), (1e-13, 1.0), (1e17, 1.0), (1e18, 1.0), (1e30, 1e5),
                                               (1e37, 1e6)])
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-6])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_at_the_ends_of_the_range(kind, eps, scale, of_gradient):
    torch, pk = require_gpu()
    for d, pairs, layout in ((32, 0, "half"), (50, 20, "interleaved"), (128, 64, "half")):
        g, q, k, _ = _inputs(torch, 7 + d, 9, 4, 2, d, "f32", fused=False)
        dq, dk = _normal(torch, g, q.shape, "f32"), _normal(torch, g, k.shape, "f32")
        for t, s in ((q, scale), (k, scale), (dq, of_gradient), (dk, of_gradient)):
            t[1::2] *= s
            t[4, 1] *= s
        if eps > 1e-30:
            q[2, 1] = 0
        dt = torch.float32 if kind == "f32" else torch.bfloat16
        q, k, dq, dk = (t.to(dt) for t in (q, k, dq, dk))
        w = _normal(torch, g, (d,), kind) + 1
        f, positions = pk.rope_frequencies(pairs), torch.arange(9, device="cuda") * 11
        gq, gk, gqw, gkw = pk.rope_qk_backward(dq, dk, q, k, positions, f, w, w, eps=eps, layout=layout)
        _compare((dq, dk), (q, k), (w, w), (gq, gk), (gqw, gkw), positions.cpu().numpy(), _f64(f), eps, layout, 1.0, kind, kind,
                 "d %d scale %g" % (d, scale))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", [(1500, 70, 10, 128, 24), (1100, 100, 3, 96, 48), (700, 260, 2, 33, 0), (1300, 40, 40, 200, 77)])
def test_many_tokens_of_many_heads(shape, kind):
    """A lane adds up to 3 tokens' rows of several rounds, and there are 6 steps over lanes, 8 waves and 8 + 16 work-groups:
    fewer than the bound's 160."""
    torch, pk = require_gpu()
    M, Hq, Hk, d, pairs = shape
    g, q, k, _ = _inputs(torch, M, M, Hq, Hk, d, kind)
    dq, dk = _normal(torch, g, (M, Hq, d), kind), _normal(torch, g, (M, Hk, d), kind)
    f, positions = pk.rope_frequencies(pairs), torch.randperm(5000, generator=g, device="cuda")[:M].contiguous()
    w = _normal(torch, g, (d,), kind) + 1
    for qw, kw, layout in ((w, w, "half"), (None, w, "interleaved"), (None, None, "half")):
        first = pk.rope_qk_backward(dq, dk, q, k, positions, f, qw, kw, layout=layout)
        _compare((dq, dk), (q, k), (qw, kw), first[:2], first[2:], positions.cpu().numpy(), _f64(f), 1e-6, layout, 1.0, kind, kind, "many")
        again = pk.rope_qk_backward(dq, dk, q, k, positions, f, qw, kw, layout=layout)
        assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(first, again))
