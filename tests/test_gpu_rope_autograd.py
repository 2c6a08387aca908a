"""rope_qk beside autograd: it records no graph by itself, and in a Function with its gradients it takes part in one."""
import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_heads import KINDS, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
def test_no_graph_without_a_function(kind):
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, w = (_normal(torch, g, s, kind).requires_grad_() for s in ((5, 4, 32), (5, 2, 32), (32,)))
    f, positions = pk.rope_frequencies(16), torch.arange(5, device="cuda")
    for given in (False, True):
        out = (torch.empty_like(q), torch.empty_like(k)) if given else (None, None)
        for y in pk.rope_qk(q, k, positions, f, w, w, q_out=out[0], k_out=out[1]):
            assert not y.requires_grad and y.grad_fn is None
    assert all(t is None or not t.requires_grad for t in pk.rope_qk_backward(q, k, q, k, positions, f, w, w))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_a_function(layout, kind):
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(2)
    f, positions = pk.rope_frequencies(12), torch.arange(7, device="cuda") * 3

    class Rope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, qw, kw):
            ctx.save_for_backward(q, k, qw, kw)
            return pk.rope_qk(q, k, positions, f, qw, kw, layout=layout)

        @staticmethod
        def backward(ctx, dq, dk):
            q, k, qw, kw = ctx.saved_tensors
            return pk.rope_qk_backward(dq.contiguous(), dk.contiguous(), q, k, positions, f, qw, kw, layout=layout)

    q, k = (_normal(torch, g, (7, h, 32), kind).requires_grad_() for h in (6, 2))
    qw, kw = ((_normal(torch, g, (32,), kind) + 1).requires_grad_() for _ in range(2))
    dq, dk = _normal(torch, g, q.shape, kind), _normal(torch, g, k.shape, kind)
    oq, ok = Rope.apply(q, k, qw, kw)
    torch.autograd.backward((oq, ok), (dq, dk))
    with torch.no_grad():
        want = pk.rope_qk(q, k, positions, f, qw, kw, layout=layout)
        grads = pk.rope_qk_backward(dq, dk, q, k, positions, f, qw, kw, layout=layout)
    assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
    for t, want in zip((q, k, qw, kw), grads):
        assert torch.equal(t.grad, want)
