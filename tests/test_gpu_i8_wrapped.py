"""Tensors that a torch.func transform has wrapped: they look like plain ones and
have no memory of their own.  The 8-bit operators refuse them with an error,
through either marshalling, whichever operand it is."""
import pytest

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


def _calls(torch, pk):
    """(operator, operands): every tensor the call takes, outputs among them."""
    f = lambda *shape: torch.ones(shape, device="cuda")  # noqa: E731
    i = lambda *shape: torch.ones(shape, dtype=torch.int8, device="cuda")  # noqa: E731
    return [
        (lambda x, out, scale: pk.quantize_i8(x, out=out, scale=scale), [f(4, 8), i(4, 8), f(4)]),
        (lambda x, w, r, h, out, scale: pk.rmsnorm_i8(x, w, residual=r, sum_out=h, out=out, scale=scale),
         [f(4, 8), f(8), f(4, 8), f(4, 8), i(4, 8), f(4)]),
        (lambda g, u, out, scale: pk.gated_i8(g, u, out=out, scale=scale), [f(4, 8), f(4, 8), i(4, 8), f(4)]),
        (lambda q, s, out: pk.dequantize_i8(q, s, out=out), [i(4, 8), f(4), f(4, 8)]),
        (lambda a, b, sa, sb, bias, out: pk.gemm_i8(a, b, sa, sb, bias=bias, out=out),
         [i(4, 8), i(5, 8), f(4), f(5), f(5), f(4, 5)]),
    ]


@pytest.mark.parametrize("native", [True, False])
def test_wrapped_by_vmap(monkeypatch, native):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    monkeypatch.setattr(binding, "_native", (binding._native or binding._load_native()) if native else _Declines())
    for op, operands in _calls(torch, pk):
        op(*operands)
        for n, t in enumerate(operands):
            def one(wrapped):
                op(*operands[:n], wrapped, *operands[n + 1:])
                return wrapped

            with pytest.raises(RuntimeError, match="storage|data pointer"):
                torch.func.vmap(one)(torch.stack([t, t]))
        op(*operands)
    torch.cuda.synchronize()


@pytest.mark.parametrize("native", [True, False])
def test_wrapped_by_grad(monkeypatch, native):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    monkeypatch.setattr(binding, "_native", (binding._native or binding._load_native()) if native else _Declines())
    for op, operands in _calls(torch, pk):
        for n, t in enumerate(operands):
            if not t.is_floating_point():
                continue

            def one(wrapped):
                op(*operands[:n], wrapped, *operands[n + 1:])
                return wrapped.sum()

            with pytest.raises(RuntimeError, match="storage|data pointer"):
                torch.func.grad(one)(t)
    torch.cuda.synchronize()


def test_plain_operands_inside_a_transform():
    """Operands that the transform does not touch are taken as ever."""
    torch, pk = require_gpu()
    x = torch.randn(4, 40, device="cuda")
    q, s = pk.quantize_i8(x)
    q2, s2 = torch.zeros_like(q), torch.zeros_like(s)

    def one(y):
        pk.quantize_i8(x, out=q2, scale=s2)
        return y.sum()

    torch.func.grad(one)(torch.ones(3, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(s, s2)
