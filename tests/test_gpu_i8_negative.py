"""Negative views, whose memory holds their values' negatives (the imaginary part of
a conjugate): refused by the 8-bit operators, through either marshalling."""
import pytest

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


@pytest.mark.parametrize("native", [True, False])
def test_negative_views(monkeypatch, native):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    monkeypatch.setattr(binding, "_native", (binding._native or binding._load_native()) if native else _Declines())

    def negative(*shape):
        t = torch.complex(torch.ones(shape, device="cuda"), torch.ones(shape, device="cuda")).conj().imag
        assert t.is_neg() and float(t.sum()) == -t.numel()
        return t

    # one column, or one element: the strides of an imaginary part are no obstacle
    x, w, one = torch.ones(5, 1, device="cuda"), torch.ones(1, device="cuda"), torch.ones(5, device="cuda")
    q = torch.ones((5, 1), dtype=torch.int8, device="cuda")
    neg = negative(5, 1)
    assert neg.stride() == (2, 2)
    calls = [lambda: pk.quantize_i8(neg), lambda: pk.quantize_i8(x[:1], scale=negative(1)), lambda: pk.rmsnorm_i8(neg, w),
             lambda: pk.rmsnorm_i8(x, negative(1)), lambda: pk.rmsnorm_i8(x, w, residual=neg),
             lambda: pk.rmsnorm_i8(x, w, residual=x, sum_out=neg), lambda: pk.gated_i8(neg, x), lambda: pk.gated_i8(x, neg),
             lambda: pk.dequantize_i8(q[:1], negative(1)), lambda: pk.dequantize_i8(q, one, out=neg),
             lambda: pk.gemm_i8(q[:1], q, negative(1), one), lambda: pk.gemm_i8(q, q[:1], one, negative(1)),
             lambda: pk.gemm_i8(q, q[:1], one, w, bias=negative(1)), lambda: pk.gemm_i8(q, q[:1], one, w, out=neg)]
    for n, call in enumerate(calls):
        with pytest.raises(ValueError, match="negative view"):
            call()
            pytest.fail("call %d was not refused" % n)
    q, s = pk.quantize_i8(neg.resolve_neg())
    assert q.flatten().tolist() == [-127] * 5
