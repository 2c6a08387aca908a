"""The feed-forward layer that runs the 8-bit operators together."""
import pytest

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _layer(torch, D, F, activation, dtype):
    from paper_1904_05347_amd.feedforward import FeedForwardI8
    g = torch.Generator(device="cuda").manual_seed(D + F)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    weights = (1 + normal(D, scale=0.1), normal(F, D, scale=D ** -0.5), normal(F, D, scale=D ** -0.5), normal(D, F, scale=F ** -0.5))
    return FeedForwardI8(*weights, activation=activation), weights, normal


@pytest.mark.parametrize("M,D,F,activation,kind", [(1, 512, 1024, "silu", "bfloat16"), (37, 333, 1001, "gelu", "float16"),
                                                   (300, 1024, 777, "silu", "float32"), (512, 1024, 2048, "gelu", "bfloat16")])
def test_layer(M, D, F, activation, kind):
    """Against float64 with the weights as they were.  Rounding a row to 255 levels
    leaves an error of a / 127 / sqrt(12), a its largest magnitude: 1.2 % of a
    normal row's length for a = 5 deviations (of up to 2048 values), so each
    product of two such operands is 1.7 % off.  The gate's and the up projection's
    1.7 % make 2.4 % of their product (the gate's share grows by at most 1.3, the
    largest of g act'(g) / act(g) in its mean square over normal gates being below
    1.3^2: 2.9 %), whose rows have a of up to 20 deviations: 4.6 %.  With the last
    weights' 1.2 % the sum is 5.6 %; 16-bit storage adds 0.4 % at most."""
    torch, pk = require_gpu()
    from paper_1904_05347_amd.feedforward import reference
    layer, weights, normal = _layer(torch, D, F, activation, getattr(torch, kind))
    x, r = normal(M, D, scale=0.5), normal(M, D)
    for residual in (r, None):
        y, h = layer(x, residual)
        want, want_h = reference(x, residual, *weights, activation=activation)
        assert y.dtype == x.dtype and y.shape == (M, D)
        assert float((y.double() - want).norm() / want.norm()) < 0.06
        assert torch.equal(h, x if residual is None else (x.float() + r.float()).to(x.dtype))
        # and bit for bit the operators one by one, their operands laid out anew
        q, s, _ = pk.rmsnorm_i8(x, layer.norm, residual=residual)
        p = pk.gemm_i8(q.contiguous(), layer.first, s, layer.first_scale, dtype=x.dtype)
        q, s = pk.gated_i8(p[:, :F].contiguous(), p[:, F:].contiguous(), activation=activation)
        assert torch.equal(y, pk.gemm_i8(q.contiguous(), layer.second, s, layer.second_scale, dtype=x.dtype))


def test_shapes_are_checked():
    torch, pk = require_gpu()
    from paper_1904_05347_amd.feedforward import FeedForwardI8
    one = torch.ones
    for norm, gate, up, down in (((8,), (16, 8), (16, 7), (8, 16)), ((8,), (16, 8), (16, 8), (16, 8)), ((7,), (16, 8), (16, 8), (8, 16))):
        with pytest.raises(ValueError):
            FeedForwardI8(*(one(s, device="cuda") for s in (norm, gate, up, down)))


def test_command(capsys):
    require_gpu()
    from paper_1904_05347_amd import feedforward
    feedforward.main(["--tokens", "1", "70", "--dim", "256", "--width", "512"])
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and all("off float64" in line for line in lines)
