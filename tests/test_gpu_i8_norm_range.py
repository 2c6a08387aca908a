"""The norm of rows whose squares leave the 32 bits' range below: with an eps that
does not cover them the scale is still that of the definition."""
import numpy as np
import pytest

from tests import i8_plain as plain
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _f64(t):
    import torch
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


SIZES = [1e-12, 1e-18, 1e-20, 1e-23, 1e-26, 1e-30, 1e-34]


def _rows(torch, M, N, kind):
    """Normal rows, row m of deviation SIZES[m % 7]; every eighth an ordinary one."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    size = torch.tensor([1.0 if m % 8 == 7 else SIZES[m % 7] for m in range(M)], dtype=torch.float64, device="cuda")
    return (torch.randn((M, N), generator=g, device="cuda").double() * size[:, None]).to(kind)


# every number of work-items a row, and rows that the registers do not hold
SHAPES = [(9, 1), (9, 5), (16, 500), (8, 1024), (9, 2048), (15, 3000), (8, 4097), (9, 9000), (8, 40000), (1030, 900), (1030, 2049)]


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-36, 7e-31, 1e-29, 1e-24, 1e-6])
@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
def test_small_rows(M, N, kind, eps):
    """Against the definition in 64 bits, with the bounds of any other row: adding
    the squares of h times a power of two rounds as adding those of h does."""
    torch, pk = require_gpu()
    T = getattr(torch, kind)
    x = _rows(torch, M, N, T)
    w = (1 + 0.2 * torch.rand(N, device="cuda")).to(T)
    q, s, _ = pk.rmsnorm_i8(x, w, eps=eps)
    plain.check_rows(_f64(q), _f64(s), plain.norm_rows(_f64(x), _f64(w), float(np.float32(eps))), (M, N, kind, eps))
    # the residual's addition, the sum stored beside and over its terms
    r = _rows(torch, M, N, T).flip(1)
    q, s, h = pk.rmsnorm_i8(x, w, residual=r, eps=eps)
    assert torch.equal(h, (x.float() + r.float()).to(T))
    plain.check_rows(_f64(q), _f64(s), plain.norm_rows(_f64(h), _f64(w), float(np.float32(eps))), (M, N, kind, eps))
    over = r.clone()
    q2, s2, _ = pk.rmsnorm_i8(x, w, residual=over, eps=eps, sum_out=over)
    assert torch.equal(q2, q) and torch.equal(s2, s) and torch.equal(over, h)


@pytest.mark.parametrize("N", [5, 1024, 2048, 9000, 40000])
def test_sum_that_is_not_stored(N):
    """The C entry without `sum`: x + residual is formed again where it is needed again."""
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    x, w = _rows(torch, 9, N, torch.float32), 1 + torch.rand(N, device="cuda")
    r = _rows(torch, 9, N, torch.float32).flip(1).contiguous()
    q, s, _ = pk.rmsnorm_i8(x, w, residual=r, eps=0.0)
    q2, s2 = torch.zeros((9, N), dtype=torch.int8, device="cuda"), torch.zeros(9, device="cuda")
    st = binding.load().pk_rmsnorm_i8(x.data_ptr(), 0, 9, N, N, r.data_ptr(), N, w.data_ptr(), 0, 0.0, None, 0,
                                      q2.data_ptr(), N, s2.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(q2, q) and torch.equal(s2, s)


@pytest.mark.parametrize("N", [5, 1024, 2048, 9000, 40000])
def test_the_least_rows(N):
    """h from the least subnormal on with weights that bring h * weight back into
    range, and results on either side of one; a single element that is not 0."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(N)
    least = 2.0 ** -149
    for weight in (1e9, 1e12, 1e20, 1e30):
        h = (torch.randint(-9, 10, (9, N), generator=g, device="cuda").double() * least).float()
        h[:, 0] = 3 * least
        h[8, 1:] = 0
        w = (1 + torch.rand(N, generator=g, device="cuda")) * weight
        for eps in (0.0, 1e-45, 1e-33):
            q, s, _ = pk.rmsnorm_i8(h, w, eps=eps)
            plain.check_rows(_f64(q), _f64(s), plain.norm_rows(_f64(h), _f64(w), float(np.float32(eps))), (N, weight, eps))
    # a below and above one beside a large weight
    h = torch.full((2, N), 1e-20, device="cuda")
    for weight in (1e15, 1e22, 1e30):
        w = torch.full((N,), weight, device="cuda")
        q, s, _ = pk.rmsnorm_i8(h, w, eps=0.0)
        plain.check_rows(_f64(q), _f64(s), plain.norm_rows(_f64(h), _f64(w), 0.0), (N, weight))


def test_products_above_the_range():
    """h * weight beyond 32 bits is an infinity, and marks its row alone."""
    torch, pk = require_gpu()
    h = torch.ones((3, 40), device="cuda")
    h[1, 7] = 1e10
    w = torch.ones(40, device="cuda")
    w[7] = 1e30
    q, s, _ = pk.rmsnorm_i8(h, w)
    assert (q[1] == 0).all() and s[1] == float("inf") and torch.isfinite(s[[0, 2]]).all() and (q[[0, 2], 7] == 127).all()
    assert torch.isnan(pk.dequantize_i8(q, s)[1]).all()
