"""Every configuration of the 8-bit product and of the 8-bit rows, at sizes that
choose it, and sizes that take more than one launch."""
import os
import re

import numpy as np
import pytest

from tests import i8_plain as plain
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (M, N, K, configuration of aligned rows, of rows that start at any byte and stay there)
SIZES = [(3000, 4100, 1500, "256x256", "128x256_any"), (2300, 2700, 777, "128x256", "128x256_any"), (675, 3052, 775, "128x128", "128x128_any"),
         (1800, 2100, 1100, "128x128", "128x128_any"), (700, 1500, 700, "64x128", "64x64_any"), (986, 519, 649, "64x64_k2", "64x64_k2_any"),
         (1327, 395, 954, "64x64_k2", "64x64_k2_any"), (500, 900, 1300, "32x64_k2", "32x32_k4_any"), (332, 784, 260, "32x64_k2", "64x64_any"),
         (405, 331, 540, "32x32_k2", "32x32_k4_any"), (160, 300, 1111, "16x16_k4", "16x16_k8_any"), (17, 1398, 500, "16x16_k4", "16x16_k8_any"),
         (5, 300, 1000, "rows", "rows"), (8, 2000, 513, "rows", "rows"), (30, 500, 3000, "rows", "rows")]


def _int8(torch, seed, rows, cols, ld):
    """Values of up to 64: the sums below are exact in fp32."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-64, 65, (rows, ld), generator=g, device="cuda", dtype=torch.int8)[:, :cols]


@pytest.mark.parametrize("M,N,K,aligned,unaligned", SIZES)
def test_product(M, N, K, aligned, unaligned):
    torch, pk = require_gpu()
    one = torch.ones(max(M, N), device="cuda")
    none = torch.empty(0, device="cuda")  # no workspace
    for ld, want_name in (((K + 15) // 16 * 16, aligned), ((K + 3) // 4 * 4, aligned), (K | 1, unaligned)):
        a, b = _int8(torch, 1, M, K, ld), _int8(torch, 2, N, K, ld)
        want = a.double() @ b.double().t().contiguous()
        c = pk.gemm_i8(a, b, one[:M], one[:N], dtype=torch.float32, workspace=none)
        assert pk.last_config_name() == "gemm_i8_" + want_name
        assert torch.equal(c.double(), want)
        for dtype in (torch.bfloat16, torch.float16):
            small = one * 2.0 ** -10
            d = pk.gemm_i8(a, b, small[:M], one[:N], bias=one[:N], dtype=dtype, workspace=none)
            assert torch.equal(d, (want * 2.0 ** -10 + 1).float().to(dtype))
        assert torch.equal(c, pk.gemm_i8(a, b, one[:M], one[:N], dtype=torch.float32))


@pytest.mark.parametrize("M,N,K,aligned,unaligned", SIZES)
def test_one_rounding_from_32_bits(M, N, K, aligned, unaligned):
    """Results in 16 bits are those in 32 bits rounded once more, whatever the tile and the column."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(7)
    sa, sb = torch.rand(M, generator=g, device="cuda") * 2.0 ** -6, torch.rand(N, generator=g, device="cuda")
    bias = torch.rand(N, generator=g, device="cuda")
    for ld in ((K + 15) // 16 * 16, K | 1):
        a, b = _int8(torch, 1, M, K, ld), _int8(torch, 2, N, K, ld)
        for given in (None, bias):
            c = pk.gemm_i8(a, b, sa, sb, bias=given, dtype=torch.float32)
            for dtype in (torch.bfloat16, torch.float16):
                assert torch.equal(pk.gemm_i8(a, b, sa, sb, bias=given, dtype=dtype), c.to(dtype))
        back = pk.dequantize_i8(a, sa)
        for dtype in (torch.bfloat16, torch.float16):
            assert torch.equal(pk.dequantize_i8(a, sa, dtype=dtype), back.to(dtype))


def test_every_configuration_is_chosen():
    src = open(os.path.join(ROOT, "paper_1904_05347_amd", "csrc", "pk_gemm_i8.hip")).read()
    names = set(re.findall(r'\{"gemm_i8_(\w+)", \d+', src))
    assert len(names) >= 15
    assert names == {n for s in SIZES for n in s[3:]}


def test_results_larger_than_the_cache():
    torch, pk = require_gpu()
    M, N, K = 5200, 5003, 70
    a, b = _int8(torch, 3, M, K, 80), _int8(torch, 4, N, K, 80)
    one = torch.ones(M, device="cuda")
    want = (a.double() @ b.double().t().contiguous())
    wide = torch.full((M, N + 3), 9.0, device="cuda")
    pk.gemm_i8(a, b, one, one[:N], out=wide[:, 1:N + 1])
    assert torch.equal(wide[:, 1:N + 1].double(), want)
    assert (wide[:, 0] == 9).all() and (wide[:, N + 1:] == 9).all()


@pytest.mark.parametrize("M,N,K", [(140000, 24, 40), (3, 140000, 40), (131073, 131, 17), (200, 131073, 33)])
def test_products_of_more_than_one_launch(M, N, K):
    torch, pk = require_gpu()
    for ld in (48, 49):
        a, b = _int8(torch, 5, M, K, ld), _int8(torch, 6, N, K, ld)
        sa, sb = torch.arange(M, device="cuda") % 7 + 1.0, torch.arange(N, device="cuda") % 5 + 1.0
        bias = torch.arange(N, device="cuda") % 11 + 0.0
        c = pk.gemm_i8(a, b, sa, sb, bias=bias, dtype=torch.float32)
        want = (a.double() @ b.double().t().contiguous()) * sa.double()[:, None] * sb.double() + bias.double()
        assert torch.equal(c.double(), want)


@pytest.mark.parametrize("N", [100, 513, 1025, 1500, 2049, 3001, 4097, 8200, 9000, 12289])
def test_many_rows(N):
    """More than 1024 rows: other numbers of work-items a row."""
    torch, pk = require_gpu()
    M = 1101
    g = torch.Generator(device="cuda").manual_seed(N)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        x = torch.randn((M, N), generator=g, device="cuda").to(dtype)
        r = torch.randn((M, N), generator=g, device="cuda").to(dtype)
        w = torch.randn(N, generator=g, device="cuda").to(dtype)
        f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
        q, s = pk.quantize_i8(x)
        plain.check_rows(f64(q), f64(s), plain.rows(f64(x)), (N, dtype, "quantize"))
        q, s, h = pk.rmsnorm_i8(x, w, residual=r)
        assert torch.equal(h, (x.float() + r.float()).to(dtype))
        plain.check_rows(f64(q), f64(s), plain.norm_rows(f64(h), f64(w), 1e-6), (N, dtype, "norm"))
        q, s = pk.gated_i8(x, r, activation="gelu")
        plain.check_rows(f64(q), f64(s), plain.gated_rows(f64(x), f64(r), "gelu"), (N, dtype, "gated"))


def test_rows_of_more_than_one_launch():
    torch, pk = require_gpu()
    M, N = (1 << 22) + 3, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((M, N), generator=g, device="cuda")
    y = torch.randn((M, N), generator=g, device="cuda")
    w = torch.ones(N, device="cuda")
    tail = slice(M - 5, M)

    def same(got, want):
        return all(torch.equal(a[tail], b) for a, b in zip(got, want))

    q, s = pk.quantize_i8(x)
    assert same((q, s), pk.quantize_i8(x[tail]))
    back = pk.dequantize_i8(q, s)
    assert float((back - x).abs().max()) <= float(x.abs().max()) / 254 * 1.001
    assert torch.equal(back[tail], pk.dequantize_i8(q[tail], s[tail]))
    assert same(pk.rmsnorm_i8(x, w, residual=y), pk.rmsnorm_i8(x[tail], w, residual=y[tail]))
    assert same(pk.gated_i8(x, y), pk.gated_i8(x[tail], y[tail]))
