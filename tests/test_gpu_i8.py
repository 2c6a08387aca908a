"""The 8-bit operators on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest

from tests import i8_plain as plain
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

KINDS = ("f32", "bf16", "f16")


def _types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rand(torch, seed, M, N, kind, ld=None, scale=1.0):
    """M x N normal values; ld: as a slice of an array that wide, from its second column on."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = N if ld is None else ld
    t = (torch.randn((M, ld), generator=g, device="cuda") * scale).to(_types(torch)[kind])
    return t[:, ld - N:]


def _rand_i8(torch, seed, M, N, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = N if ld is None else ld
    return torch.randint(-128, 128, (M, ld), generator=g, device="cuda", dtype=torch.int8)[:, ld - N:]


def _f64(t):
    import torch
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


# lengths at which a work-item's chunk, a wave's, a team's and the registers' capacity end
ROW_SHAPES = [(1, 1), (3, 7), (5, 64), (2, 255), (4, 512), (3, 513), (1, 1000), (2, 1024), (3, 1030), (1, 2048), (2, 2049),
              (2, 4096), (3, 4097), (1, 8191), (2, 8200), (1, 16384), (2, 16390), (1, 33000), (1, 70001)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N", ROW_SHAPES)
def test_quantize_rows(M, N, kind):
    torch, pk = require_gpu()
    for ld in (N, N + 1, N + 8):
        x = _rand(torch, M * 7 + N, M, N, kind, ld)
        q, s = pk.quantize_i8(x)
        assert q.dtype == torch.int8 and q.shape == (M, N) and s.shape == (M,)
        plain.check_rows(_f64(q), _f64(s), plain.rows(_f64(x)), (M, N, kind, ld))
        assert pk.last_config_name() == "quantize_i8"


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N", ROW_SHAPES)
def test_rmsnorm_rows(M, N, kind):
    torch, pk = require_gpu()
    T = _types(torch)[kind]
    for seed, (ld, wide, residual) in enumerate([(N, False, True), (N + 3, True, True), (N + 8, True, False), (N, False, False)]):
        x = _rand(torch, 10 * N + seed, M, N, kind, ld)
        r = _rand(torch, 10 * N + seed + 5, M, N, kind, ld, 3.0) if residual else None
        w = (1 + 0.2 * _rand(torch, seed, 1, N, "f32")[0]).to(torch.float32 if wide else T)
        q, s, h = pk.rmsnorm_i8(x, w, residual=r, eps=1e-5)
        want_h = (x.float() + r.float()).to(T) if residual else x
        if not residual:
            assert h is x
        assert torch.equal(h, want_h)
        plain.check_rows(_f64(q), _f64(s), plain.norm_rows(_f64(h), _f64(w), 1e-5), (M, N, kind, ld, wide, residual))
        if residual:
            # the sum written over the residual, and over x
            for over in (1, 0):
                terms = [x.clone(), r.clone()]
                q2, s2, h2 = pk.rmsnorm_i8(terms[0], w, residual=terms[1], eps=1e-5, sum_out=terms[over])
                assert h2 is terms[over] and torch.equal(h2, h) and torch.equal(q2, q) and torch.equal(s2, s)
                assert torch.equal(terms[1 - over], x if over else r)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N", ROW_SHAPES)
def test_gated_rows(M, N, kind):
    torch, pk = require_gpu()
    for act in ("silu", "gelu"):
        p = _rand(torch, N + 3, M, 2 * N, kind, 2 * N + (1 if act == "gelu" else 0), 2.0)
        gate, up = p[:, :N], p[:, N:]
        q, s = pk.gated_i8(gate, up, activation=act)
        plain.check_rows(_f64(q), _f64(s), plain.gated_rows(_f64(gate), _f64(up), act), (M, N, kind, act))


def test_gated_over_the_range_of_the_exponential():
    """Gates from -87 to 87 in rows of their own, so that each sets its row's scale."""
    torch, pk = require_gpu()
    g = torch.linspace(-87, 87, 349, device="cuda")[:, None]
    for act, gate in (("silu", g), ("gelu", g / 12)):
        q, s = pk.gated_i8(gate, torch.full_like(gate, 3.0), activation=act)
        plain.check_rows(_f64(q), _f64(s), plain.gated_rows(_f64(gate), np.full((349, 1), 3.0), act), act)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N", ROW_SHAPES)
def test_dequantize_rows(M, N, kind):
    torch, pk = require_gpu()
    for ld in (N, N + 5):
        q = _rand_i8(torch, N, M, N, ld)
        s = _rand(torch, N + 1, 1, M, "f32")[0].abs()
        x = pk.dequantize_i8(q, s, dtype=_types(torch)[kind])
        want = _f64(q) * _f64(s)[:, None]
        plain.check_values(_f64(x), want, plain.U32 * np.abs(want), kind, (M, N, kind, ld))
        wide = torch.full((M, N + 2), 7.0, dtype=_types(torch)[kind], device="cuda")
        assert pk.dequantize_i8(q, s, out=wide[:, 1:N + 1]) is not None
        assert torch.equal(wide[:, 1:N + 1], x) and (wide[:, 0] == 7).all() and (wide[:, N + 1] == 7).all()


def test_rows_of_zeros_infinities_and_nan():
    """A row of zeros and a row too small for its scale give zeros; an infinity or
    a NaN is kept in its row's scale, reads back as NaN and multiplies as NaN, and
    touches no other row.  For every length class, at both ends of the row."""
    torch, pk = require_gpu()
    inf, nan = float("inf"), float("nan")
    for N in (5, 512, 1030, 4097, 40000):
        x = _rand(torch, N, 12, N, "f32")
        x[1] = 0
        x[2] = 0
        x[2, 0] = 1e-37
        x[3, N - 1] = inf
        x[4, 0] = -inf
        x[5, N // 2] = nan
        x[6, 0], x[6, N - 1] = nan, inf
        x[7] = -0.0
        x[8] = 1e30
        q, s = pk.quantize_i8(x)
        assert (q[1:8] == 0).all() and (s[[1, 2, 7]] == 0).all()
        assert (s[3:5] == inf).all() and torch.isnan(s[5:7]).all()
        assert (q[8] == 127).all()
        plain.check_rows(_f64(q), _f64(s), plain.rows(_f64(x)), N)
        back = pk.dequantize_i8(q, s)
        assert torch.isnan(back[3:7]).all() and torch.isfinite(back[[0, 1, 2, 7, 8, 9, 10, 11]]).all()
        c = pk.gemm_i8(q, q[9:], s, s[9:], dtype=torch.float32)
        assert torch.isnan(c[3:7]).all() and torch.isfinite(c[[0, 1, 2, 7, 8, 9, 10, 11]]).all()
        # the norm and the gated activation
        w = torch.ones(N, device="cuda")
        q, s, _ = pk.rmsnorm_i8(x, w)
        assert (q[1:8] == 0).all() and (s[[1, 2, 7]] == 0).all() and not torch.isfinite(s[3:7]).any()
        assert torch.isfinite(s[[0, 9, 10, 11]]).all()
        # 1e30: the sum of squares leaves 32 bits, as stated
        assert s[8] == 0
        q, s = pk.gated_i8(torch.ones_like(x), x)
        assert (q[1:8] == 0).all() and (s[[1, 2, 7]] == 0).all() and not torch.isfinite(s[3:7]).any()
        assert torch.isfinite(s[[0, 8, 9, 10, 11]]).all()


def test_ties_go_to_the_even_integer():
    torch, pk = require_gpu()
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -126.5]], device="cuda")
    q, s = pk.quantize_i8(x)
    assert q.tolist() == [[127, 0, 2, 2, 0, -2, 126, -126]] and s.tolist() == [1.0]


def test_outputs_given_and_views_of_wider_arrays():
    torch, pk = require_gpu()
    M, N = 6, 333
    x = _rand(torch, 1, M, N, "bf16")
    q, s = pk.quantize_i8(x)
    wide = torch.full((M, N + 9), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((M + 2,), -1.0, device="cuda")
    q2, s2 = pk.quantize_i8(x, out=wide[:, 3:N + 3], scale=scales[1:M + 1])
    assert torch.equal(q2, q) and torch.equal(s2, s)
    assert (wide[:, :3] == 99).all() and (wide[:, N + 3:] == 99).all() and scales[0] == -1 and scales[-1] == -1
    assert q.stride(0) % 16 == 0


# ------------------------------------------------------------------ products

GEMM_SHAPES = [(1, 1, 1), (1, 16, 3), (1, 17, 15), (2, 5, 16), (1, 64, 17), (3, 33, 127), (7, 100, 128), (1, 1000, 129), (16, 64, 256),
               (17, 65, 300), (1, 4096, 1024), (5, 31, 2000), (32, 256, 511), (33, 130, 640), (48, 96, 1000), (64, 512, 512),
               (65, 129, 777), (96, 1000, 4096), (128, 128, 128), (129, 257, 257), (200, 300, 1500), (256, 256, 64),
               (255, 511, 1023), (300, 70, 5000), (257, 1025, 130), (512, 768, 640), (1021, 531, 777), (16, 16, 131071)]


@pytest.mark.parametrize("M,N,K", GEMM_SHAPES)
def test_gemm(M, N, K):
    """Every alignment of the operands' rows, with and without a bias, in each type."""
    torch, pk = require_gpu()
    kinds = [("bf16", 0, False), ("f32", 16, True), ("f16", 4, False), ("bf16", 3, True), ("f32", 1, False)]
    for seed, (kind, slack, with_bias) in enumerate(kinds):
        ld = (K + 15) // 16 * 16 + slack if slack % 4 == 0 else K + slack
        a, b = _rand_i8(torch, seed + 1, M, K, ld), _rand_i8(torch, seed + 2, N, K, ld)
        sa = _rand(torch, seed, 1, M, "f32")[0].abs() * 0.01
        sb = _rand(torch, seed + 9, 1, N, "f32")[0] * 0.01 / K ** 0.5
        bias = _rand(torch, seed + 8, 1, N, "f32")[0] if with_bias else None
        c = pk.gemm_i8(a, b, sa, sb, bias=bias, dtype=_types(torch)[kind])
        assert pk.last_config_name().startswith("gemm_i8_")
        want, bound = plain.gemm(_f64(a), _f64(b), _f64(sa), _f64(sb), None if bias is None else _f64(bias))
        plain.check_values(_f64(c), want, bound, kind, (M, N, K, kind, slack))


@pytest.mark.parametrize("M,N,K", [(2, 3, 131071), (70, 300, 131071), (300, 300, 131071)])
def test_gemm_largest_sums(M, N, K):
    """Every product 128 * 128: the sum's largest magnitude, in either sign, is exact."""
    torch, pk = require_gpu()
    a = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    b = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    b[1::2] = 127
    one = torch.ones(max(M, N), device="cuda")
    c = pk.gemm_i8(a, b, one[:M], one[:N], dtype=torch.float32)
    want = torch.where(torch.arange(N, device="cuda") % 2 == 0, 16384.0 * K, -16256.0 * K).double()
    assert torch.equal(c.double(), want.float().double().expand(M, N))


@pytest.mark.parametrize("M,N,K", [(3, 40, 50), (70, 90, 200), (300, 300, 333), (1, 500, 1000)])
def test_gemm_reads_and_writes_nothing_else(M, N, K):
    """What lies beside the operands' rows in wider arrays has no part in the result,
    and what lies beside the result's rows stays."""
    torch, pk = require_gpu()
    for left, right in ((0, 13), (16, 16), (3, 1), (4, 8)):
        wide_a, wide_b = _rand_i8(torch, 1, M, left + K + right), _rand_i8(torch, 2, N, left + K + right)
        one = torch.ones(max(M, N), device="cuda")
        got = []
        for fill in (None, 0, 127):
            wa, wb = wide_a.clone(), wide_b.clone()
            for w in (wa, wb):
                if fill is not None:
                    w[:, :left] = fill
                    w[:, left + K:] = fill
            out = torch.full((M, N + 7), 5.0, device="cuda")
            pk.gemm_i8(wa[:, left:left + K], wb[:, left:left + K], one[:M], one[:N], out=out[:, 2:N + 2])
            assert (out[:, :2] == 5).all() and (out[:, N + 2:] == 5).all()
            got.append(out)
        want = _f64(wide_a[:, left:left + K]) @ _f64(wide_b[:, left:left + K]).T
        assert np.array_equal(_f64(got[0][:, 2:N + 2]), want)
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_gemm_operands_beyond_32_bit_offsets():
    """Rows that lie more than 2^32 bytes from the first one, in either operand and the result."""
    torch, pk = require_gpu()
    rows, ld, K, m = 1100, 1 << 22, 200, 37
    big = torch.zeros((rows, ld), dtype=torch.int8, device="cuda")
    big[:, 5:K + 5] = _rand_i8(torch, 1, rows, K)
    small = _rand_i8(torch, 2, m, K)
    one = torch.ones(rows, device="cuda")
    far = big[:, 5:K + 5]
    want = _f64(far) @ _f64(small).T
    assert np.array_equal(_f64(pk.gemm_i8(far, small, one, one[:m], dtype=torch.float32)), want)
    assert np.array_equal(_f64(pk.gemm_i8(small, far, one[:m], one, dtype=torch.float32)), want.T)
    near = far.contiguous()
    assert np.array_equal(_f64(pk.gemm_i8(near, near, one, one, dtype=torch.float32)), _f64(near) @ _f64(near).T)
    q, s = pk.quantize_i8(pk.dequantize_i8(far, one), out=far, scale=torch.empty(rows, device="cuda"))
    back = pk.dequantize_i8(far, s)
    assert (back - near.float()).abs().max() <= 0.505   # half a step of at most 128 / 127
    del big, far, q
    wide = torch.zeros((rows, 1 << 21), dtype=torch.bfloat16, device="cuda")
    out = wide[:, 9:m + 9]
    pk.gemm_i8(near, small, one, one[:m], out=out)
    assert torch.equal(out, pk.gemm_i8(near, small, one, one[:m]))
    assert (wide[:, :9] == 0).all() and (wide[:, m + 9:m + 100] == 0).all()
    q, s = pk.quantize_i8(out)
    q2, s2 = pk.quantize_i8(out.contiguous())
    assert torch.equal(q, q2) and torch.equal(s, s2)


def test_empty():
    torch, pk = require_gpu()
    e = lambda *shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    i8 = torch.int8
    assert pk.gemm_i8(e(0, 8, t=i8), e(5, 8, t=i8), e(0), e(5)).shape == (0, 5)
    assert pk.gemm_i8(e(4, 8, t=i8), e(0, 8, t=i8), e(4), e(0)).shape == (4, 0)
    bias = torch.arange(5.0, device="cuda")
    a, b = e(4, 0, t=i8), e(5, 0, t=i8)
    nan4, nan5 = torch.full((4,), float("nan"), device="cuda"), torch.full((5,), float("nan"), device="cuda")
    assert torch.equal(pk.gemm_i8(a, b, nan4, nan5, bias=bias, dtype=torch.float32), bias.expand(4, 5))
    assert torch.equal(pk.gemm_i8(a, b, nan4, nan5, dtype=torch.float16), torch.zeros(4, 5, dtype=torch.float16, device="cuda"))
    for M, N in ((0, 7), (3, 0)):
        x = e(M, N)
        for q, s in (pk.quantize_i8(x), pk.rmsnorm_i8(x, e(N), residual=x)[:2], pk.gated_i8(x, x)):
            assert q.shape == (M, N) and s.tolist() == [0.0] * M
        assert pk.dequantize_i8(q, s).shape == (M, N)


def test_another_stream_and_graph_replays():
    """Calls go to the current stream; a captured feed-forward layer replays to the eager bits."""
    torch, pk = require_gpu()
    D, F = 640, 1000
    w1, s1 = pk.quantize_i8(_rand(torch, 1, 2 * F, D, "f32"))
    w2, s2 = pk.quantize_i8(_rand(torch, 2, D, F, "f32"))
    norm = torch.ones(D, dtype=torch.bfloat16, device="cuda")

    def layer(x, r):
        q, s, h = pk.rmsnorm_i8(x, norm, residual=r)
        p = pk.gemm_i8(q, w1, s, s1)
        q, s = pk.gated_i8(p[:, :F], p[:, F:])
        return pk.gemm_i8(q, w2, s, s2), h

    for M in (1, 40, 300):
        x, r = _rand(torch, 3, M, D, "bf16"), _rand(torch, 4, M, D, "bf16")
        want = [t.clone() for t in layer(x, r)]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            late = x.clone().mul_(0).add_(x)   # made on this stream just before
            got = layer(late, r)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        sx, sr = torch.zeros_like(x), torch.zeros_like(r)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer(sx, sr)
        for k in range(3):
            sx.copy_(x + k)
            sr.copy_(r)
            g.replay()
            eager = layer(x + k, r)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, eager)), (M, k)
        del g


def test_calls_are_deterministic():
    torch, pk = require_gpu()
    for M, N, K in ((1, 4096, 4096), (40, 1000, 3000), (520, 1030, 2000)):
        a, b = _rand_i8(torch, 1, M, K), _rand_i8(torch, 2, N, K)
        sa, sb = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
        first = pk.gemm_i8(a, b, sa, sb, dtype=torch.float32)
        x = _rand(torch, 5, M, K, "bf16")
        w = torch.rand(K, device="cuda")
        q, s, _ = pk.rmsnorm_i8(x, w)
        for _ in range(3):
            assert torch.equal(first, pk.gemm_i8(a, b, sa, sb, dtype=torch.float32))
            q2, s2, _ = pk.rmsnorm_i8(x, w)
            assert torch.equal(q, q2) and torch.equal(s, s2)


# ------------------------------------------------------------------ marshalling and refusals

class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


def test_native_marshalling_equals_python(monkeypatch):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    native = binding._native or binding._load_native()
    x, r, w = _rand(torch, 1, 9, 100, "bf16", 103), _rand(torch, 2, 9, 100, "bf16"), torch.ones(100, device="cuda")
    a, b = _rand_i8(torch, 3, 9, 100, 117), _rand_i8(torch, 4, 30, 100)
    sa, sb = torch.rand(9, device="cuda"), torch.rand(30, device="cuda")
    qo = torch.empty((9, 100), dtype=torch.int8, device="cuda")
    calls = [
        ("quantize_i8", lambda: pk.quantize_i8(x)), ("quantize_i8", lambda: pk.quantize_i8(x, out=qo, scale=sa.clone())),
        ("rmsnorm_i8", lambda: pk.rmsnorm_i8(x, w, residual=r)), ("rmsnorm_i8", lambda: pk.rmsnorm_i8(x, w, eps=0.5)),
        ("rmsnorm_i8", lambda: pk.rmsnorm_i8(x, w.bfloat16(), residual=r, sum_out=torch.empty_like(r))),
        ("gated_i8", lambda: pk.gated_i8(x, r)), ("gated_i8", lambda: pk.gated_i8(x, r, activation="gelu")),
        ("dequantize_i8", lambda: (pk.dequantize_i8(a, sa),)),
        ("dequantize_i8", lambda: (pk.dequantize_i8(a, sa, dtype=torch.float16),)),
        ("dequantize_i8", lambda: (pk.dequantize_i8(a, sa, out=torch.empty(9, 100, device="cuda")),)),
        ("gemm_i8", lambda: (pk.gemm_i8(a, b, sa, sb),)),
        ("gemm_i8", lambda: (pk.gemm_i8(a, b, sa, sb, bias=sb, dtype=torch.float32),)),
        ("gemm_i8", lambda: (pk.gemm_i8(a, b, sa, sb, out=torch.empty(9, 30, device="cuda")),)),
    ]
    for name, call in calls:
        took = []

        class Watch:
            def __getattr__(self, f):
                def g(*args):
                    v = getattr(native, f)(*args)
                    took.append((f, v is not None))
                    return v
                return g

        monkeypatch.setattr(binding, "_native", Watch())
        first = [t.clone() for t in call()]
        assert took == [(name, True)]
        monkeypatch.setattr(binding, "_native", _Declines())
        second = call()
        monkeypatch.setattr(binding, "_native", native)
        assert len(first) == len(second)
        for p, q in zip(first, second):
            assert p.dtype == q.dtype and torch.equal(p, q), name


def test_refusals(monkeypatch):
    """The same errors through either marshalling."""
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    native = binding._native or binding._load_native()
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda")
    q, s = pk.quantize_i8(x)
    v = torch.ones(4, device="cuda")
    T, V, P = TypeError, ValueError, pk.PkError
    bad = [
        (T, lambda: pk.quantize_i8(x.double())), (T, lambda: pk.quantize_i8(x.cpu())), (V, lambda: pk.quantize_i8(x[0])),
        (V, lambda: pk.quantize_i8(x.t())), (V, lambda: pk.quantize_i8(x, out=q[:2])), (T, lambda: pk.quantize_i8(x, out=x)),
        (V, lambda: pk.quantize_i8(x, scale=torch.ones(5, device="cuda"))), (T, lambda: pk.quantize_i8(x, scale=q[:, 0])),
        (V, lambda: pk.quantize_i8(x[:1].expand(4, 8))),
        (P, lambda: pk.quantize_i8(x, out=x.view(torch.int8).as_strided((4, 8), (8, 1)))),
        (T, lambda: pk.rmsnorm_i8(x, w.bfloat16())), (V, lambda: pk.rmsnorm_i8(x, w[:7])), (T, lambda: pk.rmsnorm_i8(x.int(), w)),
        (V, lambda: pk.rmsnorm_i8(x, w, residual=x[:3])), (T, lambda: pk.rmsnorm_i8(x, w, residual=x.half())),
        (V, lambda: pk.rmsnorm_i8(x, w, sum_out=x)), (P, lambda: pk.rmsnorm_i8(x, w, eps=-1.0)),
        (P, lambda: pk.rmsnorm_i8(x, w, eps=float("nan"))),
        (P, lambda: pk.rmsnorm_i8(x[:3], w, residual=x[:3], sum_out=x[1:])),
        (V, lambda: pk.gated_i8(x, x, activation="relu")), (V, lambda: pk.gated_i8(x, x[:3])), (T, lambda: pk.gated_i8(x, x.half())),
        (T, lambda: pk.dequantize_i8(x, s)), (V, lambda: pk.dequantize_i8(q, s[:3])), (T, lambda: pk.dequantize_i8(q, s, dtype=torch.int8)),
        (T, lambda: pk.dequantize_i8(q, s, dtype=torch.float16, out=x)), (V, lambda: pk.dequantize_i8(q, s, out=x[:3])),
        (T, lambda: pk.gemm_i8(x, q, s, s)), (V, lambda: pk.gemm_i8(q, q[:, :7], s, s)), (V, lambda: pk.gemm_i8(q, q, s[:3], s)),
        (V, lambda: pk.gemm_i8(q, q, s, s, bias=w)), (T, lambda: pk.gemm_i8(q, q, s, s, bias=v.half())),
        (T, lambda: pk.gemm_i8(q, q, s, s, dtype=torch.float64)), (V, lambda: pk.gemm_i8(q, q, s, s, out=x)),
        (V, lambda: pk.gemm_i8(q.t(), q, w, s)), (T, lambda: pk.gemm_i8(q.cpu(), q, s, s)),
        (T, lambda: pk.gemm_i8(q, q, s.double(), s)), (V, lambda: pk.gemm_i8(q, q, s, torch.ones(8, device="cuda")[::2])),
    ]
    for n, (error, call) in enumerate(bad):
        for marshalling in (native, _Declines()):
            monkeypatch.setattr(binding, "_native", marshalling)
            with pytest.raises(error):
                call()
                pytest.fail("call %d was not refused" % n)
    monkeypatch.setattr(binding, "_native", native)
    k = torch.zeros((2, 131072), dtype=torch.int8, device="cuda")
    with pytest.raises(P) as e:
        pk.gemm_i8(k, k, v[:2], v[:2])
    assert e.value.status == binding.PK_ERR_NOT_SUPPORTED


def test_new_outputs_rows_start_at_memory_lines(monkeypatch):
    """Through either marshalling; the bytes behind a row are not part of it."""
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    native = binding._native or binding._load_native()
    for N, ld in ((1, 16), (333, 336), (1008, 1008), (1023, 1024), (1024, 1024), (1025, 1152), (5003, 5120)):
        x = _rand(torch, N, 3, N, "bf16")
        for marshalling in (native, _Declines()):
            monkeypatch.setattr(binding, "_native", marshalling)
            for q in (pk.quantize_i8(x)[0], pk.rmsnorm_i8(x, torch.ones(N, device="cuda"))[0], pk.gated_i8(x, x)[0]):
                assert q.shape == (3, N) and q.stride() == (ld, 1) and q.data_ptr() % 16 == 0
        monkeypatch.setattr(binding, "_native", native)
