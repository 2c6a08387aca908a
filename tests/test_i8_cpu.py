"""The 8-bit operators' host side, on the CPU: which argument a refused call
names, empty calls, and the Python checks that come before the library.  No
call here reaches the GPU."""
import numpy as np
import pytest

from tests import i8_plain as plain

FAKE = 1 << 20   # addresses that are never read: every call fails its checks or is empty


@pytest.fixture(scope="module")
def lib():
    import os

    from paper_1904_05347_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    return binding.load()


def _cases(lib, fn, good, bad, not_supported=()):
    order = list(good)
    for key, value, position in bad:
        st = fn(*[{**good, key: value}[k] for k in order], None)
        assert (st, lib.pk_last_invalid_param()) == (1, position), (key, value, st, lib.pk_last_invalid_param())
    for key, value in not_supported:
        assert fn(*[{**good, key: value}[k] for k in order], None) == 2, (key, value)


def test_quantize_arguments(lib):
    good = dict(x=FAKE, dtype=0, M=4, N=8, ldx=8, q=2 * FAKE, ldq=8, scale=3 * FAKE)
    _cases(lib, lib.pk_quantize_i8, good,
           [("dtype", 3, 2), ("dtype", -1, 2), ("M", -1, 3), ("N", -1, 4), ("ldx", 7, 5), ("ldq", 7, 7), ("x", None, 1),
            ("x", FAKE + 2, 1), ("q", None, 6), ("scale", None, 8), ("scale", FAKE + 1, 8), ("q", FAKE + 127, 6),
            ("scale", FAKE, 8), ("scale", 2 * FAKE + 28, 8)],
           [("ldx", (1 << 30) + 1), ("ldq", 1 << 40)])
    assert lib.pk_quantize_i8(None, 0, 0, 8, 8, None, 8, None, None) == 0


def test_rmsnorm_arguments(lib):
    good = dict(x=FAKE, dtype=1, M=4, N=8, ldx=8, r=2 * FAKE, ldr=8, w=3 * FAKE, wt=1, eps=1e-6, sum=4 * FAKE, lds=8,
                q=5 * FAKE, ldq=8, scale=6 * FAKE)
    _cases(lib, lib.pk_rmsnorm_i8, good,
           [("dtype", 9, 2), ("M", -1, 3), ("N", -1, 4), ("ldx", 7, 5), ("ldr", 7, 7), ("wt", 2, 9), ("wt", 7, 9),
            ("eps", -1e-6, 10), ("eps", float("nan"), 10), ("r", None, 11), ("lds", 7, 12), ("ldq", 7, 14), ("x", None, 1),
            ("x", FAKE + 1, 1), ("r", 2 * FAKE + 1, 6), ("w", None, 8), ("w", 3 * FAKE + 1, 8), ("sum", 4 * FAKE + 1, 11),
            ("q", None, 13), ("scale", None, 15), ("scale", 6 * FAKE + 2, 15), ("sum", FAKE + 2, 11), ("sum", 2 * FAKE - 2, 11),
            ("sum", 3 * FAKE, 11), ("q", FAKE, 13), ("q", 2 * FAKE, 13), ("q", 3 * FAKE, 13), ("q", 4 * FAKE, 13),
            ("scale", FAKE, 15), ("scale", 2 * FAKE, 15), ("scale", 3 * FAKE, 15), ("scale", 4 * FAKE, 15), ("scale", 5 * FAKE, 15)],
           [("lds", 1 << 31), ("ldr", 1 << 31)])
    # over a term with another leading dimension
    _cases(lib, lib.pk_rmsnorm_i8, dict(good, lds=9), [("sum", FAKE, 11), ("sum", 2 * FAKE, 11)])
    assert lib.pk_rmsnorm_i8(None, 1, 0, 8, 8, None, 0, None, 1, 0.0, None, 0, None, 8, None, None) == 0


def test_gated_arguments(lib):
    good = dict(g=FAKE, ldg=16, u=FAKE + 32, ldu=16, dtype=0, act=0, M=4, N=8, q=2 * FAKE, ldq=8, scale=3 * FAKE)
    _cases(lib, lib.pk_gated_i8, good,
           [("dtype", 3, 5), ("act", 2, 6), ("act", -1, 6), ("M", -1, 7), ("N", -1, 8), ("ldg", 7, 2), ("ldu", 7, 4), ("ldq", 7, 10),
            ("g", None, 1), ("g", FAKE + 2, 1), ("u", None, 3), ("u", FAKE + 2, 3), ("q", None, 9), ("q", FAKE + 40, 9),
            ("scale", None, 11), ("scale", FAKE, 11), ("scale", 2 * FAKE, 11)], [("ldu", 1 << 31)])
    assert lib.pk_gated_i8(None, 8, None, 8, 0, 0, 0, 8, None, 8, None, None) == 0


def test_dequantize_arguments(lib):
    good = dict(q=FAKE, ldq=8, scale=2 * FAKE, M=4, N=8, x=3 * FAKE, dtype=2, ldx=8)
    _cases(lib, lib.pk_dequantize_i8, good,
           [("M", -1, 4), ("N", -1, 5), ("dtype", 5, 7), ("ldq", 7, 2), ("ldx", 7, 8), ("q", None, 1), ("scale", None, 3),
            ("scale", 2 * FAKE + 1, 3), ("x", None, 6), ("x", 3 * FAKE + 1, 6), ("x", FAKE, 6), ("x", 2 * FAKE, 6)], [("ldq", 1 << 31)])
    assert lib.pk_dequantize_i8(None, 8, None, 4, 0, None, 2, 8, None) == 0


def test_gemm_arguments(lib):
    good = dict(M=4, N=5, K=6, A=FAKE, lda=6, sa=2 * FAKE, B=3 * FAKE, ldb=6, sb=4 * FAKE, bias=5 * FAKE, C=6 * FAKE,
                dtype=0, ldc=5)
    _cases(lib, lib.pk_gemm_i8, good,
           [("M", -1, 1), ("N", -1, 2), ("K", -1, 3), ("lda", 5, 5), ("ldb", 5, 8), ("dtype", 3, 12), ("ldc", 4, 13),
            ("A", None, 4), ("sa", None, 6), ("sa", 2 * FAKE + 2, 6), ("B", None, 7), ("sb", None, 9), ("sb", 4 * FAKE + 1, 9),
            ("bias", 5 * FAKE + 2, 10), ("C", None, 11), ("C", 6 * FAKE + 2, 11), ("C", FAKE, 11), ("C", 2 * FAKE, 11),
            ("C", 3 * FAKE + 28, 11), ("C", 4 * FAKE, 11), ("C", 5 * FAKE, 11)],
           [("lda", 1 << 31), ("ldc", 1 << 31)])
    _cases(lib, lib.pk_gemm_i8, dict(good, lda=1 << 18, ldb=1 << 18), [], [("K", 131072)])
    assert lib.pk_gemm_i8(0, 5, 6, None, 6, None, None, 6, None, None, None, 0, 5, None) == 0
    assert lib.pk_gemm_i8(4, 0, 6, None, 6, None, None, 6, None, None, None, 0, 1, None) == 0
    assert lib.pk_last_config_name() == b""


def test_gemm_workspace_arguments(lib):
    good = dict(M=4, N=5, K=6, A=FAKE, lda=6, sa=2 * FAKE, B=3 * FAKE, ldb=6, sb=4 * FAKE, bias=5 * FAKE, C=6 * FAKE,
                dtype=0, ldc=5, workspace=None, workspace_bytes=0)
    _cases(lib, lib.pk_gemm_i8_ws, good, [("M", -1, 1), ("lda", 5, 5), ("A", None, 4), ("C", None, 11), ("dtype", 3, 12), ("ldc", 4, 13)],
           [("lda", 1 << 31)])
    # a product whose rows are laid out: 4096 + 4096 rows of 4097 bytes, 16 MiB each operand and the result
    at = [(8 + i) << 28 for i in range(7)]
    big = dict(M=4096, N=4096, K=4097, A=at[0], lda=4097, sa=at[1], B=at[2], ldb=4097, sb=at[3], bias=at[4], C=at[5],
               dtype=0, ldc=4096, workspace=at[6], workspace_bytes=1 << 28)
    need = lib.pk_gemm_i8_workspace_bytes_for(4096, 4096, 4097, at[0], 4097, at[2], 4097)
    assert need == 8192 * 4224
    overlapping = [(name, at[i] - need + 16) for i, name in enumerate(("A", "sa", "B", "sb", "bias", "C"))]
    _cases(lib, lib.pk_gemm_i8_ws, big, [("workspace", w, 14) for _, w in overlapping], [])


def test_gemm_workspace_query(lib):
    def need(M, N, K, lda, ldb, A=FAKE, B=3 * FAKE):
        return lib.pk_gemm_i8_workspace_bytes_for(M, N, K, A, lda, B, ldb)
    assert need(4096, 4096, 4096, 4096, 4096) == need(4096, 4096, 4096, 4100, 4100) == 0
    assert need(4096, 4096, 4096, 4097, 4096) == need(4096, 4096, 4096, 4096, 4097) == 4096 * 4096
    assert need(4096, 4096, 4096, 4096, 4096, A=FAKE + 1) == 4096 * 4096
    assert need(4096, 4096, 4001, 4001, 4003) == 8192 * 4096
    assert need(1, 4096, 4096, 4097, 4097) == need(64, 64, 64, 65, 65) == need(8192, 8192, 127, 127, 127) == 0
    for bad in ((-1, 9, 9, 9, 9), (9, 0, 9, 9, 9), (9, 9, 0, 9, 9), (4096, 4096, 4001, 4000, 4001), (4096, 4096, 4001, 4001, 1 << 31),
                (4096, 4096, 131073, 131073, 131073)):
        assert need(*bad) == 0
    assert 0 < need(200000, 4096, 5001, 5001, 5001) <= 1 << 30 and need(1 << 20, 4096, 5001, 5001, 5001) == 0


def test_tensors_on_the_cpu_are_refused(lib):
    import torch

    import paper_1904_05347_amd as pk
    x, q, s = torch.ones(4, 8), torch.ones(4, 8, dtype=torch.int8), torch.ones(4)
    for call in (lambda: pk.quantize_i8(x), lambda: pk.rmsnorm_i8(x, torch.ones(8)), lambda: pk.gated_i8(x, x),
                 lambda: pk.dequantize_i8(q, s), lambda: pk.gemm_i8(q, q, s, s)):
        with pytest.raises(TypeError, match="on a HIP device"):
            call()


# ------------------------------------------------------------------ the plain forms themselves

def _in_32_bits(z):
    """The rows of fp32 z quantised as the operators are defined to, in numpy's fp32."""
    a = np.abs(z).max(axis=1, keepdims=True)
    inv = np.float32(127) / a
    return np.rint(z * inv).astype(np.int64), (a / np.float32(127))[:, 0]


def test_plain_rows_hold_32_bit_rounding_and_no_more():
    """The bounds the GPU results are held to pass fp32 arithmetic, and fail it
    with one value a step off, a scale four units off, or a row's sign turned."""
    rng = np.random.default_rng(5)
    z = rng.standard_normal((20, 300)).astype(np.float32)
    q, s = _in_32_bits(z)
    want = plain.rows(z)
    plain.check_rows(q, s, want, "plain")
    for mistake in ((7, 11, 1), (0, 0, -1), (19, 299, 1)):
        off = q.copy()
        off[mistake[0], mistake[1]] += mistake[2]
        with pytest.raises(AssertionError):
            plain.check_rows(off, s, want, "step")
    with pytest.raises(AssertionError):
        plain.check_rows(q, s * np.float32(1 + 2 ** -20), want, "scale")
    with pytest.raises(AssertionError):
        plain.check_rows(-q, s, want, "sign")


def test_plain_norm_gated_and_gemm_against_torch_in_64_bits():
    import torch
    rng = np.random.default_rng(6)
    h, w, u = rng.standard_normal((5, 40)), rng.standard_normal(40), rng.standard_normal((5, 40))
    y = torch.nn.functional.rms_norm(torch.from_numpy(h), (40,), torch.from_numpy(w), 1e-3).numpy()
    assert np.allclose(plain.norm_rows(h, w, 1e-3)[2], np.abs(y).max(axis=1) / 127, rtol=1e-14)
    F = torch.nn.functional
    for name, f in (("silu", F.silu), ("gelu", lambda t: F.gelu(t, approximate="tanh"))):
        z = (f(torch.from_numpy(h)) * torch.from_numpy(u)).numpy()
        lo, hi, s, _, _ = plain.gated_rows(h, u, name)
        assert np.allclose(s, np.abs(z).max(axis=1) / 127, rtol=1e-13)
        assert np.allclose((lo + hi) / 2 * s[:, None], z, atol=1e-13)
    a, b = rng.integers(-128, 128, (4, 9)), rng.integers(-128, 128, (3, 9))
    sa, sb, bias = rng.random(4), rng.random(3), rng.random(3)
    c, _ = plain.gemm(a, b, sa, sb, bias)
    for m in range(4):
        for n in range(3):
            assert np.isclose(c[m, n], sa[m] * sb[n] * sum(int(a[m, k]) * int(b[n, k]) for k in range(9)) + bias[n], rtol=1e-13)
