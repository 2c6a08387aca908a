"""The 8-bit operators from their definitions, in 64 bits (numpy), and how far
32-bit arithmetic may be from them."""
import numpy as np

U32 = 2.0 ** -24   # half a unit in the last place of a 32-bit value, relative
LEAST = 127.0 * 2.0 ** -126   # a row whose largest magnitude is below it is a row of zeros


def rows(z, rel=0.0, row_factor=None, row_rel=U32):
    """What a row z (64-bit, each value known to the relative error `rel`) may be
    quantised to: (lo, hi) bounds of q as real numbers, the scale and its
    relative error.  q rounds z * (127 / a): two more roundings, each half a unit
    of 32 bits, of a value of at most 127.  row_factor: a factor of the whole
    row, in the scale alone, known to row_rel."""
    z = np.asarray(z, np.float64)
    M, N = z.shape
    rel = np.broadcast_to(np.asarray(rel, np.float64), z.shape)
    a = np.abs(z).max(axis=1) if N else np.zeros(M)
    live = (a >= LEAST) & np.isfinite(a)
    near = np.abs(z) >= (a * (1 - 1e-2))[:, None]   # whose magnitude may come out as the largest
    arel = np.where(near, rel, 0.0).max(axis=1) if N else np.zeros(M)
    with np.errstate(all="ignore"):
        y = np.where(live[:, None], z * (127.0 / a)[:, None], 0.0)
    slack = np.abs(y) * (rel + arel[:, None] + 3 * U32)
    f = np.ones(M) if row_factor is None else row_factor
    scale = np.where(live, a * f / 127.0, np.where(np.isfinite(a), 0.0, a))
    return y - 0.5 - slack, y + 0.5 + slack, scale, arel + row_rel + 4 * U32, live


def check_rows(q, scale, want, what):
    lo, hi, s, srel, live = want
    q = np.asarray(q, np.float64)
    assert q.shape == lo.shape, what
    bad = ~((q >= lo) & (q <= hi))
    assert not bad.any(), (what, np.argwhere(bad)[:4], q[bad][:4], lo[bad][:4], hi[bad][:4])
    scale = np.asarray(scale, np.float64)
    assert np.array_equal(np.isnan(scale), np.isnan(s)), what
    inf = np.isinf(s)
    assert np.array_equal(scale[inf], s[inf]), what
    fin = np.isfinite(s)
    assert (np.abs(scale[fin] - s[fin]) <= s[fin] * srel[fin]).all(), (what, scale[fin][:4], s[fin][:4])
    assert (q[~live] == 0).all() and (scale[~live & fin] == 0).all(), what


def norm_rows(h, w, eps):
    """h (as stored) and w in 64 bits -> rows() of the norm.  h * w is rounded
    once; the sum of squares is added in chains of at most N / 256 + 8 terms in a
    work-item and 22 across them, each addition half a unit, and a root halves
    what that comes to; the mean, the addition of eps, the root, its reciprocal
    and the product are five more roundings."""
    N = h.shape[1]
    with np.errstate(all="ignore"):
        f = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return rows(h * w, rel=U32, row_factor=f, row_rel=((N / 256 + 30) / 2 + 5) * U32)


def act(g, name):
    with np.errstate(all="ignore"):
        t = g if name == "silu" else 2 * np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
        return g / (1 + np.exp(-t)), t


def gated_rows(g, u, name):
    """act(g) * u.  exp(-t) is known to two units plus what t's own error (four
    units of it in gelu's polynomial, none in silu's, and one where the
    exponential reduces it) makes of it, |t| times that; the sum, the quotient
    and the product are three more roundings."""
    a, t = act(g, name)
    return rows(a * u, rel=(7 + 6 * np.minimum(np.abs(t), 200.0)) * U32)


def gemm(a, b, sa, sb, bias):
    """(c, bound of the 32-bit arithmetic): the integer sum is exact; its
    conversion, the scales' product, the product of both and the addition of
    the bias each round once."""
    acc = a.astype(np.float64) @ b.astype(np.float64).T   # below 2^53: exact
    p = acc * (sa.astype(np.float64)[:, None] * sb.astype(np.float64)[None, :])
    c = p if bias is None else p + bias.astype(np.float64)
    size = np.abs(p) + (0 if bias is None else np.abs(bias.astype(np.float64)))
    return c, 4.01 * U32 * size


def check_values(got, want, bound, kind, what):
    """got, a 32-bit value within `bound` of the 64-bit `want` and then rounded to
    `kind`: rounding keeps order, so it lies between the bounds' own roundings."""
    import torch
    T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, what
    lo, hi = (torch.from_numpy(np.ascontiguousarray(v)).float().to(T).double().numpy() for v in (want - bound, want + bound))
    ok = (got >= lo) & (got <= hi)
    assert ok.all(), (what, np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4])
