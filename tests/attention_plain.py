"""The attention operators from their definitions, in numpy's 64 bits, with bounds on
what fp32 arithmetic and one rounding of the result may add.

U is 2^-24, the largest relative error of an fp32 rounding; HALF[kind] that of the
result's type (half of its eps); TINY[kind] half the spacing of its least numbers."""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def pairs_of(d, pairs, layout):
    i = np.arange(pairs)
    return (i, i + pairs) if layout == "half" else (2 * i, 2 * i + 1)


def rotate(y, positions, frequencies, layout, amplitude, back=False):
    """y (tokens x heads x d) rotated, and for each channel the sum of its pair's magnitudes."""
    out, size = y.copy(), np.abs(y)
    n = len(frequencies)
    if n:
        a, b = pairs_of(y.shape[2], n, layout)
        t = positions.astype(np.longdouble)[:, None] * frequencies.astype(np.longdouble)[None]
        cos, sin = np.cos(t).astype(np.float64)[:, None], np.sin(t).astype(np.float64)[:, None]
        if back:
            sin = -sin
        out[..., a] = amplitude * (y[..., a] * cos - y[..., b] * sin)
        out[..., b] = amplitude * (y[..., b] * cos + y[..., a] * sin)
        size[..., a] = size[..., b] = abs(amplitude) * (np.abs(y[..., a]) + np.abs(y[..., b]))
    return out, size


def rope(x, positions, frequencies, weight, eps, layout, amplitude, kind):
    """(y, bound): a sum of squares of up to 16 values a lane and 6 steps over the lanes
    (23 u, half of that after the root), root, quotient and the two products (6 u),
    cosine and sine (2 units, 4 u), their angle rounded at up to half a turn (pi u), the
    amplitude (u) and the rotation itself (2 u): below 32 u of the pair's magnitudes."""
    y = x
    if weight is not None:
        y = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * weight
    out, size = rotate(y, positions, frequencies, layout, amplitude)
    return out, 32 * U * size + HALF[kind] * np.abs(out) * (1 + 2.0 ** -8) + TINY[kind]


def rope_backward(dy, x, positions, frequencies, weight, eps, layout, amplitude, kind, weight_kind):
    """(dx, bound, dw, bound).  The gradient turned back is off by 12 u of its pair's
    magnitudes G; dx = n (h - s mean(h s)), s = x n, h = g w: 12 + 1 for h, 20 for s
    (twice in the second term), 25 for the mean's sum, 5 for the rest: below 96 u of n (H + |s| mean(H |s|)).
    A weight's gradient is a sum of at most 160 steps for up to 1024 tokens (rounds of a
    work-group, 6 steps over lanes, 8 waves, 64 + 16 work-groups), of terms off by 33 u."""
    g, size = rotate(dy, positions, frequencies, layout, amplitude, back=True)
    if weight is None:
        return g, 12 * U * size + HALF[kind] * np.abs(g) * (1 + 2.0 ** -8) + TINY[kind], None, None
    n = 1 / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    s, h, H = x * n, g * weight, size * np.abs(weight)
    dx = n * (h - s * (h * s).mean(axis=2, keepdims=True))
    bound = 96 * U * n * (H + np.abs(s) * (H * np.abs(s)).mean(axis=2, keepdims=True))
    dw = (g * s).sum(axis=(0, 1))
    return (dx, bound + HALF[kind] * np.abs(dx) * (1 + 2.0 ** -8) + TINY[kind], dw,
            (160 + 33) * U * (size * np.abs(s)).sum(axis=(0, 1)) + HALF[weight_kind] * np.abs(dw) * (1 + 2.0 ** -8) + TINY[weight_kind])


def seen_of(i, length, tokens, word):
    """The positions that token i of a sequence sees, as booleans over length + tokens."""
    bits = np.array([(word >> e & 1) == 1 if word is not None else e <= i for e in range(tokens)], dtype=bool)
    return np.concatenate((np.ones(length, dtype=bool), bits))


def attention(q, kc, vc, table, lengths, starts, most, mask, scale, cap, kind):
    """(out, bound, lse, bound, written): rows that are in no sequence have written False.

    A score's sum of d products is off by d u of the sum of their magnitudes, S (as the
    products of two 16-bit values are exact), its factors and the subtraction of the largest by
    6 u of it, the tanh by 6 u of the score more; a weight by that, both in it and in the sum
    of weights, and by 2 units of the exponential; weights are rounded to 16 bits (half
    a step, or half the least step) before they are multiplied; the sums have n / 4 + 64
    steps (a wave's share and the joining)."""
    M, Hq, d = q.shape
    pages, size, Hk, _ = kc.shape
    G, P = Hq // Hk, table.shape[1]
    out, lse = np.zeros((M, Hq, d)), np.zeros((M, Hq))
    ob, lb, written = np.zeros((M, Hq, d)), np.zeros((M, Hq)), np.zeros(M, dtype=bool)
    for b in range(len(lengths)):
        tokens = min(int(starts[b + 1]) - int(starts[b]), most)
        length = min(max(int(lengths[b]), 0), P * size)
        for i in range(tokens):
            m = int(starts[b]) + i
            written[m] = True
            word = None if mask is None else int(mask[m]) & (1 << 64) - 1
            seen = seen_of(i, length, tokens, word)[:P * size]
            at = [(int(table[b, j // size]), j % size) for j in range(len(seen)) if seen[j]]
            at = [(p, o) for p, o in at if 0 <= p < pages]
            page, place = np.array([p for p, _ in at], dtype=int), np.array([o for _, o in at], dtype=int)
            for h in range(Hq):
                if not at:
                    lse[m, h] = -np.inf
                    continue
                k, v = kc[page, place, h // G], vc[page, place, h // G]
                x = scale * (k @ q[m, h])
                S = abs(scale) * (np.abs(k) @ np.abs(q[m, h]))
                off = (d + 6) * U * S.max()
                if cap:
                    x = cap * np.tanh(x / cap)
                    off += 6 * U * np.abs(x).max()
                off += 4 * U * np.abs(x).max()
                top = x.max()
                p = np.exp(x - top)
                total = p.sum()
                out[m, h], lse[m, h] = p @ v / total, top + np.log(total)
                steps = (len(at) / 4 + 64) * U
                rounding = 0.0 if kind == "f32" else HALF[kind]
                A = p @ np.abs(v) / total
                ob[m, h] = A * (2 * (off + 4 * U + steps) + rounding) * 1.01 + HALF[kind] * np.abs(out[m, h]) * 1.01 + TINY[kind]
                if kind == "f16":
                    ob[m, h] += TINY[kind] * np.abs(v).sum(axis=0) / total
                lb[m, h] = off + 4 * U + steps + 4 * U * abs(lse[m, h])
    return out, ob, lse, lb, written


def check(got, want, bound, what):
    got = np.asarray(got, np.float64)
    bad = ~(np.abs(got - want) <= bound) & ~(np.isinf(want) & (got == want)) & ~(np.isnan(want) & np.isnan(got))
    assert not bad.any(), "%s: %d of %d outside, first at %s: got %r want %r bound %.3g" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(bound, want.shape)[bad][0])
