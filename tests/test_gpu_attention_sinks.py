"""attention_tree where one position's score is far above the others': these are many, so that
their shares count together, however small each is beside the largest."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu
from tests.test_gpu_heads import KINDS, _f64, _type

pytestmark = pytest.mark.gpu

U = plain.U


def _sequence(torch, kind, scores, values, d, T, G, seed):
    """One sequence whose position j has the score scores[j] (exact in `kind`) in every row, times the
    row's first channel of q, 1 or 1/2; values: of channel 0 and, weaker by position, of the others."""
    n = len(scores)
    page = 16
    pages = -(-(n + T) // page)
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randperm(pages, generator=g, device="cuda").int()[None]
    at = table[0].long().repeat_interleave(page) * page + torch.arange(page, device="cuda").repeat(pages)
    kc = torch.zeros((pages, page, 1, d), dtype=_type(torch, kind), device="cuda")
    vc = torch.zeros_like(kc)
    rows = torch.zeros((n + T, d), dtype=kc.dtype, device="cuda")
    rows[:n, 0] = torch.from_numpy(scores).cuda().to(kc.dtype)
    rows[n:, 0] = -60000.0 if kind == "f16" else -2.0 ** 17   # the drafted tokens take no part
    kc.view(-1, d)[at[:n + T]] = rows
    held = torch.zeros_like(rows)
    held[:n] = torch.from_numpy(values).cuda().to(kc.dtype)[:, None]
    held[:n, 1:] *= (torch.rand((n, d - 1), generator=g, device="cuda") + 0.5).to(kc.dtype)
    vc.view(-1, d)[at[:n + T]] = held
    q = torch.zeros((T, G, d), dtype=kc.dtype, device="cuda")
    q[:, :, 0] = 1.0
    q[1::2, :, 0] = 0.5
    assert np.array_equal(_f64(rows[:n, 0]), scores)
    return dict(q=q, kc=kc, vc=vc, table=table, lengths=torch.tensor([n], dtype=torch.int32, device="cuda"),
                starts=torch.tensor([0, T], dtype=torch.int32, device="cuda"), held=held[:n])


def _check(torch, pk, kind, scores, values, d, T, G, what):
    """A score is one product, exact but for its factor log2(e) and the largest's subtraction (4 U of the
    largest score each), an exponential is off by 2 units; sums of n / 4 + 64 steps; a weight is rounded to 16 bits,
    half a step, at most, and off by two of its type's least numbers where the largest of its tile of 64 positions has
    at least 1: fewer than 2^-15 of a tile's share."""
    s = _sequence(torch, kind, scores, values, d, T, G, len(scores) + d + T)
    n = len(scores)
    v = _f64(s["held"])
    for workspace in (None, torch.empty(0, device="cuda")):
        out, lse = pk.attention_tree(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["starts"], T, scale=1.0, lse=True,
                                     workspace=workspace)
        for row, factor in ((0, 1.0), (1, 0.5)):
            if row >= T:
                continue
            x = scores * factor
            p = np.exp(x - x.max())
            total = p.sum()
            want, share = p @ v / total, p @ np.abs(v) / total
            off = 2 * 4 * U * np.abs(x).max() + 4 * U + (n / 4 + 64) * U
            rounding = 0.0 if kind == "f32" else plain.HALF[kind]
            bound = share * (2 * off + rounding + 2.0 ** -15) * 1.01 + plain.HALF[kind] * np.abs(want) * 1.01 + plain.TINY[kind]
            for h in range(G):
                plain.check(_f64(out)[row, h], want, bound, "%s row %d" % (what, row))
            logs = x.max() + np.log(total)
            plain.check(_f64(lse)[row], np.full(G, logs), np.full(G, off + 4 * U * (1 + abs(logs) + np.abs(x).max())), what + " lse")


# tokens, query heads, channels: few rows (a wave has all), many (the waves share tiles), each of 16 and 32 a wave
FORMS = [(1, 1, 64), (2, 12, 128), (2, 1, 256), (40, 1, 64), (40, 2, 128), (20, 1, 256)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("gap", [12.0, 17.5, 20.0, 26.0, 35.0])
def test_one_far_above_many(gap, form, kind):
    """The first position holds nothing but the largest score; what the others hold has to come through."""
    torch, pk = require_gpu()
    T, G, d = form
    n = 1 << 17
    scores, values = np.full(n, -4.0), np.full(n, 1.0 if gap < 20 else 2.0 ** 14)
    scores[0], values[0] = gap - 4.0, 0.0
    _check(torch, pk, kind, scores, values, d, T, G, "gap %g" % gap)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
def test_scores_that_fall_and_rise(form, kind):
    """Scores that fall by steps far below the first ones', and rise again, with as many positions each time
    as keep a share; far ones at last, which take no part."""
    torch, pk = require_gpu()
    T, G, d = form
    parts = [(8.0, 3), (0.0, 2000), (-6.0, 9000), (-14.0, 30000), (2.0, 500), (9.0, 2), (-8.0, 20000), (-2000.0, 5000), (-16.0, 40000)]
    scores = np.concatenate([np.full(n, s) for s, n in parts])
    values = np.concatenate([np.full(n, 2.0 ** round(min(12.0, (9.0 - s) * 0.7))) for s, n in parts])
    _check(torch, pk, kind, scores, values, d, T, G, "falling")
