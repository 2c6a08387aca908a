"""What a softmax's weights lose on their way to the values: less than the result's own rounding."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu
from tests.test_gpu_attention import Call
from tests.test_gpu_heads import _f64

pytestmark = pytest.mark.gpu

U = plain.U
# of a weight: bf16's two numbers hold 2^-16 of it; fp16's are each cut off, at 2^-10 of themselves (the second is
# below 2^-10 of the weight) or at 2^-24, where the largest of a tile's 64 positions is 1 or more: 2^-17 of the
# largest value for all of them
OF_WEIGHT = {"bf16": 2.0 ** -16, "f16": 2.0 ** -20}
OF_VALUE = {"bf16": 0.0, "f16": 2.0 ** -17}


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("T,G,d,page", [(1, 1, 64, 16), (1, 4, 128, 16), (3, 8, 128, 16), (1, 16, 256, 16), (5, 4, 80, 24), (9, 4, 33, 7),
                                        (20, 2, 64, 16), (40, 2, 128, 16), (64, 4, 128, 32), (40, 1, 250, 16), (33, 4, 100, 7)])
def test_weights_lose_less_than_the_result(T, G, d, page, kind):
    """The bound of the other tests without the rounding of weights to 16 bits.  Few positions, so that each weight counts."""
    torch, pk = require_gpu()
    lengths, tokens = [0, 1, 2, 5, 40], [min(T, n) for n in (3, 4, T, T, T)]
    call = Call(torch, d + T, lengths, tokens, 2, G, d, kind, page)
    for workspace in (None, torch.empty(0, device="cuda")):
        out, lse = call(pk, lse=True, workspace=workspace)
        q, kc, vc = _f64(call.q), _f64(call.kc), _f64(call.vc)
        table, words = call.table.cpu().numpy(), call.mask.cpu().numpy()
        m = 0
        for b, (n, t) in enumerate(zip(lengths, tokens)):
            at = [(int(table[b, j // page]), j % page) for j in range(n + t)]
            k, v = (np.stack([c[p, o] for p, o in at]) for c in (kc, vc))
            for i in range(t):
                seen = plain.seen_of(i, n, t, int(words[m]) & (1 << 64) - 1)
                for h in range(2 * G):
                    x = d ** -0.5 * (k[seen, h // G] @ q[m, h])
                    size = d ** -0.5 * (np.abs(k[seen, h // G]) @ np.abs(q[m, h])).max()
                    off = (d + 6) * U * size + 4 * U * np.abs(x).max() + 4 * U + (seen.sum() / 4 + 64) * U
                    p = np.exp(x - x.max())
                    p /= p.sum()
                    held = v[seen, h // G]
                    want, share = p @ held, p @ np.abs(held)
                    bound = (share * (2 * off + OF_WEIGHT[kind]) + OF_VALUE[kind] * np.abs(held).max(axis=0)) * 1.01 \
                        + plain.HALF[kind] * np.abs(want) * 1.01 + plain.TINY[kind]
                    plain.check(_f64(out[m, h]), want, bound, "token %d of sequence %d, head %d" % (i, b, h))
                m += 1


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,G,d,page", [(2, 2, 64, 16), (2, 12, 128, 16), (1, 4, 40, 7), (2, 2, 256, 16), (40, 1, 64, 16), (40, 2, 128, 32),
                                        (40, 3, 120, 24), (20, 2, 72, 7), (20, 1, 250, 16)])
def test_infinities_that_all_rows_see(T, G, d, page, kind):
    """Infinities and NaN among a context's values, in tiles that every row sees whole: weights of exactly 1 (equal
    scores), of other sizes, and small ones."""
    torch, pk = require_gpu()
    for scale in (0.0, 1.5, 4.0):
        call = Call(torch, d + T, [700, 300], [T, 1], 2, G, d, kind, page, scale=scale)
        where = call.table.cpu()

        def place(b, j):
            return int(where[b, j // page]), j % page

        def inf(b, j, h, c, what):
            call.vc[place(b, j)][h, c] = float(what)

        clean, _ = call(pk, lse=True)
        inf(0, 3, 0, 5, "inf"), inf(0, 70, 0, 6, "-inf"), inf(0, 333, 1, d - 1, "inf"), inf(1, 64, 1, 0, "-inf")
        inf(0, 200, 1, 1, "inf"), inf(0, 650, 1, 1, "-inf"), inf(0, 100, 1, 2, "nan")
        for more in (dict(), dict(workspace=torch.empty(0, device="cuda"))):
            out, lse = call.check(pk, what="scale %g" % scale, **more)
            a, b = out[:T], out[T:]
            assert bool((a[:, :G, 5] == float("inf")).all()) and bool((a[:, :G, 6] == -float("inf")).all())
            assert bool((a[:, G:, d - 1] == float("inf")).all()) and bool((b[:, G:, 0] == -float("inf")).all())
            assert a[:, G:, 1].isnan().all() and a[:, G:, 2].isnan().all() and torch.isfinite(lse).all()
            rest = torch.ones_like(out, dtype=torch.bool)
            rest[:T, :G, 5:7] = rest[:T, G:, 1:3] = False
            rest[:T, G:, d - 1] = rest[T:, G:, 0] = False
            assert torch.isfinite(out[rest]).all()
            # another order of the same sums
            assert float((out[rest].double() - clean[rest].double()).abs().max()) < 0.05
        # a part that is gone through again, its rows' memory being the result's
        q = call.q.clone()
        out = call(pk)
        for workspace in (None, torch.empty(0, device="cuda")):
            want = call(pk, workspace=workspace)
            assert call(pk, out=call.q, workspace=workspace) is call.q and torch.equal(call.q.nan_to_num(7.0), want.nan_to_num(7.0))
            call.q.copy_(q)
        again = call(pk, lse=True)
        assert torch.equal(again[0].nan_to_num(7.0), call(pk).nan_to_num(7.0))


@pytest.mark.parametrize("T,G,d", [(1, 1, 64), (2, 12, 128), (40, 1, 64), (40, 2, 128)])
def test_an_infinity_of_little_weight(T, G, d):
    """fp16: an infinite value far below the largest score, in another tile than that."""
    torch, pk = require_gpu()
    call = Call(torch, 3, [500], [T], 1, G, d, "f16", tree=False)
    call.kc.nan_to_num_(0.0).zero_(), call.vc.nan_to_num_(0.0)
    call.q.zero_()
    call.q[..., 0] = 1
    table = call.table[0].long()
    call.kc[table[0], 0, 0, 0] = 21.0   # e^-21 = 2^-30.3 for all others
    call.vc[table[20], 3, 0, 1] = float("inf")
    out, _ = call.check(pk, scale=1.0, what="little")
    assert bool((out[:, :, 1] == float("inf")).all()) and torch.isfinite(out[:, :, 2:]).all() and torch.isfinite(out[:, :, 0]).all()
