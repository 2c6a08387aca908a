"""attention_tree on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu
from tests.test_gpu_heads import KINDS, _f64, _normal, _type

pytestmark = pytest.mark.gpu


class Call:
    """One call's inputs: ragged sequences over shuffled pages, NaN in every place that none of them has."""

    def __init__(self, torch, seed, lengths, tokens, Hk, G, d, kind, page=16, tree=True, order="phd", spare=2, scale=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lengths, self.tokens, self.kind, self.G = lengths, tokens, kind, G
        need = [max(1, -(-(max(n, 0) + t) // page)) for n, t in zip(lengths, tokens)]
        pages = sum(need) + spare
        shape, axes = {"phd": ((pages, page, Hk, d), (0, 1, 2, 3)), "hpd": ((pages, Hk, page, d), (0, 2, 1, 3)),
                       "odd": ((pages, page, Hk, d + 1), (0, 1, 2, 3))}[order]
        self.kc, self.vc = (torch.full(shape, float("nan"), dtype=_type(torch, kind), device="cuda").permute(axes)[..., :d]
                            for _ in range(2))
        places = torch.randperm(pages, generator=g, device="cuda").int()
        self.table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, (n, t) in enumerate(zip(lengths, tokens)):
            self.table[b, :need[b]] = places[at:at + need[b]]
            at += need[b]
            j = torch.arange(max(n, 0) + t, device="cuda")
            p, o = self.table[b, j // page].long(), j % page
            self.kc[p, o] = _normal(torch, g, (len(j), Hk, d), kind)
            self.vc[p, o] = _normal(torch, g, (len(j), Hk, d), kind)
        self.q = _normal(torch, g, (sum(tokens), Hk * G, d), kind, 1.5 if scale is None else scale)
        words, starts, rng = [], [0], np.random.default_rng(seed)
        for t in tokens:
            starts.append(starts[-1] + t)
            for i in range(t):
                words.append((words[starts[-2] + int(rng.integers(0, i))] if i else 0) | 1 << i)
        self.set_mask(torch, words if tree else None)
        self.len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.most = max(max(tokens), 1)

    def set_mask(self, torch, words):
        self.mask = None if words is None else torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64,
                                                            device="cuda")

    def __call__(self, pk, **more):
        return pk.attention_tree(self.q, self.kc, self.vc, self.table, self.len, self.starts, self.most, mask=self.mask, **more)

    def check(self, pk, cap=0.0, scale=None, what="", **more):
        out, lse = self(pk, cap=cap, scale=scale, lse=True, **more)
        self.compare(out, lse, cap, scale, what)
        return out, lse

    def compare(self, out, lse, cap=0.0, scale=None, what=""):
        d = self.q.shape[2]
        with np.errstate(invalid="ignore"):
            want, ob, wl, lb, written = plain.attention(
                _f64(self.q), _f64(self.kc), _f64(self.vc), self.table.cpu().numpy(), self.len.cpu().numpy(),
                self.starts.cpu().numpy(), self.most, None if self.mask is None else self.mask.cpu().numpy(),
                d ** -0.5 if scale is None else scale, cap, self.kind)
        assert out.dtype == self.q.dtype and out.shape == self.q.shape
        plain.check(_f64(out)[written], want[written], ob[written], what + " out")
        plain.check(_f64(lse)[written], wl[written], lb[written], what + " lse")


# lengths before the tokens, tokens, heads, query heads of each, channels, positions of a page
CASES = [([0], [1], 1, 1, 64, 16), ([1], [1], 1, 1, 1, 1), ([31, 32, 33], [1, 1, 1], 2, 4, 128, 16),
         ([0, 0, 5], [3, 1, 2], 1, 3, 32, 4), ([127, 128, 129], [1, 2, 3], 2, 1, 80, 24), ([700], [1], 1, 16, 128, 16),
         ([300, 0, 5, 64], [7, 0, 16, 64], 2, 2, 64, 64), ([1000, 10], [5, 33], 1, 7, 96, 7), ([513], [3], 3, 5, 256, 32),
         ([2000], [4], 1, 8, 255, 16), ([259], [64], 1, 4, 7, 256), ([4100], [2], 1, 2, 50, 1), ([40] * 30, [1] * 30, 2, 2, 64, 8),
         ([90] * 300, [1] * 300, 1, 1, 16, 8)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("case", CASES)
def test_attention(case, kind):
    torch, pk = require_gpu()
    lengths, tokens, Hk, G, d, page = case
    for i, (tree, order, cap) in enumerate(((True, "phd", 0.0), (False, "hpd", 0.0), (True, "odd", 3.0))):
        call = Call(torch, 10 * d + i, lengths, tokens, Hk, G, d, kind, page, tree, order)
        call.check(pk, cap=cap, what="%s %s" % (order, tree))
        # without a workspace: nothing is divided
        out, lse = call(pk, cap=cap, lse=True, workspace=torch.empty(0, device="cuda"))
        call.compare(out, lse, cap, None, "undivided")


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_see_nothing(kind):
    torch, pk = require_gpu()
    call = Call(torch, 3, [0, 0, 40], [3, 2, 3], 2, 2, 64, kind)
    call.set_mask(torch, [0, 2, 0, 0, 0, 0, 1, 2 ** 64 - 1])
    out, lse = call.check(pk, what="masks")
    for m in (0, 2, 3, 4):
        assert not out[m].any() and bool((lse[m] == -float("inf")).all())
    # bits of tokens that the sequence does not have are nothing
    call.set_mask(torch, [2 ** 64 - 8, 2, 4, 2 ** 63, 1, 7, 1, 2])
    call.check(pk, what="bits beyond")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128, 200])
def test_nan_and_infinity_reach_the_rows_that_see_them(kind, D):
    torch, pk = require_gpu()
    call = Call(torch, 4, [37, 128], [5, 4], 2, 3, D, kind)
    call.set_mask(torch, [1, 3, 5, 9, 17, 1, 2, 4, 8])
    clean, _ = call(pk, lse=True)
    page = call.table.cpu()

    def place(b, j):
        return int(page[b, j // 16]), j % 16

    # values of tokens 1 and 3 of the first sequence, the key of token 2 of the second
    call.vc[place(0, 37 + 1)][0, 3] = float("nan")
    call.vc[place(0, 37 + 3)][1, D - 1] = -float("inf")
    call.kc[place(1, 128 + 2)][0, 0] = float("nan")
    out, lse = call(pk, lse=True)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[1, :3, 3] = True
    hit[3, 3:, D - 1] = True
    hit[7, :3] = True
    # in the tile that holds them products are made one by one: another order of the same sum
    call_rows = ~hit
    assert torch.isfinite(out[call_rows]).all() and not torch.isfinite(out[hit]).any()
    assert float((out[call_rows].double() - clean[call_rows].double()).abs().max()) < 0.05
    assert bool((out[3, 3:, D - 1] == -float("inf")).all()) and out[7, :3].isnan().all() and lse[7, :3].isnan().all()
    # all that sees a NaN position of the context is NaN, nothing else
    call.kc[place(1, 0)][1, 0] = float("nan")
    out = call(pk)
    assert out[5:, 3:].isnan().all() and torch.isfinite(out[:1]).all() and torch.isfinite(out[5, :3]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_pages_that_are_none_beside_infinities(kind, D):
    """Few rows and many: positions without a page, in tiles whose others hold infinities."""
    torch, pk = require_gpu()
    for T in (2, 40):
        call = Call(torch, 21, [150], [T], 1, 2, D, kind, tree=False)
        p = call.table[0].tolist()
        call.vc[p[2], 3, 0, 5], call.vc[p[5], 1, 0, 6] = float("inf"), -float("inf")
        call.table[0, 1], call.table[0, 4], call.table[0, 7] = -1, 1 << 20, -1
        out, _ = call.check(pk, what="%d tokens" % T)
        assert bool((out[..., 5] == float("inf")).all()) and bool((out[..., 6] == -float("inf")).all())
        # a cache without pages at all
        none = call.kc[:0]
        out = pk.attention_tree(call.q, none, none, call.table, call.len, call.starts, T)
        assert not out.any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,G,T", [(64, 2, 2), (128, 2, 2), (128, 8, 4), (200, 2, 2), (256, 1, 5)])
def test_several_tiles_a_wave(kind, d, G, T):
    """Long sequences: a wave goes from tile to tile, with two stages (a table of many more pages) and with one."""
    torch, pk = require_gpu()
    call = Call(torch, 5 + d, [20001, 77], [T, 1], 3, G, d, kind, page=16)
    one, _ = call.check(pk, what="one stage")
    call.table = torch.cat((call.table, torch.full((2, 20000), -1, dtype=torch.int32, device="cuda")), dim=1)
    two, _ = call.check(pk, what="two stages")
    if d <= 128:   # the shares are other ones, the sums' order too
        assert float((one.double() - two.double()).abs().max()) < 0.02


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_many_rows_over_several_tiles(kind, d):
    torch, pk = require_gpu()
    call = Call(torch, 31 + d, [3001, 0, 700], [20, 5, 33], 2, 4, d, kind, page=48)
    call.check(pk, what="wide")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,Hk,T", [(70, 1, 1), (70, 2, 17), (40, 16, 1), (6, 1, 17), (1, 1, 33)])
def test_joins_of_many_items_and_of_few(B, Hk, T, kind):
    """Parts joined by borders (more than 64 sequences, more items than work-groups) and by items, uneven and empty ones among them."""
    torch, pk = require_gpu()
    lengths = [(997 * b * b) % 2500 if b % 5 else 0 for b in range(B)]
    lengths[-1] = 3000
    tokens = [1 + (b * 7) % T if b % 3 else T for b in range(B)]
    tokens[B // 2] = 0 if B > 1 else T
    call = Call(torch, B + Hk + T, lengths, tokens, Hk, 2, 64, kind)
    call.check(pk, what="B = %d" % B)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [2, 3, 9, 10, 11, 12, 13, 14, 15, 250])
def test_last_chunks_of_every_size(kind, d):
    """A head's end inside 16 bytes, over several tiles of a few rows and of many; nothing beside a head's row is taken."""
    torch, pk = require_gpu()
    for T in (1, 9):
        call = Call(torch, 71 + d, [700, 3], [T, 1], 3, 4, d, kind)
        call.check(pk, what="T = %d" % T)
        before = call.kc[:, :, 1:2].clone(), call.vc[:, :, 1:2].clone(), call.check(pk)[0][:, 4:8].clone()
        call.kc.fill_(float("nan"))
        call.vc.fill_(float("inf"))
        call.kc[:, :, 1:2], call.vc[:, :, 1:2] = before[:2]
        assert torch.equal(call(pk)[:, 4:8], before[2])


@pytest.mark.parametrize("page", [1, 7, 8, 16, 24, 40, 64, 256])
def test_page_sizes_and_layouts_of_their_own(page):
    """Keys and values laid out apart, from any element on."""
    torch, pk = require_gpu()
    for kind, d, T in (("bf16", 128, 1), ("f16", 80, 12), ("f32", 36, 3), ("bf16", 33, 20)):
        call = Call(torch, page + d, [333, 1, 90], [T, 1, 2], 2, 4, d, kind, page)
        n, size, Hk, _ = call.kc.shape
        flat = torch.full((n * size * Hk * d + 1,), float("nan"), dtype=call.kc.dtype, device="cuda")
        shifted = flat[1:].view(n, size, Hk, d)
        shifted.copy_(call.kc)
        call.kc = shifted
        turned = torch.full((Hk, n, size, d + 8), float("nan"), dtype=call.vc.dtype, device="cuda")[..., :d].permute(1, 2, 0, 3)
        turned.copy_(call.vc)
        call.vc = turned
        call.check(pk, what="page %d" % page)


def test_scores_at_the_ends():
    """Large scores of both signs, and equal ones."""
    torch, pk = require_gpu()
    for kind in KINDS:
        for scale in (100.0, 0.0):
            Call(torch, 6, [300, 20], [2, 3], 1, 4, 64, kind, scale=scale).check(pk, what="scale %g" % scale)
        Call(torch, 6, [300], [2], 1, 4, 64, kind).check(pk, scale=-0.3, what="negative")
        Call(torch, 6, [300], [2], 1, 4, 64, kind, scale=100.0).check(pk, cap=0.5, what="capped")


def test_indices_out_of_range_are_left_out():
    """Host and device agree on what is left out (its arithmetic is tested by itself on the CPU)."""
    torch, pk = require_gpu()
    call = Call(torch, 7, [100, 60, 30], [3, 2, 4], 2, 2, 64, "bf16")
    call.table[0, 1], call.table[1, 0], call.table[0, 3] = -5, 1 << 30, call.kc.shape[0]
    call.check(pk, what="pages")
    call.len[2] = -7
    call.table[2, 0] = 0
    call.kc.nan_to_num_(0.5), call.vc.nan_to_num_(0.25)
    call.check(pk, what="negative length")
    call.len[1] = 2 ** 31 - 1   # beyond the table: its tokens have no place
    call.check(pk, what="long length")
    out = torch.full_like(call.q, 7.0)
    lse = torch.full((9, 4), 7.0, device="cuda")
    call.starts = torch.tensor([0, 3, 3, 6], dtype=torch.int32, device="cuda")
    call(pk, out=out, lse=lse)
    assert bool((out[6:] == 7.0).all()) and bool((lse[6:] == 7.0).all()) and not bool((out[:6] == 7.0).all(dim=2).any())
    # tokens beyond `most`, starts that are no rows of q
    call.most, kept = 2, out.fill_(7.0)
    call(pk, out=kept)
    assert bool((kept[2] == 7.0).all()) and bool((kept[5] == 7.0).all()) and not bool((kept[4] == 7.0).all())
    call.starts = torch.tensor([-3, 8, 20, 5], dtype=torch.int32, device="cuda")
    kept.fill_(7.0)
    call(pk, out=kept)
    assert bool((kept[:8] == 7.0).all()) and not bool((kept[8] == 7.0).all())


def test_in_place_strides_and_no_mask_equals_chain():
    torch, pk = require_gpu()
    for kind in KINDS:
        call = Call(torch, 8, [70, 400], [6, 9], 2, 4, 96, kind, tree=False)
        out = call(pk)
        call.set_mask(torch, [(2 << i) - 1 for t in (6, 9) for i in range(t)])
        assert torch.equal(call(pk), out)
        wide = torch.zeros((8, 15, 101), dtype=call.q.dtype, device="cuda")
        view = wide[:, :, 3:99].transpose(0, 1)
        assert call(pk, out=view) is view and torch.equal(view, out) and not wide[:, :, 99:].any() and not wide[:, :, :3].any()
        assert call(pk, out=call.q) is call.q and torch.equal(call.q, out)


def test_deterministic_and_divided_alike():
    torch, pk = require_gpu()
    call = Call(torch, 9, [5000, 3, 900], [4, 1, 2], 2, 4, 128, "bf16")
    a, b = call(pk, lse=True), call(pk, lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_tokens_no_sequences():
    torch, pk = require_gpu()
    call = Call(torch, 9, [5], [1], 1, 2, 64, "f16")
    none = call.q[:0]
    assert pk.attention_tree(none, call.kc, call.vc, call.table, call.len, call.starts * 0, 1).shape == (0, 2, 64)
    out = torch.full_like(call.q, 3.0)
    pk.attention_tree(call.q, call.kc, call.vc, call.table[:0], call.len[:0], call.starts[:1], 1, out=out)
    assert bool((out == 3.0).all())
    # a table without pages: nothing is seen
    out, lse = pk.attention_tree(call.q, call.kc, call.vc, call.table[:, :0], call.len, call.starts, 1, out=out, lse=True)
    assert not out.any() and bool((lse == -float("inf")).all())


def test_cache_beyond_4_gib():
    torch, pk = require_gpu()
    page, d = 16, 128
    pages = (1 << 32) // (page * d) + 64
    kc = torch.zeros((pages, page, 1, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    small = Call(torch, 11, [500], [3], 1, 4, d, "bf16", page)
    n = small.kc.shape[0]
    kc[pages - n:], vc[pages - n:] = small.kc, small.vc
    out = pk.attention_tree(small.q, kc, vc, small.table + (pages - n), small.len, small.starts, 3, mask=small.mask)
    assert torch.equal(out, small(pk))


def test_streams_and_graph():
    torch, pk = require_gpu()
    call = Call(torch, 12, [900, 20, 3000], [4, 1, 8], 2, 4, 128, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = call(pk).clone()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, call(pk))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = call(pk, lse=True)
    for i in range(4):
        # lengths change from replay to replay, as a serving loop's do
        call.len.copy_(torch.tensor([900 - 13 * i, 20 - i, 3000 - 700 * i], dtype=torch.int32, device="cuda"))
        call.q.copy_(torch.randn_like(call.q))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = call(pk, lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i


def test_together():
    """A step of generation: keys and values appended, then attended to, against the same from 64 bits' queries."""
    torch, pk = require_gpu()
    for kind in KINDS:
        call = Call(torch, 13, [50, 7], [3, 2], 2, 4, 64, kind)
        g = torch.Generator(device="cuda").manual_seed(1)
        x = [_normal(torch, g, (5, h, 64), kind) for h in (8, 2, 2)]
        w, f = _normal(torch, g, (64,), kind, 0.1) + 1, pk.rope_frequencies(32)
        positions = torch.tensor([50, 51, 51, 7, 8], device="cuda")
        table = call.table.cpu()
        slots = torch.tensor([int(table[b, j // 16]) * 16 + j % 16 for b, j in ((0, 50), (0, 51), (0, 52), (1, 7), (1, 8))],
                             device="cuda")
        call.q = pk.cache_append(x[1], x[2], call.kc, call.vc, slots, positions, f, w, q=x[0], q_weight=w)
        want_q, want_k = pk.rope_qk(x[0], x[1], positions, f, w, w)
        assert torch.equal(call.q, want_q) and torch.equal(call.kc.reshape(-1, 2, 64)[slots], want_k)
        call.set_mask(torch, [1, 3, 5, 1, 3])
        call.check(pk, what="together")
