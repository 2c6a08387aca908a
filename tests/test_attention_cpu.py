"""The attention operators' host side, on the CPU: which argument a refused call names,
empty calls, which tensors share memory, how work is divided, and the plain forms
themselves.  No call here reaches the GPU."""
import ctypes
import itertools
import os
import subprocess

import numpy as np
import pytest

from tests import attention_plain as plain

AT = 1 << 20   # addresses that are never read: every call fails its checks or is empty


@pytest.fixture(scope="module")
def lib():
    from paper_1904_05347_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    return binding.load()


@pytest.fixture(scope="module")
def shim(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    out = str(tmp_path_factory.mktemp("heads") / "heads_shim.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", "-o", out, os.path.join(here, "heads_shim.cpp")],
                   check=True)
    s = ctypes.CDLL(out)
    s.shim_share.restype = ctypes.c_int64
    s.shim_share.argtypes = [ctypes.c_int64] * 2
    s.shim_slot.argtypes = [ctypes.c_int64] * 2
    return s


def _heads(at, heads, token, head, M=None):
    from paper_1904_05347_amd.binding import Heads
    return Heads(at * AT if at else None, heads, token, head)


def _rot(pairs=4, positions=30, frequencies=31):
    from paper_1904_05347_amd.binding import Rotation
    return Rotation(positions * AT if positions else None, frequencies * AT if frequencies else None, pairs, 0, 1.0)


def _cache(key=20, value=22, pages=4, size=16, heads=2, k=(16 * 16, 16, 8), v=(16 * 16, 16, 8)):
    from paper_1904_05347_amd.binding import Cache
    i3 = ctypes.c_int64 * 3
    return Cache(key * AT if key else None, value * AT if value else None, pages, size, heads, i3(*k), i3(*v))


def _cases(lib, fn, good, bad, not_supported=()):
    def call(**change):
        args = [{**good, **change}[k] for k in good]
        return fn(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args], None)
    for key, value, position in bad:
        st = call(**{key: value})
        assert (st, lib.pk_last_invalid_param()) == (1, position), (key, getattr(value, "_fields_", value), st, lib.pk_last_invalid_param())
    for key, value in not_supported:
        assert call(**{key: value}) == 2, key


def test_rope_arguments(lib):
    q, k = _heads(1, 4, 48, 8), _heads(2, 2, 48, 8)
    good = dict(dtype=0, M=3, d=8, q=q, k=k, rot=_rot(), qw=5 * AT, kw=6 * AT, wt=0, eps=1e-6, qo=_heads(7, 4, 32, 8),
                ko=_heads(8, 2, 16, 8))
    _cases(lib, lib.pk_rope_qk, good,
           [("dtype", 3, 1), ("M", -1, 2), ("d", 0, 3), ("q", _heads(0, 4, 48, 8), 4), ("q", _heads(1, -4, 48, 8), 11),
            ("q", _heads(1, 4, -1, 8), 4), ("k", _heads(2, 2, 48, -8), 5), ("rot", _rot(5), 6), ("rot", _rot(-1), 6),
            ("rot", _rot(4, 0), 6), ("rot", _rot(4, 30, 0), 6), ("qw", 5 * AT + 1, 7), ("kw", 6 * AT + 2, 8), ("wt", 1, 9),
            ("wt", 7, 9), ("eps", -1.0, 10), ("eps", float("nan"), 10), ("qo", None, 11), ("qo", _heads(7, 3, 32, 8), 11),
            ("qo", _heads(0, 4, 32, 8), 11), ("qo", _heads(7, 4, 31, 8), 11), ("qo", _heads(7, 4, 0, 8), 11),
            ("qo", _heads(1, 4, 32, 8), 11), ("qo", _heads(2, 4, 48, 8), 11), ("qo", _heads(5, 4, 32, 8), 11),
            ("qo", _heads(30, 4, 32, 8), 11), ("qo", _heads(31, 4, 32, 8), 11), ("ko", None, 12), ("ko", _heads(8, 1, 16, 8), 12),
            ("ko", _heads(7, 2, 16, 8), 12), ("ko", _heads(1, 2, 16, 8), 12), ("ko", _heads(6, 2, 16, 8), 12), ("q", None, 7), ("k", None, 8)],
           [("d", 257), ("M", 1 << 31), ("q", _heads(1, 4, 1 << 31, 8))])
    for more in (dict(M=0), dict(q=_heads(0, 0, 0, 0), qo=_heads(0, 0, 0, 0), k=None, ko=None, kw=None)):
        args = {**good, **more}
        assert lib.pk_rope_qk(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args.values()], None) == 0
    assert lib.pk_last_config_name() == b""


def test_rope_backward_arguments(lib):
    good = dict(dtype=0, M=3, d=8, dq=_heads(1, 4, 48, 8), dk=_heads(2, 2, 48, 8), q=_heads(3, 4, 32, 8), k=_heads(4, 2, 16, 8),
                rot=_rot(), qw=5 * AT, kw=6 * AT, wt=0, eps=1e-6, gq=_heads(7, 4, 32, 8), gk=_heads(8, 2, 16, 8), gqw=9 * AT,
                gkw=10 * AT, ws=11 * AT, bytes=3 * 2 * 8 * 4)
    assert lib.pk_rope_qk_backward_workspace_bytes(3, 8) == 192
    assert lib.pk_rope_qk_backward_workspace_bytes(0, 8) == lib.pk_rope_qk_backward_workspace_bytes(3, 257) == 0
    assert lib.pk_rope_qk_backward_workspace_bytes(10 ** 6, 256) == 1024 * 512 * 4
    _cases(lib, lib.pk_rope_qk_backward, good,
           [("dtype", -1, 1), ("M", -1, 2), ("d", 0, 3), ("dq", _heads(1, 3, 48, 8), 6), ("dk", None, 7), ("q", None, 6), ("k", None, 7),
            ("q", _heads(3, 3, 32, 8), 6), ("q", _heads(0, 4, 32, 8), 6), ("rot", _rot(5), 8), ("qw", 5 * AT + 1, 9),
            ("kw", 6 * AT + 2, 10), ("wt", 2, 11), ("eps", -1.0, 12), ("gq", None, 13), ("gq", _heads(7, 4, 16, 8), 13),
            ("gq", _heads(3, 4, 32, 8), 13), ("gq", _heads(1, 4, 40, 8), 13), ("gk", None, 14), ("gk", _heads(7, 2, 16, 8), 14),
            ("gk", _heads(6, 2, 16, 8), 14), ("gqw", None, 15), ("gqw", 9 * AT + 2, 15), ("gqw", 5 * AT, 15), ("gqw", 7 * AT, 15),
            ("gkw", None, 16), ("gkw", 9 * AT + 4, 16), ("qw", None, 15), ("ws", 11 * AT + 8, 17), ("ws", 9 * AT + 16, 17),
            ("ws", 3 * AT, 17), ("ws", 31 * AT, 17)], [("d", 300)])
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in good.values()]
    for ws, n in ((None, 1 << 20), (11 * AT, 191)):
        assert lib.pk_rope_qk_backward(*args[:16], ws, n, None) == 3


def test_append_arguments(lib):
    good = dict(dtype=0, M=3, d=8, q=_heads(1, 4, 64, 8), k=_heads(2, 2, 64, 8), v=_heads(3, 2, 64, 8), rot=_rot(), qw=5 * AT,
                kw=6 * AT, wt=0, eps=0.0, qo=_heads(7, 4, 32, 8), cache=_cache(), slots=9 * AT)
    _cases(lib, lib.pk_cache_append, good,
           [("dtype", 3, 1), ("M", -1, 2), ("d", 0, 3), ("q", _heads(0, 4, 64, 8), 4), ("k", None, 5), ("k", _heads(0, 2, 64, 8), 5),
            ("v", None, 6), ("v", _heads(3, 1, 64, 8), 6), ("v", _heads(0, 2, 64, 8), 6), ("rot", _rot(5), 7), ("qw", 5 * AT + 1, 8),
            ("kw", 6 * AT + 1, 9), ("wt", 1, 10), ("eps", float("nan"), 11), ("qo", None, 12), ("qo", _heads(3, 4, 32, 8), 12),
            ("qo", _heads(9, 4, 32, 8), 12), ("cache", None, 13), ("cache", _cache(heads=3), 13), ("cache", _cache(key=0), 13),
            ("cache", _cache(size=0), 13), ("cache", _cache(pages=-1), 13), ("cache", _cache(k=(256, 15, 8)), 13),
            ("cache", _cache(v=(255, 16, 8)), 13), ("cache", _cache(v=(256, 16, 7)), 13), ("cache", _cache(key=20, value=20), 13),
            ("cache", _cache(key=2), 13), ("cache", _cache(value=3), 13), ("cache", _cache(value=9), 13), ("cache", _cache(key=7), 13),
            ("cache", _cache(key=30), 13), ("cache", _cache(k=(-256, 16, 8)), 13), ("slots", None, 14), ("slots", 9 * AT + 4, 14),
            ("q", None, 8)],
           [("d", 257), ("cache", _cache(k=(1 << 41, 16, 8)))])


def test_attention_arguments(lib):
    def wide(**more):   # three pages of 256: enough units for a workspace to be used
        return _cache(**{**dict(size=256, k=(4096, 16, 8), v=(4096, 16, 8)), **more})

    good = dict(dtype=0, M=3, d=8, q=_heads(1, 4, 32, 8), cache=wide(), table=4 * AT, B=2, P=3, ld=3, lengths=5 * AT, starts=6 * AT,
                most=3, mask=7 * AT, scale=1.0, cap=0.0, out=_heads(8, 4, 32, 8), lse=9 * AT, ld_lse=4, ws=10 * AT, bytes=1 << 20)
    _cases(lib, lib.pk_attention_tree, good,
           [("dtype", 3, 1), ("M", -1, 2), ("d", 0, 3), ("q", None, 4), ("q", _heads(0, 4, 32, 8), 4), ("cache", None, 5),
            ("cache", wide(heads=0), 5), ("cache", wide(heads=3), 5), ("cache", wide(value=0), 5), ("cache", wide(size=0), 5),
            ("table", None, 6), ("table", 4 * AT + 2, 6), ("B", -1, 7), ("P", -1, 8), ("ld", 2, 9), ("lengths", None, 10),
            ("lengths", 5 * AT + 1, 10), ("starts", None, 11), ("starts", 6 * AT + 2, 11), ("most", 0, 12), ("mask", 7 * AT + 4, 13),
            ("cap", -1.0, 15), ("cap", float("nan"), 15), ("cap", float("inf"), 15), ("out", None, 16), ("out", _heads(8, 2, 32, 8), 16),
            ("out", _heads(1, 4, 40, 8), 16), ("out", _heads(20, 4, 32, 8), 16), ("out", _heads(8, 4, 24, 8), 16), ("out", _heads(7, 4, 32, 8), 16),
            ("lse", 9 * AT + 2, 17), ("lse", 8 * AT, 17), ("lse", 5 * AT, 17), ("ld_lse", 3, 18), ("ws", 10 * AT + 8, 19),
            ("ws", 9 * AT + 16, 19), ("ws", 8 * AT, 19), ("ws", 22 * AT, 19)],
           [("d", 257), ("most", 65), ("ld", 1 << 31), ("cache", wide(size=1 << 30))])
    args = [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in good.values()]
    for i, v in ((1, 0), (6, 0)):
        assert lib.pk_attention_tree(*args[:i], v, *args[i + 1:], None) == 0


def test_attention_workspace(lib):
    need = lib.pk_attention_tree_workspace_bytes
    # (type, channels, query heads, heads, sequences, pages, positions of a page, tokens)
    assert need(1, 128, 32, 8, 1, 256, 16, 1) > 0
    assert need(1, 128, 32, 8, 1, 32, 16, 1) == 0         # a few units: not divided
    for bad in ((3, 128, 32, 8, 1, 256, 16, 1), (1, 0, 32, 8, 1, 256, 16, 1), (1, 257, 32, 8, 1, 256, 16, 1), (1, 128, 31, 8, 1, 256, 16, 1),
                (1, 128, 32, 0, 1, 256, 16, 1), (1, 128, 32, 8, 0, 256, 16, 1), (1, 128, 32, 8, 1, 0, 16, 1), (1, 128, 32, 8, 1, 256, 0, 1),
                (1, 128, 32, 8, 1, 256, 16, 0), (1, 128, 32, 8, 1, 256, 16, 65), (1, 128, 32, 8, 1, 1 << 30, 1 << 30, 1)):
        assert need(*bad) == 0
    assert need(0, 256, 1 << 16, 1 << 16, 1 << 30, 1 << 15, 1 << 15, 64) < 1 << 31


def test_tensors_on_the_cpu_are_refused(lib):
    import torch

    import paper_1904_05347_amd as pk
    x, i = torch.ones(2, 4, 8), torch.zeros(2, dtype=torch.int64)
    cache = torch.ones(2, 4, 4, 8)
    n = i.int()
    for call in (lambda: pk.rope_qk(x, x, None, None), lambda: pk.rope_qk_backward(x, x, x, x, None, None),
                 lambda: pk.cache_append(x, x, cache, cache, i),
                 lambda: pk.attention_tree(x, cache, cache, n.view(1, 2), n[:1], n, 1)):
        with pytest.raises(TypeError, match="on a HIP device"):
            call()


# ------------------------------------------------------------------ where tensors lie

def _bytes_of(v):
    at, run, dims = v[0], v[1], [(v[2 + 2 * i], v[3 + 2 * i]) for i in range(3)]
    return [at + sum(i * s for i, (_, s) in zip(index, dims)) + e
            for index in itertools.product(*(range(n) for n, _ in dims)) for e in range(run)]


def test_shared_memory_is_found(shim):
    """Against sets of bytes: what is shared is always found; and views that a program cuts
    from one tensor are told apart."""
    rng = np.random.default_rng(0)
    arr = ctypes.c_int64 * 8

    def draw():
        return [int(rng.integers(0, 60)), int(rng.integers(1, 5))] + [int(x) for _ in range(3) for x in (rng.integers(1, 4), rng.integers(0, 20))]

    apart = 0
    for _ in range(4000):
        a, b = draw(), draw()
        if rng.random() < 0.5:
            b[2:] = a[2:]
        truth = bool(set(_bytes_of(a)) & set(_bytes_of(b)))
        told = bool(shim.shim_shared(arr(*a), arr(*b)))
        assert told or not truth, (a, b)
        apart += not told
        own = _bytes_of(a)
        if shim.shim_distinct(arr(*a)):
            assert len(set(own)) == len(own), a
    assert apart > 500
    # queries, keys and values of one projection; halves of one cache; heads in between
    row, d = 60, 4
    q, k, v = ([0, d, 9, row, 8, d, 1, 0], [8 * d, d, 9, row, 3, d, 1, 0], [11 * d, d, 9, row, 3, d, 1, 0])
    for a, b in itertools.permutations((q, k, v), 2):
        assert not shim.shim_shared(arr(*a), arr(*b))
        assert shim.shim_distinct(arr(*a))
    for a, b in (([0, 4, 5, 128, 8, 8, 2, 4], [64, 4, 5, 128, 8, 8, 2, 4]), ([0, 4, 5, 128, 8, 16, 1, 4], [4, 4, 5, 128, 8, 16, 1, 4]),
                 ([0, 4, 5, 256, 8, 32, 2, 8], [4, 4, 5, 256, 8, 32, 2, 8])):
        assert not shim.shim_shared(arr(*a), arr(*b)) and not shim.shim_shared(arr(*b), arr(*a))


# ------------------------------------------------------------------ how work is divided

def test_heads_fit_their_lanes(shim):
    out = (ctypes.c_int * 6)()
    for E in (4, 8):
        for d in range(1, 257):
            for pairs in {0, 1, d // 4, d // 2}:
                if 2 * pairs > d:
                    continue
                for rows in (1, 2, 3, 7, 16, 40, 48, 129, 1000, 200000):
                    shim.shim_tiling(d, pairs, E, ctypes.c_int64(rows), out)
                    pc, chunks, team, threads, teams, tokens = out
                    assert pc * E >= pairs and (pc - 1) * E < max(pairs, 1)
                    assert (chunks - pc) * 2 * E >= d - 2 * pairs
                    assert chunks <= team <= 64 and team & team - 1 == 0
                    assert threads % 64 == 0 and 64 <= threads <= 512 and teams == threads // team
                    assert tokens >= 1 and (tokens == 1 or tokens * rows <= teams) and tokens * pairs <= 2048
                    if tokens == 1:
                        rounds = -(-rows // teams)
                        assert rounds * teams < rows + teams


def _divide(shim, M, capacity, heads, group, most, rows, unit, tail, starts, lengths, groups):
    """The kernel's walk: {(sequence, head, group): [(work-group, slot, begin, end)]}."""
    o = (ctypes.c_int64 * 6)()
    line = []
    for b in range(len(lengths)):
        shim.shim_sequence(*(ctypes.c_int64(v) for v in (M, capacity)), group, most, rows, unit, tail,
                           *(ctypes.c_int64(v) for v in (starts[b], starts[b + 1], lengths[b])), o)
        for h in range(heads):
            for g in range(o[4]):
                line.append(((b, h, g), o[5]))
    total = sum(n for _, n in line)
    each = shim.shim_share(total, groups)
    assert each * groups >= total
    parts, at = {}, 0
    for item, n in line:
        u = at
        while u < at + n:
            w = u // each
            end = min(at + n, (w + 1) * each)
            parts.setdefault(item, []).append((w, shim.shim_slot(u, w * each), u - at, end - at))
            u = end
        at += n
    return parts, total, each


def test_units_are_divided_once(shim):
    rng = np.random.default_rng(1)
    for _ in range(300):
        B, heads, group, rows = (int(rng.integers(1, n)) for n in (9, 4, 6, 3))
        rows *= 16
        tokens = rng.integers(0, 9, B)
        starts = [0] + [int(x) for x in np.cumsum(tokens)]
        lengths = [int(x) for x in rng.integers(-3, 3000, B)]
        capacity, groups = int(rng.integers(1, 3000)), int(rng.integers(1, 40))
        parts, total, each = _divide(shim, starts[-1], capacity, heads, group, 8, rows, 128, int(rng.choice([0, 64])), starts, lengths, groups)
        used = {}
        for item, ps in parts.items():
            assert ps[0][2] == 0 and all(a[3] == b[2] for a, b in zip(ps, ps[1:]))
            if len(ps) > 1:
                for w, slot, *_ in ps:
                    assert w < groups and used.setdefault((w, slot), item) == item, "two items in one slot"
        for b in range(B):
            if tokens[b]:
                assert (b, heads - 1, -(-int(tokens[b]) * group // rows) - 1) in parts
            else:
                assert not any(i[0] == b for i in parts)


def test_indices_are_held_to_what_is_there(shim):
    o = (ctypes.c_int64 * 6)()
    odd = [0, 1, 5, 9, 10, 11, -1, -7, 2 ** 31 - 1, -2 ** 31, 64, 100]
    for start, end, length in itertools.product(odd, odd, odd):
        for M, capacity, most, tail in ((10, 48, 4, 0), (10, 0, 64, 64), (10, 1000, 64, 64), (70, 1000, 64, 0)):
            shim.shim_sequence(ctypes.c_int64(M), ctypes.c_int64(capacity), 3, most, 16, 128, tail, ctypes.c_int64(start), ctypes.c_int64(end),
                               ctypes.c_int64(length), o)
            first, n, keys, tokens, groups, units = o
            assert 0 <= tokens <= most and (tokens == 0 or 0 <= first and first + tokens <= M)
            assert 0 <= n <= keys <= capacity and groups * 16 >= tokens * 3 and units >= 1 and units * 128 + tail >= keys and (units == 1 or (units - 1) * 128 + tail < keys)


# ------------------------------------------------------------------ the plain forms themselves

def test_plain_rotation_by_complex_numbers_and_gradient_by_differences():
    rng = np.random.default_rng(2)
    x, w, f = rng.standard_normal((3, 2, 10)), rng.standard_normal(10), np.array([1.0, 0.1, 0.01])
    positions, dy = np.array([0, 7, -3]), rng.standard_normal((3, 2, 10))
    for layout in ("half", "interleaved"):
        a, b = plain.pairs_of(10, 3, layout)
        y, _ = plain.rotate(x, positions, f, layout, 1.5)
        z = 1.5 * (x[..., a] + 1j * x[..., b]) * np.exp(1j * positions[:, None] * f)[:, None]
        assert np.allclose(y[..., a], z.real) and np.allclose(y[..., b], z.imag) and np.array_equal(y[..., 6:], x[..., 6:])

        def loss(x, w):
            return (plain.rope(x, positions, f, w, 1e-3, layout, 1.5, "f32")[0] * dy).sum()

        dx, _, dw, _ = plain.rope_backward(dy, x, positions, f, w, 1e-3, layout, 1.5, "f32", "f32")
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = 1e-6
            assert abs((loss(x + e, w) - loss(x - e, w)) / 2e-6 - dx[i]) < 1e-6
        for i in range(10):
            e = np.zeros(10)
            e[i] = 1e-6
            assert abs((loss(x, w + e) - loss(x, w - e)) / 2e-6 - dw[i]) < 1e-6


def test_plain_attention_against_torch_in_64_bits():
    import torch
    rng = np.random.default_rng(3)
    d, page, Hk, G = 5, 4, 2, 2
    lengths, starts = np.array([6, 3]), np.array([0, 3, 5])
    kc, vc, q = rng.standard_normal((6, page, Hk, d)), rng.standard_normal((6, page, Hk, d)), rng.standard_normal((5, Hk * G, d))
    table = np.array([[5, 0, 2], [1, 3, 4]])
    out, _, lse, _, written = plain.attention(q, kc, vc, table, lengths, starts, 3, None, 0.7, 0.0, "f32")
    assert written.all()
    for b in range(2):
        n, t = lengths[b], starts[b + 1] - starts[b]
        k = torch.from_numpy(kc[table[b]].reshape(-1, Hk, d)[:n + t]).repeat_interleave(G, 1).transpose(0, 1)
        v = torch.from_numpy(vc[table[b]].reshape(-1, Hk, d)[:n + t]).repeat_interleave(G, 1).transpose(0, 1)
        mask = torch.ones(t, n + t, dtype=torch.bool).tril(n)
        x = torch.from_numpy(q[starts[b]:starts[b + 1]]).transpose(0, 1)
        want = torch.nn.functional.scaled_dot_product_attention(x, k, v, attn_mask=mask, scale=0.7).transpose(0, 1)
        assert np.allclose(out[starts[b]:starts[b + 1]], want.numpy(), atol=1e-12)
    capped = plain.attention(q, kc, vc, table, lengths, starts, 3, None, 0.7, 1e9, "f32")
    assert np.allclose(capped[0], out, atol=1e-7) and np.allclose(capped[2], lse, atol=1e-7)


def test_bounds_see_a_step():
    """One weight's rounding too many, a position too many or too few, a sine's sign: all outside."""
    rng = np.random.default_rng(4)
    q, kc, vc = rng.standard_normal((1, 1, 16)), rng.standard_normal((4, 16, 1, 16)), rng.standard_normal((4, 16, 1, 16))
    args = (q, kc, vc, np.array([[0, 1, 2, 3]]))
    want, bound, lse, lb, _ = plain.attention(*args, np.array([40]), np.array([0, 1]), 1, None, 0.25, 0.0, "bf16")
    for n in (39, 41):
        off, _, off_lse, _, _ = plain.attention(*args, np.array([n]), np.array([0, 1]), 1, None, 0.25, 0.0, "bf16")
        with pytest.raises(AssertionError):
            plain.check(off, want, bound, "a position")
        with pytest.raises(AssertionError):
            plain.check(off_lse, lse, lb, "lse")
    x, positions, f = rng.standard_normal((2, 3, 8)), np.array([3, 4]), np.array([1.0, 0.5])
    y, bound = plain.rope(x, positions, f, None, 0, "half", 1.0, "bf16")
    for off in (plain.rope(x, -positions, f, None, 0, "half", 1.0, "bf16")[0], plain.rope(x, positions, f, None, 0, "interleaved", 1.0, "bf16")[0]):
        with pytest.raises(AssertionError):
            plain.check(off, y, bound, "turn")


def test_frequencies_stretch_by_their_turns(lib):
    import math

    import paper_1904_05347_amd as pk
    base = pk.rope_frequencies(64, device="cpu").numpy()
    f = pk.rope_frequencies(64, factor=8.0, original=4096, low=1.0, high=4.0, device="cpu").numpy()
    turns = base * 4096 / (2 * math.pi)
    assert np.array_equal(f[turns >= 4], base[turns >= 4]) and np.allclose(f[turns <= 1], base[turns <= 1] / 8, rtol=1e-15)
    middle = (turns > 1) & (turns < 4)
    assert middle.any() and (f[middle] < base[middle]).all() and (f[middle] > base[middle] / 8).all()
    for bad in (dict(pairs=-1), dict(pairs=4, base=0), dict(pairs=4, factor=0), dict(pairs=4, low=2, high=2)):
        with pytest.raises(ValueError):
            pk.rope_frequencies(device="cpu", **bad)
