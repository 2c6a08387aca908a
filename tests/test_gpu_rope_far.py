"""rope_qk, its gradients and cache_append at far positions, against angles that are reduced exactly:
position and frequency are whole numbers over powers of two, 1 / (2 pi) is taken to 400 bits."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu
from tests.test_gpu_heads import KINDS, _f64, _inputs, _normal, _type

BITS = 400


def _arctan_of_inverse(n, one):
    total, term, k = 0, one // n, 1
    while term:
        total += term // k if k % 4 == 1 else -(term // k)
        term //= n * n
        k += 2
    return total


def _inverse_of_two_pi():
    """2^BITS / (2 pi), pi = 16 arctan(1/5) - 4 arctan(1/239)."""
    one = 1 << BITS + 64
    pi = 16 * _arctan_of_inverse(5, one) - 4 * _arctan_of_inverse(239, one)
    return (one << BITS) // (2 * pi)


INVERSE = _inverse_of_two_pi()


def _angle(position, frequency):
    """position * frequency, less whole turns, in radians from -pi to pi."""
    n, den = float(frequency).as_integer_ratio()
    shift = BITS + den.bit_length() - 1
    part = int(position) * n * INVERSE % (1 << shift)
    if part >> shift - 1:
        part -= 1 << shift
    keep = max(0, shift - 80)
    return (part >> keep) / 2.0 ** (shift - keep) * (2 * np.pi)


def test_angles_by_hand():
    assert abs(_angle(7, 1.0) - (7 - 2 * np.pi)) < 2e-15 and abs(_angle(-1, 0.5) + 0.5) < 1e-15
    # 355 = 113 pi + 3.0144353359e-5
    assert abs(_angle(355, 1.0) - (3.0144353359e-5 - np.pi)) < 1e-14


def _turned(x, positions, f, layout, amplitude, back=False):
    out, size = x.copy(), np.abs(x)
    a, b = plain.pairs_of(x.shape[2], len(f), layout)
    t = np.array([[_angle(p, w) for w in f] for p in positions])
    cos, sin = np.cos(t)[:, None], np.sin(t)[:, None] * (-1 if back else 1)
    out[..., a] = amplitude * (x[..., a] * cos - x[..., b] * sin)
    out[..., b] = amplitude * (x[..., b] * cos + x[..., a] * sin)
    size[..., a] = size[..., b] = abs(amplitude) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return out, size


def _far(torch):
    near = [(1 << e) + o for e in (20, 28, 31, 33, 36, 39) for o in (-3, 0, 7)]
    return torch.tensor(near + [-p for p in near] + [1 << 40, -(1 << 40), (1 << 40) - 1, 987654321987], device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(layout, kind):
    """Nothing is added to the bounds of near positions: 32 U of a pair's magnitudes, 12 U for the gradient."""
    torch, pk = require_gpu()
    positions = _far(torch)
    M = len(positions)
    g, q, k, v = _inputs(torch, 3, M, 2, 1, 64, kind)
    f = pk.rope_frequencies(24)
    f[1], f[2] = 6.25, 1e-9   # frequencies of a program's own
    at, w = positions.tolist(), _f64(f)
    oq, ok = pk.rope_qk(q, k, positions, f, layout=layout, amplitude=1.25)
    gq, gk, _, _ = pk.rope_qk_backward(q, k, None, None, positions, f, layout=layout, amplitude=1.25)
    for x, y, back, u in ((q, oq, False, 32), (k, ok, False, 32), (q, gq, True, 12), (k, gk, True, 12)):
        want, size = _turned(_f64(x), at, w, layout, 1.25, back)
        bound = u * plain.U * size + plain.HALF[kind] * np.abs(want) * (1 + 2.0 ** -8) + plain.TINY[kind]
        plain.check(_f64(y), want, bound, "back" if back else "forward")
    kc, vc = (torch.zeros((M, 1, 1, 64), dtype=_type(torch, kind), device="cuda") for _ in range(2))
    out = pk.cache_append(k, v, kc, vc, torch.arange(M, device="cuda"), positions, f, q=q, layout=layout, amplitude=1.25)
    assert torch.equal(out, oq) and torch.equal(kc.view(M, 1, 64), ok)


@pytest.mark.gpu
def test_neighbouring_positions_keep_their_angle():
    """Products of a query and a key depend on how far apart they are, wherever they are."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k = _normal(torch, g, (1, 1, 64), "f32"), _normal(torch, g, (1, 1, 64), "f32")
    f = pk.rope_frequencies(32)
    near = None
    for base in (0, 1 << 20, 1 << 30, (1 << 40) - 100):
        positions = torch.tensor([base, base + 5], device="cuda")
        a = pk.rope_qk(q.expand(2, 1, 64).contiguous(), k.expand(2, 1, 64).contiguous(), positions, f)
        dot = float((a[0][1].double() * a[1][0].double()).sum())
        near = dot if near is None else near
        # each of a pair's channels is off by 32 U of its pair's magnitudes, in q and in k, here and near
        q_size, k_size = (t[0, 0, :32].abs().double() + t[0, 0, 32:].abs().double() for t in (q, k))
        assert abs(dot - near) < 2 * 4 * 32 * plain.U * float((q_size * k_size).sum())
