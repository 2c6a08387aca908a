"""The gated activation where 1 + exp(-t) leaves the 32 bits' range or its reciprocal
does: gates far below zero, whose small activation a large `up` brings back."""
import numpy as np
import pytest

from tests import i8_plain as plain
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _f64(t):
    import torch
    torch.cuda.synchronize()
    return t.detach().double().cpu().numpy()


def _want(gate, up, name):
    """gated_rows' bounds, and the rounding of an activation below the normal
    numbers: half of 2^-149."""
    a, t = plain.act(gate, name)
    with np.errstate(all="ignore"):
        small = np.where(a != 0, 2.0 ** -150 / np.abs(a), 0.0)
    return plain.rows(a * up, rel=(7 + 6 * np.minimum(np.abs(t), 200.0)) * plain.U32 + np.minimum(small, 1.0))


@pytest.mark.parametrize("act,lo,hi", [("silu", -103.0, -80.0), ("gelu", -11.2, -9.0)])
@pytest.mark.parametrize("up", [3.0, -2e10, 1e30, -3e37])
def test_a_gate_a_row(act, lo, hi, up):
    torch, pk = require_gpu()
    gate = torch.linspace(lo, hi, 693, device="cuda")[:, None]
    ups = torch.full_like(gate, up)
    q, s = pk.gated_i8(gate, ups, activation=act)
    want = _want(_f64(gate), _f64(ups), act)
    if up == 3.0:   # rows that end up beside the least scale are either way
        clear = np.abs(np.abs(plain.act(_f64(gate), act)[0][:, 0] * up) / plain.LEAST - 1) > 1e-3
        q, s, want = q[torch.from_numpy(clear).cuda()], s[torch.from_numpy(clear).cuda()], tuple(w[clear] for w in want)
    plain.check_rows(_f64(q), _f64(s), want, (act, up))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_beyond_every_number(act):
    """Activations that round to zero, and infinite gates: zero times infinity below, infinity above."""
    torch, pk = require_gpu()
    inf = float("inf")
    g = torch.tensor([-150.0, -1e3, -1e5, -1e10, -1e19, -1e25, -3.4e38], device="cuda")[:, None]
    q, s = pk.gated_i8(g, torch.full_like(g, 3e38), activation=act)
    assert (q == 0).all() and (s == 0).all()
    g = torch.tensor([90.0, 1e3, 1e10, 1e25, 3e38], device="cuda")[:, None]
    q, s = pk.gated_i8(g, torch.ones_like(g), activation=act)
    plain.check_rows(_f64(q), _f64(s), plain.rows(_f64(g)), act)
    g = torch.tensor([inf, -inf, float("nan")], device="cuda")[:, None]
    q, s = pk.gated_i8(g, torch.ones_like(g), activation=act)
    assert (q == 0).all() and s[0] == inf and torch.isnan(s[1:]).all()


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("M,N", [(3, 7), (4, 512), (3, 1030), (2, 4097), (3, 16390), (1, 70001), (1101, 1500)])
def test_among_ordinary_gates(M, N, kind):
    """A few gates far below zero in rows of ordinary ones, whose `up` makes them count."""
    torch, pk = require_gpu()
    T = getattr(torch, kind)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    big = 6e4 if kind == "float16" else 1e30
    for act, far in (("silu", -92.0), ("gelu", -10.9)):
        gate = torch.randn((M, N), generator=g, device="cuda") - 4
        up = torch.randn((M, N), generator=g, device="cuda")
        there = torch.rand((M, N), generator=g, device="cuda") < 0.01
        there[:, N // 2] = True
        gate = torch.where(there, far + gate, gate)
        # the ordinary ones at the size of the others
        up = torch.where(there, up.sign() * big, up * (1e-6 if kind == "float16" else 1e-9))
        gate, up = gate.to(T), up.to(T)
        q, s = pk.gated_i8(gate, up, activation=act)
        plain.check_rows(_f64(q), _f64(s), _want(_f64(gate), _f64(up), act), (M, N, kind, act))


@pytest.mark.parametrize("up", [1.0, -1e30])
def test_silu_holds_its_last_bits(up):
    """However far below zero the gate is, SiLU is within 12 half units: the two
    factors of the exponential have 2 and 3, 1 + q, the reciprocal and the three
    products that make the activation 1, 2 and 3, and the product with `up` has 1."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(3)
    for lo, hi in ((-87.0, -40.0), (-40.0, -10.0), (-10.0, 0.0), (0.0, 90.0)):
        gate = lo + (hi - lo) * torch.rand((4000, 1), generator=g, device="cuda")
        if up == 1.0:
            gate = gate.clamp(min=-80.0)   # above the least scale
        ups = torch.full_like(gate, up)
        q, s = pk.gated_i8(gate, ups)
        z = plain.act(_f64(gate), "silu")[0] * _f64(ups)
        plain.check_rows(_f64(q), _f64(s), plain.rows(z, rel=12 * plain.U32), (lo, hi, up))


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_large_gates_are_their_own_activation(act):
    """Where q / (1 + q) rounds to 1 no bit of the gate changes, up to the largest number."""
    torch, pk = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(5)
    size = torch.rand((3000, 1), generator=g, device="cuda") * 36 + 2   # 10^2 to 10^38
    gate = torch.cat([10.0 ** size, 20 + 80 * torch.rand((1000, 1), generator=g, device="cuda"),
                      torch.full((1, 1), torch.finfo(torch.float32).max, device="cuda")])
    gate = gate[torch.isfinite(gate)][:, None]
    q, s = pk.gated_i8(gate, torch.ones_like(gate), activation=act)
    same, scale = pk.quantize_i8(gate)
    assert torch.equal(q, same) and torch.equal(s, scale) and torch.isfinite(s).all()
