"""The attention operators' two marshallings: the same bits from the same C-ABI call, the same
refusals, and the tensors that neither takes."""
import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_native_call import _both, _Declines

pytestmark = pytest.mark.gpu


class _Calls:
    def __init__(self, torch, pk, kind=None):
        g = torch.Generator(device="cuda").manual_seed(3)
        f = lambda *s: torch.randn(s, generator=g, device="cuda").to(kind or torch.bfloat16)  # noqa: E731
        self.q, self.k, self.v = f(5, 4, 64), f(5, 2, 64), f(5, 2, 64)
        self.dq, self.dk, self.w, self.w32 = f(5, 4, 64), f(5, 2, 64), f(64), torch.ones(64, device="cuda")
        self.f, self.positions = pk.rope_frequencies(32), torch.arange(5, device="cuda")
        self.kc, self.vc = f(9, 16, 2, 64), f(9, 16, 2, 64)
        self.slots = torch.tensor([3, 20, 40, 61, 99], device="cuda")
        self.table = torch.arange(9, dtype=torch.int32, device="cuda").view(1, 9)
        self.len, self.starts = torch.tensor([130], dtype=torch.int32, device="cuda"), torch.tensor([0, 5], dtype=torch.int32, device="cuda")
        self.mask = torch.tensor([1, 3, 5, 9, 17], device="cuda")
        self.lse, self.ws = torch.zeros(5, 4, device="cuda"), torch.zeros(1 << 20, device="cuda")
        self.pk, self.torch = pk, torch

    def plain(self):
        pk, s, empty = self.pk, self, self.torch.empty_like

        def appended(**more):
            kc, vc = s.kc.clone(), s.vc.clone()
            q = pk.cache_append(s.k, s.v, kc, vc, s.slots, **more)
            return (kc, vc) if q is None else (q, kc, vc)

        attend = lambda *a, **m: pk.attention_tree(s.q, s.kc, s.vc, s.table, s.len, s.starts, 5, *a, **m)  # noqa: E731
        return [
            lambda: pk.rope_qk(s.q, s.k, s.positions, s.f, s.w, s.w, eps=1e-5),
            lambda: pk.rope_qk(s.q, s.k, s.positions, s.f, None, s.w32, layout="interleaved", amplitude=0.5, q_out=empty(s.q)),
            lambda: pk.rope_qk(s.q, None, None, None, s.w),
            lambda: pk.rope_qk_backward(s.dq, s.dk, s.q, s.k, s.positions, s.f, s.w, s.w),
            lambda: pk.rope_qk_backward(s.dq, s.dk, None, s.k, s.positions, s.f, None, s.w32, k_grad=empty(s.dk)),
            lambda: pk.rope_qk_backward(s.dq, None, None, None, s.positions, s.f, amplitude=2, layout="interleaved"),
            lambda: appended(positions=s.positions, frequencies=s.f, k_weight=s.w, q=s.q, q_weight=s.w),
            lambda: appended(),
            lambda: appended(positions=s.positions, frequencies=s.f, layout="interleaved", amplitude=0.25, q=s.q, q_out=empty(s.q)),
            lambda: attend(),
            lambda: attend(mask=s.mask, scale=0.2, cap=5, lse=True),
            lambda: attend(mask=s.mask, lse=self.torch.zeros_like(s.lse), workspace=s.ws, out=empty(s.q)),
            lambda: attend(scale=1, workspace=s.ws[:0], lse=False),
        ]


def _same(torch, a, b):
    if isinstance(a, torch.Tensor):
        return a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b)
    return a is b is None or len(a) == len(b) and all(_same(torch, x, y) for x, y in zip(a, b))


def test_native_calls_equal_python_calls(monkeypatch):
    torch, pk = require_gpu()
    for kind in (torch.bfloat16, torch.float16, torch.float32):
        for i, call in enumerate(_Calls(torch, pk, kind).plain()):
            first, second = _both(pk, monkeypatch, call)
            assert type(first) is type(second) and _same(torch, first, second), i


@pytest.mark.parametrize("native", [True, False])
def test_refusals(monkeypatch, native):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    monkeypatch.setattr(binding, "_native", (binding._native or binding._load_native()) if native else _Declines())
    s = _Calls(torch, pk)
    attend = lambda q=s.q, kc=s.kc, vc=s.vc, table=s.table, n=s.len, starts=s.starts, most=5, **m: pk.attention_tree(  # noqa: E731
        q, kc, vc, table, n, starts, most, **m)
    append = lambda k=s.k, v=s.v, kc=s.kc, vc=s.vc, slots=s.slots, **m: pk.cache_append(k, v, kc, vc, slots, **m)  # noqa: E731
    rope = lambda q=s.q, k=s.k, positions=s.positions, f=s.f, **m: pk.rope_qk(q, k, positions, f, **m)  # noqa: E731
    back = lambda dq=s.dq, dk=s.dk, q=s.q, k=s.k, positions=s.positions, f=s.f, **m: pk.rope_qk_backward(dq, dk, q, k, positions, f, **m)  # noqa: E731
    wide = torch.ones(1, 4, 257, device="cuda")
    before = [t.clone() for t in (s.q, s.k, s.kc, s.vc)]
    for error, calls in {
        TypeError: [
            lambda: rope(q=s.q.double()), lambda: rope(q=s.q.cpu()), lambda: rope(k=s.k.float()), lambda: rope(positions=s.positions.int()),
            lambda: rope(f=s.f.float()), lambda: rope(q_weight=s.w.half()), lambda: rope(q_weight=s.w, k_weight=s.w32),
            lambda: back(dk=s.dk.float()), lambda: back(q=s.q.float(), q_weight=s.w),
            lambda: append(v=s.v.float()), lambda: append(kc=s.kc.float()), lambda: append(slots=s.slots.int()),
            lambda: attend(kc=s.kc.float()), lambda: attend(table=s.table.long()), lambda: attend(n=s.len.long()), lambda: attend(starts=s.starts.long()),
            lambda: attend(mask=s.mask.int()), lambda: attend(lse=s.lse.half()), lambda: attend(workspace=s.ws.half()), lambda: attend(q=None)],
        ValueError: [
            lambda: rope(q=s.q[0]), lambda: rope(k=s.k[:4]), lambda: rope(q=s.q[:, :, ::2]), lambda: rope(positions=s.positions[:4]),
            lambda: rope(f=pk.rope_frequencies(33)), lambda: rope(f=None), lambda: rope(positions=None), lambda: rope(layout="thirds"),
            lambda: rope(q_weight=s.w[:63]), lambda: rope(k=None, k_weight=s.w), lambda: rope(q_out=s.k), lambda: rope(k=None, k_out=s.k),
            lambda: back(q=None, q_weight=s.w), lambda: back(k=s.k[:4], k_weight=s.w), lambda: back(q_grad=s.k), lambda: back(dk=None, k_weight=s.w),
            lambda: append(v=s.v[:, :1]), lambda: append(kc=s.kc[0]), lambda: append(vc=s.vc[:8]), lambda: append(kc=s.kc[..., :63], vc=s.vc[..., :63]),
            lambda: append(slots=s.slots[:4]), lambda: append(q_weight=s.w), lambda: append(q_out=s.q), lambda: append(k=s.k[:, :1], v=s.v[:, :1]),
            lambda: attend(q=s.q[:, :3]), lambda: attend(kc=s.kc[..., :32], vc=s.vc[..., :32]), lambda: attend(table=s.table[0]),
            lambda: attend(n=s.len.repeat(2)), lambda: attend(starts=s.starts[:1]), lambda: attend(mask=s.mask[:4]), lambda: attend(out=s.k),
            lambda: attend(lse=s.lse[:, :3]), lambda: attend(workspace=torch.ones(64, 64, device="cuda")[:, ::2]),
            lambda: attend(table=s.table.expand(2, 9), n=s.len.repeat(2), starts=s.starts.repeat(2)[:3])],
        pk.PkError: [
            lambda: rope(q=wide, k=None, positions=s.positions[:1]), lambda: rope(eps=-1.0, q_weight=s.w), lambda: rope(q_out=s.q.flip(0).as_strided(s.q.shape, (0, 64, 1))),
            lambda: rope(k_out=s.q[:, :2]), lambda: rope(q_out=torch.empty(6, 4, 64, device="cuda").bfloat16()[:5].copy_(s.q), k_out=s.q[:, 2:]),
            lambda: back(q_grad=s.q, q_weight=s.w), lambda: append(kc=s.vc), lambda: append(q=s.q, q_out=s.v.repeat(1, 2, 1)[:, :4].as_strided(s.q.shape, (64, 64, 1))),
            lambda: append(k=s.kc[:5, 0]), lambda: attend(most=0), lambda: attend(most=65), lambda: attend(cap=-1.0), lambda: attend(out=s.q[:1].expand(5, 4, 64)),
            lambda: attend(workspace=s.ws[1:])]}.items():
        for n, call in enumerate(calls):
            with pytest.raises(error):
                call()
                pytest.fail("%s %d was not refused" % (error.__name__, n))
    assert all(torch.equal(a, b) for a, b in zip(before, (s.q, s.k, s.kc, s.vc)))


def _operands(torch, pk):
    """(operator, operands): every tensor that a call takes, outputs among them."""
    s = _Calls(torch, pk, torch.float32)
    e = torch.empty_like
    return [
        (lambda q, k, p, f, qw, kw, qo, ko: pk.rope_qk(q, k, p, f, qw, kw, q_out=qo, k_out=ko),
         [s.q, s.k, s.positions, s.f, s.w, s.w32, e(s.q), e(s.k)]),
        (lambda dq, dk, q, k, p, f, qw, kw, gq, gk: pk.rope_qk_backward(dq, dk, q, k, p, f, qw, kw, q_grad=gq, k_grad=gk),
         [s.dq, s.dk, s.q, s.k, s.positions, s.f, s.w, s.w32, e(s.q), e(s.k)]),
        (lambda k, v, kc, vc, slots, p, f, kw, q, qw, qo: pk.cache_append(k, v, kc, vc, slots, p, f, kw, q=q, q_weight=qw, q_out=qo),
         [s.k, s.v, s.kc, s.vc, s.slots, s.positions, s.f, s.w, s.q, s.w32, e(s.q)]),
        (lambda q, kc, vc, t, n, st, m, o, lse, ws: pk.attention_tree(q, kc, vc, t, n, st, 5, mask=m, out=o, lse=lse, workspace=ws),
         [s.q, s.kc, s.vc, s.table, s.len, s.starts, s.mask, e(s.q), s.lse, s.ws]),
    ]


@pytest.mark.parametrize("native", [True, False])
def test_wrapped_tensors(monkeypatch, native):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    monkeypatch.setattr(binding, "_native", (binding._native or binding._load_native()) if native else _Declines())
    for op, operands in _operands(torch, pk):
        op(*operands)
        for n, t in enumerate(operands):
            def one(wrapped):
                op(*operands[:n], wrapped, *operands[n + 1:])
                return wrapped

            with pytest.raises(RuntimeError, match="storage|data pointer"):
                torch.func.vmap(one)(torch.stack([t, t]))
    torch.cuda.synchronize()


@pytest.mark.parametrize("native", [True, False])
def test_negative_views(monkeypatch, native):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    monkeypatch.setattr(binding, "_native", (binding._native or binding._load_native()) if native else _Declines())

    def negative(*shape):
        t = torch.complex(torch.ones(shape, device="cuda"), torch.ones(shape, device="cuda")).conj().imag
        assert t.is_neg()
        return t

    x, neg = torch.ones(3, 2, 1, device="cuda"), negative(3, 2, 1)
    slots, kc, table = torch.arange(3, device="cuda"), torch.ones(2, 4, 2, 1, device="cuda"), torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    n, starts = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    attend = lambda q=x, k=kc, v=kc.clone(), **m: pk.attention_tree(q, k, v, table, n, starts, 3, **m)  # noqa: E731
    for call in (lambda: pk.rope_qk(neg, None, None, None), lambda: pk.rope_qk(x, neg, None, None), lambda: pk.rope_qk(x, None, None, None, negative(1)),
                 lambda: pk.rope_qk(x, None, None, None, q_out=neg), lambda: pk.rope_qk_backward(neg, None, None, None, None, None),
                 lambda: pk.cache_append(x, neg, kc, kc.clone(), slots), lambda: pk.cache_append(x, x, kc, negative(2, 4, 2, 1), slots),
                 lambda: attend(q=neg), lambda: attend(k=negative(2, 4, 2, 1)), lambda: attend(out=neg), lambda: attend(lse=negative(3, 2))):
        with pytest.raises(ValueError, match="negative view|unit column stride"):
            call()
