"""Products of 8-bit rows that start at odd addresses: laid out in a workspace at
memory lines first, they give the result of the rows where they are, bit for bit."""
import pytest

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _int8(torch, seed, rows, cols, ld, offset=0):
    """rows x cols at `offset` of a row of `ld` (< ld), full range; what lies beside it is not zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randint(-127, 128, (rows, ld), generator=g, device="cuda", dtype=torch.int8)
    return wide[:, offset:offset + cols]


def _need(pk, a, b):
    from paper_1904_05347_amd import binding
    return binding.load().pk_gemm_i8_workspace_bytes_for(a.size(0), b.size(0), a.size(1), a.data_ptr(), a.stride(0),
                                                         b.data_ptr(), b.stride(0))


def _both(torch, pk, a, b, dtype=None):
    """The default call, checked against the one without a workspace; whether it laid rows out."""
    g = torch.Generator(device="cuda").manual_seed(9)
    sa = torch.rand(a.size(0), generator=g, device="cuda")
    sb, bias = torch.rand(b.size(0), generator=g, device="cuda"), torch.rand(b.size(0), generator=g, device="cuda")
    c = pk.gemm_i8(a, b, sa, sb, bias=bias, dtype=dtype or torch.float32)
    name = pk.last_config_name()
    d = pk.gemm_i8(a, b, sa, sb, bias=bias, dtype=dtype or torch.float32, workspace=torch.empty(0, device="cuda"))
    assert torch.equal(c, d)
    assert name == pk.last_config_name() if _need(pk, a, b) == 0 else not name.endswith("_any")
    return c, sa, sb, bias


@pytest.mark.parametrize("K", list(range(2033, 2066)) + [128, 129, 143, 1023, 4097])
def test_every_end_of_a_row(K):
    """Against the product in 64 bits: sums of up to 2^26 in fp32 with scales of one and no bias are within its rounding."""
    torch, pk = require_gpu()
    M, N = (1500, 2900) if K > 1000 else (5000, 9000)
    a, b = _int8(torch, 1, M, K, K | 1), _int8(torch, 2, N, K, (K | 1) + 2, 1)
    one = torch.ones(N, device="cuda")
    c = pk.gemm_i8(a, b, one[:M], one, dtype=torch.float32)
    assert not pk.last_config_name().endswith("_any") and _need(pk, a, b) == (M + N) * ((K + 127) // 128 * 128)
    assert torch.equal(c, (a.double() @ b.double().t().contiguous()).float())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("M,N,K", [(4096, 4096, 4096), (600, 2100, 9001), (3000, 100, 12000), (33, 5000, 7001), (1, 300, 500), (70, 70, 16383)])
def test_one_operand_or_both(M, N, K, dtype):
    torch, pk = require_gpu()
    line, odd = (K + 127) // 128 * 128, K + 4 - K % 2 - 1
    for lda, ldb in ((odd, odd), (odd, line), (line, odd)):
        a, b = _int8(torch, 3, M, K, lda), _int8(torch, 4, N, K, ldb)
        _both(torch, pk, a, b, getattr(torch, dtype))
    # rows a multiple of four apart that start at an odd address
    _both(torch, pk, _int8(torch, 5, M, K, line + 128, 3), _int8(torch, 6, N, K, line + 128, 66), getattr(torch, dtype))


def test_more_than_one_launch():
    torch, pk = require_gpu()
    a, b = _int8(torch, 7, 140001, 1153, 1153), _int8(torch, 8, 500, 1153, 1155)
    assert _need(pk, a, b) == (140001 + 500) * 1280
    _both(torch, pk, a, b)
    _both(torch, pk, b, a)


def test_workspaces():
    """Given ones: whole, one too small, misaligned, overlapping; nothing past its end is written."""
    torch, pk = require_gpu()
    a, b = _int8(torch, 1, 1000, 2001, 2001), _int8(torch, 2, 1100, 2001, 2003)
    need = _need(pk, a, b)
    assert need == 2100 * 2048
    one = torch.ones(1100, device="cuda")
    want = (a.double() @ b.double().t().contiguous()).float()
    room = torch.full((need // 4 + 64,), 7.0, device="cuda")
    for ws, laid in ((room[16:16 + need // 4], True), (room[16:16 + need // 4 - 1], False), (room[17:17 + need // 4], False), (room, True)):
        room.fill_(7.0)
        c = pk.gemm_i8(a, b, one[:1000], one, dtype=torch.float32, workspace=ws)
        assert torch.equal(c, want)
        assert pk.last_config_name().endswith("_any") != laid
        first = (ws.data_ptr() - room.data_ptr()) // 4
        assert (room[:first] == 7).all() and (room[first + need // 4:] == 7).all()
        assert laid or (room == 7).all()
    out = torch.empty((1000, 1100), device="cuda")
    assert out.numel() * 4 >= need
    with pytest.raises(pk.PkError):
        pk.gemm_i8(a, b, one[:1000], one, out=out, workspace=out.view(-1))
    with pytest.raises(TypeError):
        pk.gemm_i8(a, b, one[:1000], one, workspace=room.cpu())
    with pytest.raises(TypeError):
        pk.gemm_i8(a, b, one[:1000], one, workspace=room.half())
    with pytest.raises(ValueError):
        pk.gemm_i8(a, b, one[:1000], one, workspace=one[:1].expand(need // 4))


def test_in_a_graph_and_on_another_stream(monkeypatch):
    torch, pk = require_gpu()
    from paper_1904_05347_amd import binding
    a, b = _int8(torch, 1, 1000, 2001, 2001), _int8(torch, 2, 1100, 2001, 2003)
    one = torch.ones(1100, device="cuda")
    call = lambda: pk.gemm_i8(a, b, one[:1000], one, dtype=torch.float32)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = call()
    stream.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in range(3):
        a.copy_(_int8(torch, 20 + seed, 1000, 2001, 2001))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())
    want = call()
    monkeypatch.setattr(binding, "_native", binding._PythonOnly())
    assert torch.equal(call(), want)
