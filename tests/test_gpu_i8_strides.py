"""Products of rows that lie far apart at multiples of four bytes: the offsets of a
tile's copies up to the largest leading dimension they take, and the form beyond it."""
import pytest

from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

MOST = 1 << 22   # bytes from row to row of the copies' largest leading dimension


def _int8(torch, seed, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-128, 128, (rows, cols), generator=g, device="cuda", dtype=torch.int8)


def _far(torch, values, ld, offset):
    """`values` as a slice of an array of rows of ld, which holds other numbers beside it."""
    rows, cols = values.shape
    wide = torch.empty((rows, ld), dtype=torch.int8, device="cuda")
    wide[:, :offset] = 99
    wide[:, offset + cols:offset + cols + 256] = 99
    far = wide[:, offset:offset + cols]
    far.copy_(values)
    return far


def _exact(a, b):
    return (a.double() @ b.double().t().contiguous()).float()


@pytest.mark.parametrize("K", [200, 203, 1024])
def test_the_largest_leading_dimension(K):
    """Tiles of every size, as A, as B and as both; sums of up to 2^24 are exact in fp32."""
    torch, pk = require_gpu()
    rows = 1100
    one = torch.ones(30000, device="cuda")
    values = _int8(torch, 1, rows, K)
    far = _far(torch, values, MOST, 4)
    assert far.stride(0) == MOST and far.data_ptr() % 4 == 0
    names = set()
    for n in (7, 37, 300, 1100, 3001, 16384, 30000):
        near = _int8(torch, n, n, (K + 3) // 4 * 4)[:, :K]
        want = _exact(values, near)
        for got, expect in ((pk.gemm_i8(far, near, one[:rows], one[:n], dtype=torch.float32), want),
                            (pk.gemm_i8(near, far, one[:n], one[:rows], dtype=torch.float32), want.t())):
            names.add(pk.last_config_name())
            assert torch.equal(got, expect), (n, pk.last_config_name())
    assert {"gemm_i8_256x256", "gemm_i8_64x128"} <= names and not any(n.endswith("_any") for n in names), names
    got = pk.gemm_i8(far, far, one[:rows], one[:rows], dtype=torch.float32)
    assert torch.equal(got, _exact(values, values))


@pytest.mark.parametrize("ld,offset", [(MOST + 4, 4), (MOST + 128, 0), (MOST + 1, 3)])
def test_beyond_it(ld, offset):
    """Any product then runs as one of few rows."""
    torch, pk = require_gpu()
    one = torch.ones(3000, device="cuda")
    values = _int8(torch, 1, 150, 777)
    far = _far(torch, values, ld, offset)
    for n in (1, 40, 3000):
        near = _int8(torch, n, n, 780)[:, :777]
        none = torch.empty(0, device="cuda")   # no workspace: rows stay where they are
        for got, expect in ((pk.gemm_i8(far, near, one[:150], one[:n], dtype=torch.float32, workspace=none), _exact(values, near)),
                            (pk.gemm_i8(near, far, one[:n], one[:150], dtype=torch.float32, workspace=none), _exact(near, values))):
            assert pk.last_config_name() == "gemm_i8_rows"
            assert torch.equal(got, expect), n
