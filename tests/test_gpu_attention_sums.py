"""How near fp32's attention comes to 64 bits as a whole: the length of the difference, where every single
bound is one of the worst case."""
import numpy as np
import pytest

from tests import attention_plain as plain
from tests.gpu_util import require_gpu
from tests.test_gpu_attention import Call
from tests.test_gpu_heads import _f64

pytestmark = pytest.mark.gpu

U = plain.U


@pytest.mark.parametrize("T,d", [(2, 192), (2, 256), (2, 250), (20, 200), (20, 256), (16, 255)])
def test_scores_of_many_channels(T, d):
    """Roundings are independent, of U / sqrt(3) at the most on average.  For q of 1.5 and k of 1 on average a sum of n
    channels is 1.5 sqrt(n).  A block of 32 channels is summed in 8 steps of 4 (4 roundings each, at worst): the squares of
    its errors are 4 sum_j (U^2 / 3) 2.25 (4 j) = 432 U^2, of 8 blocks 3456 U^2, of their 8 additions sum_j (U^2 / 3)
    2.25 (32 j) = 864 U^2: 66 U, times 256^-1/2 4.1 U of a score, which a weight's relative error is.  The exponential
    adds 2 U, the factor of the scores (three roundings, for scores of 1.5 to 4) 3 U to 5 U, quotient and result 1 U: 7 U.
    Twice that holds for inputs of any luck; in one sum over all channels the first part alone were 4 * 8^1/2 U = 12 U and
    more."""
    torch, pk = require_gpu()
    call = Call(torch, d + T, [500, 300, 700], [T] * 3, 2, 2, d, "f32")
    out, lse = call(pk, lse=True)
    want, _, wl, _, _ = plain.attention(_f64(call.q), np.nan_to_num(_f64(call.kc)), np.nan_to_num(_f64(call.vc)), call.table.cpu().numpy(),
                                        call.len.cpu().numpy(), call.starts.cpu().numpy(), call.most, call.mask.cpu().numpy(), d ** -0.5,
                                        0.0, "f32")
    off = np.linalg.norm(_f64(out) - want) / np.linalg.norm(want)
    assert off < 14 * U, "%.1f U" % (off / U)
    # a row's sum of exponentials has its scores' errors, and the logarithm's own rounding
    assert np.sqrt(((_f64(lse) - wl) ** 2).mean()) < 14 * U + U * np.abs(wl).max()
