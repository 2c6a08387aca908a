"""attention_tree with scales and caps at the ends of what it takes, against the definition in 64 bits."""
import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_attention import Call
from tests.test_gpu_heads import KINDS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,d", [(2, 64), (40, 128)])
@pytest.mark.parametrize("scale,cap", [(0.0, 1e-42), (0.0, 2.3e38), (0.0, 30.0), (0.125, 8e36), (1e-30, 1e-3), (-0.25, 1e-36), (0.25, 1e20),
                                       (1e-44, 0.0)])
def test_factors_at_the_ends(scale, cap, T, d, kind):
    torch, pk = require_gpu()
    Call(torch, 40 + d, [300, 5], [T, 1], 1, 2, d, kind).check(pk, cap=cap, scale=scale, what="scale %g cap %g" % (scale, cap))
