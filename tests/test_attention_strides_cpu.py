"""A cache without pages may have any strides; what they say is asked before the call is refused for
another argument.  No call here reaches the GPU."""
import ctypes

import pytest

from tests.test_attention_cpu import AT, _cache, _heads, lib  # noqa: F401 (a fixture)


@pytest.mark.parametrize("stride", [16, 1 << 30, 1 << 40])
@pytest.mark.parametrize("dtype,size", [(0, 1 << 30), (0, 1 << 22), (1, 1 << 30), (2, 8)])
def test_strides_of_no_pages(lib, dtype, size, stride):  # noqa: F811
    q, out = _heads(1, 4, 32, 8), _heads(8, 4, 32, 8)
    cache = _cache(pages=0, size=size, k=(16, stride, 8), v=(16, stride, 8))
    # lse lies over the lengths
    assert lib.pk_attention_tree(dtype, 3, 8, ctypes.byref(q), ctypes.byref(cache), 4 * AT, 2, 1, 1, 5 * AT, 6 * AT, 3, None, 1.0, 0.0,
                                 ctypes.byref(out), 5 * AT, 4, None, 0, None) == 1
    assert lib.pk_last_invalid_param() == 17
