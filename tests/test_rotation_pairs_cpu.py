"""Numbers of pairs that no head has, up to the largest integers, are refused; on the CPU."""
import ctypes

import pytest

from tests.test_attention_cpu import AT, _cache, _heads, _rot, lib  # noqa: F401 (a fixture)


def _ref(*args):
    return [ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args]


@pytest.mark.parametrize("pairs", [5, 1 << 31, 1 << 32, 1 << 62, (1 << 62) + 4, (1 << 63) - 1, -1, -(1 << 62), -(1 << 63)])
def test_too_many_pairs(lib, pairs):  # noqa: F811
    q, k, v, oq, ok = _heads(1, 4, 32, 8), _heads(2, 2, 16, 8), _heads(3, 2, 16, 8), _heads(7, 4, 32, 8), _heads(8, 2, 16, 8)
    rot, cache = _rot(pairs), _cache()
    # without tokens nothing is launched, whatever is taken
    for M in (0, 3):
        assert lib.pk_rope_qk(*_ref(0, M, 8, q, k, rot, None, None, 0, 0.0, oq, ok), None) == 1
        assert lib.pk_last_invalid_param() == 6
        assert lib.pk_rope_qk_backward(*_ref(0, M, 8, q, k, None, None, rot, None, None, 0, 0.0, oq, ok), None, None, None, 0, None) == 1
        assert lib.pk_last_invalid_param() == 8
        assert lib.pk_cache_append(*_ref(0, M, 8, q, k, v, rot, None, None, 0, 0.0, oq, cache), 9 * AT, None) == 1
        assert lib.pk_last_invalid_param() == 7


def test_as_many_as_a_head_has(lib):  # noqa: F811
    q, oq = _heads(1, 4, 36, 9), _heads(7, 4, 36, 9)
    for d, pairs, status in ((9, 4, 0), (9, 5, 1), (8, 4, 0), (1, 0, 0), (1, 1, 1)):
        assert lib.pk_rope_qk(*_ref(0, 0, d, q, None, _rot(pairs), None, None, 0, 0.0, oq, None), None) == status
