"""Scales and caps whose factors 32 bits do not hold are refused by attention_tree: scores are made with
scale * log2(e), or with scale / cap and cap * log2(e).  No call here reaches the GPU."""
import ctypes

import numpy as np
import pytest

from tests.test_attention_cpu import AT, _cache, _heads, lib  # noqa: F401 (a fixture)

F = np.float32
LARGE, LEAST = float(np.finfo(F).max), float(np.finfo(F).tiny)
LOG2E = 1.4426950408889634


def _call(lib, scale, cap, M=0):
    q, cache, out = _heads(1, 4, 32, 8), _cache(), _heads(8, 4, 32, 8)
    return lib.pk_attention_tree(0, M, 8, ctypes.byref(q), ctypes.byref(cache), 4 * AT, 2, 3, 3, 5 * AT, 6 * AT, 3, None, scale, cap,
                                 ctypes.byref(out), None, 0, None, 0, None)


@pytest.mark.parametrize("scale,cap", [(1.0, 2.5e38), (1.0, 3e38), (0.1, 1e37), (0.1, 9e36), (1e-10, 1e30), (1e-38, 1.0001), (1.0, 1e-39),
                                       (100.0, 1e-37), (0.0, 2.4e38), (-1.0, 1e38), (-1.0, 1e-42)])
def test_caps_without_a_factor(lib, scale, cap):  # noqa: F811
    assert _call(lib, scale, cap) == 1 and lib.pk_last_invalid_param() == 15
    assert _call(lib, scale, cap, 3) == 1 and lib.pk_last_invalid_param() == 15


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, LARGE])
def test_scales_without_a_factor(lib, scale):  # noqa: F811
    assert _call(lib, scale, 0.0) == 1 and lib.pk_last_invalid_param() == 14


@pytest.mark.parametrize("scale,cap", [(1.0, 0.0), (0.0, 0.0), (0.0, 1e-42), (0.0, 2.3e38), (1.0, 8e37), (0.1, 8e36), (1e-38, 0.5), (1.0, 3e-39),
                                       (-0.25, 50.0), (2.3e38, 0.0), (1e-44, 0.0), (1e38, 1.0), (1e38, 2.3e38)])
def test_those_that_have_one(lib, scale, cap):  # noqa: F811
    scale32, cap32 = float(F(scale)), float(F(cap))
    if cap:
        assert cap32 * LOG2E <= LARGE and (scale == 0 or LEAST <= abs(scale32) / cap32 <= LARGE)
    assert _call(lib, scale, cap) == 0
