"""The argument checks of the attention operators at the ends of their integers and numbers, under
AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU."""
import pytest

from tests.test_sanitize import _run_child, _sanitized_library


@pytest.mark.parametrize("file", ["test_rotation_pairs_cpu", "test_attention_factors_cpu", "test_attention_strides_cpu"])
def test_ends_under_asan_ubsan(file):
    lib, rt = _sanitized_library()
    code = "import sys, pytest\nsys.exit(pytest.main(['-x', '-q', '-p', 'no:cacheprovider', 'tests/%s.py']))\n" % file
    proc = _run_child(code, rt, {"PK_LIBRARY": lib})
    out = proc.stdout + proc.stderr
    assert proc.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert " passed" in proc.stdout
