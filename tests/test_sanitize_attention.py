"""The host side of the attention operators (argument checks, where tensors lie, how work is
divided) under AddressSanitizer and UndefinedBehaviorSanitizer: the CPU tests of it on
the library whose host code is instrumented."""
from tests.test_sanitize import _run_child, _sanitized_library


def test_attention_host_logic_under_asan_ubsan():
    lib, rt = _sanitized_library()
    code = ("import sys, pytest\n"
            "sys.exit(pytest.main(['-x', '-q', '-p', 'no:cacheprovider', 'tests/test_attention_cpu.py', '-k', 'arguments or workspace']))\n")
    proc = _run_child(code, rt, {"PK_LIBRARY": lib})
    out = proc.stdout + proc.stderr
    assert proc.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert " passed" in proc.stdout
