"""The native marshalling's source: what runs without the interpreter lock.  A
tensor's method may throw there, and the exception would be turned into a Python
error by a thread that does not hold the lock: the process ends."""
import os
import re

from paper_1904_05347_amd import build


def test_only_the_library_is_called_without_the_interpreter_lock():
    with open(os.path.join(build.CSRC, "pk_torch.cpp")) as fh:
        text = fh.read()
    parts = re.findall(r"Py_BEGIN_ALLOW_THREADS\n(.*?)Py_END_ALLOW_THREADS", text, re.S)
    assert len(parts) == text.count("Py_BEGIN_ALLOW_THREADS\n") >= 8
    for part in parts:
        # calls of the bound entry points, and arguments that are plain values: no call inside one
        for statement in filter(None, (s.strip() for s in part.split(";"))):
            call = re.fullmatch(r"st = (f_\w+)\((.*)\)", statement, re.S)
            assert call, statement
            assert "(" not in re.sub(r"\((const )?\w+ \*\)", "", call.group(2)), statement
