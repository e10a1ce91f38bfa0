"""The host side of the operators around the layer (argument checks, workspace arithmetic, error strings) under AddressSanitizer and
UndefinedBehaviorSanitizer: their boundary tests in a child process whose first library is the sanitizer runtime.  Host code
only, no GPU."""
import os

import pytest

from test_sanitizers_cpu import _run


def test_block_host_code_under_asan_and_ubsan():
    from paper_2604_23108_amd import build
    rt = build.asan_runtime()
    if not rt:
        pytest.skip("the compiler's shared AddressSanitizer runtime is not installed")
    build.build_sanitized()
    preload = rt + (":" + os.environ["LD_PRELOAD"] if os.environ.get("LD_PRELOAD") else "")
    code = ("import sys, pytest\n"
            "from paper_2604_23108_amd import binding, build\n"
            "binding._LIB_PATH = build.SAN_LIB\n"
            "sys.exit(pytest.main(['-x', '-q', '-p', 'no:cacheprovider', 'tests/test_block_cpu.py']))\n")
    assert " passed" in _run({"LD_PRELOAD": preload}, code)
