"""The packed attention's and the 8-bit cache's host code (argument validation,
workspace plans, dispatch) under AddressSanitizer and
UndefinedBehaviorSanitizer, as test_sanitize.py has the others."""
import sys

from test_sanitize import _child, _clang_asan, _newer_than_sources


def test_packed_and_q8_host_code_under_asan_ubsan():
    from paper_2402_07901_amd import build
    if not _newer_than_sources(build.LIB_ASAN, build.CSRC):
        build.build(sanitize=True)
    r = _child([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                "tests/test_packed_host.py", "tests/test_q8_host.py"],
               {"LD_PRELOAD": _clang_asan(), "FASTMAX_LIB": build.LIB_ASAN})
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "Sanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert " passed" in out
