"""The host tests of the rotation and of int8 caches under AddressSanitizer and
UndefinedBehaviorSanitizer, as ``test_sanitizers`` runs the host ABI's (and with
its builds, where they are newer than the sources)."""
import os

import pytest

from test_sanitizers import ROOT, SAN_DIR, _run


@pytest.fixture(scope="module")
def env():
    from paper_2609_02029_amd import build as pb
    rt = pb.sanitizer_runtime()
    if not os.path.isabs(rt) or not os.path.exists(rt):
        pytest.skip("clang's shared sanitizer runtime is not installed")
    lib = os.path.join(SAN_DIR, "libhwkv_san.so")
    files = [os.path.join(d, f) for d in (pb.CSRC, pb.INCLUDE) for f in os.listdir(d)]
    if not os.path.exists(lib) or os.path.getmtime(lib) <= max(os.path.getmtime(f) for f in files):
        lib = pb.build_host_sanitized(SAN_DIR)
    return dict(os.environ, HWKV_LIBRARY=lib, LD_PRELOAD=rt, HIP_VISIBLE_DEVICES="",
                ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1",
                UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")


def test_rope_and_i8_host_tests_under_sanitizers(env):
    rc, out = _run(env, ["-m", "pytest", "-q", "-x", "-m", "not gpu", "-p", "no:cacheprovider",
                         os.path.join(ROOT, "tests", "test_host_rope_i8.py")])
    assert "Sanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert rc == 0, out[-6000:]
    assert " passed" in out and "failed" not in out, out[-2000:]
