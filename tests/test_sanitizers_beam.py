"""The host tests of beam selection, reordering, moving and shared decode under
AddressSanitizer and UndefinedBehaviorSanitizer, as ``test_sanitizers_rope_i8`` runs its
own."""
import os

from test_sanitizers import ROOT, _run
from test_sanitizers_rope_i8 import env  # noqa: F401


def test_beam_host_tests_under_sanitizers(env):  # noqa: F811
    rc, out = _run(env, ["-m", "pytest", "-q", "-x", "-m", "not gpu", "-p", "no:cacheprovider",
                         os.path.join(ROOT, "tests", "test_host_beam.py")])
    assert "Sanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert rc == 0, out[-6000:]
    assert " passed" in out and "failed" not in out, out[-2000:]
