"""GPU tests of decode attention over shared pages where families of unequal sizes
fill the card, in the workspace that the library asks for.  Bounds: those of
test_gpu_shared."""
import pytest

from test_gpu_shared import Forked, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,G,D,fmt,families,prompt", [
    (8, 4, 64, "bf16", [9] + [2] * 43, 300), (32, 4, 128, "bf16", [9] + [2] * 9, 300), (16, 2, 64, "f16", [17] + [2] * 15, 300),
    (8, 4, 256, "bf16", [9] + [2] * 31, 800), (8, 4, 64, "i8", [9] + [2] * 43, 300), (8, 8, 64, "fp8", [5] + [2] * 40, 300)])
def test_a_wide_family_beside_pairs(H, G, D, fmt, families, prompt):
    """More items than run at once, blocks of several column groups among them."""
    r = Forked(D, G, [(prompt, n) for n in families], [20] * sum(families), levels=(1,) * H, fmt=fmt)
    r.check(seqs=(0, families[0] - 1, families[0], r.B - 1), heads=(0, H - 1))
