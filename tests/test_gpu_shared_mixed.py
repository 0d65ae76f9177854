"""GPU tests of decode attention over shared pages where families of unequal sizes
fill the card, in the workspace that the library asks for, and against a twin of the
cache that shares nothing.  Bounds: those of test_gpu_shared."""
import pytest
import torch

from paper_2609_02029_amd import hwkv
from test_gpu_shared import DEV, Forked, _gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,G,D,fmt,families,prompt", [
    (8, 4, 64, "bf16", [9] + [2] * 43, 300), (32, 4, 128, "bf16", [9] + [2] * 9, 300), (16, 2, 64, "f16", [17] + [2] * 15, 300),
    (8, 4, 256, "bf16", [9] + [2] * 31, 800), (8, 4, 64, "i8", [9] + [2] * 43, 300), (8, 8, 64, "fp8", [5] + [2] * 40, 300)])
def test_a_wide_family_beside_pairs(H, G, D, fmt, families, prompt):
    """More items than run at once, blocks of several column groups among them."""
    r = Forked(D, G, [(prompt, n) for n in families], [20] * sum(families), levels=(1,) * H, fmt=fmt)
    r.check(seqs=(0, families[0] - 1, families[0], r.B - 1), heads=(0, H - 1))


@pytest.mark.parametrize("fmt", ["bf16", "f16", "fp8", "i8"])
def test_shared_or_not(fmt):
    """The same rows in pages that are shared and in pages of each sequence's own."""
    D, H, G, B, scale = 128, 2, 4, 6, 128 ** -0.5
    pol = hwkv.policy_set(1, H, H * G, D, 4, [70, 0], [[0, 1]])
    g = torch.Generator(device=DEV).manual_seed(9)
    rows = lambda n, h=H: torch.randn((n, h, D), generator=g, device=DEV).to(torch.bfloat16)   # noqa: E731
    kw = dict(k_scale=0.03, v_scale=0.02) if fmt == "fp8" else {}
    forked, twin = (hwkv.cache_alloc(pol, B, 4000, kv_format=fmt, n_pages=16 * B, **kw) for _ in range(2))
    k, v = rows(3000), rows(3000)
    hwkv.prefill_write(forked, 0, 0, 0, k, v)
    hwkv.cache_reorder(forked, [0] * B)
    for b in range(B):
        hwkv.prefill_write(twin, 0, b, 0, k, v)
        tail = rows(1 + 111 * b), rows(1 + 111 * b)
        for c in (forked, twin):
            hwkv.prefill_write(c, 0, b, 3000, *tail)
    assert hwkv.cache_pages(forked)[1] > hwkv.cache_pages(twin)[1]
    q, outs = rows(B, H * G), []
    for c in (forked, twin):
        ws = torch.full((hwkv.decode_shared_workspace_bytes(c),), 0xff, dtype=torch.uint8, device=DEV)
        outs.append(torch.full(q.shape, float("nan"), device=DEV))
        hwkv.decode_attn_shared(c, 0, q, scale, outs[-1], ws)
    # (each within 2e-5 of the largest value that it sees)
    assert (outs[0] - outs[1]).abs().max() <= 4e-5 * v.float().abs().max()
