"""GPU tests of int8 decode where every logit of a head lies far below zero: the
softmax is that of the differences, however far down the largest is."""
import numpy as np
import pytest
import torch

from oracle import kvformat as KF
from paper_2609_02029_amd import hwkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


# by item in one launch, split with a merge, and by item with a merge
@pytest.mark.parametrize("lens,hkv", [([1, 65, 300], 2), ([5000], 2), ([6000] + [40 + i for i in range(23)], 4)])
@pytest.mark.parametrize("D,G", [(64, 8), (128, 4), (256, 1)])
@pytest.mark.parametrize("power", [100, 118])
def test_logits_far_below_zero(D, G, lens, hkv, power):
    """Keys of -2^power (and, every 50th row, the first among them, half that: the
    largest logit, and no other row has weight) under queries of one, and of minus
    one for the odd heads (the other rows then share the weight)."""
    B = len(lens)
    pol = hwkv.policy_set(1, hkv, hkv * G, D, 0, [0], [[0] * hkv])
    cache = hwkv.cache_alloc(pol, B, max(lens) + 8, kv_format="i8")
    r = np.random.default_rng(D)
    want = np.empty((B, hkv * G, D))
    q = torch.ones((B, hkv * G, D), device=DEV).to(torch.bfloat16)
    q[:, 1::2] = -1.0
    for b, n in enumerate(lens):
        half = np.arange(n) % 50 == 0
        k = torch.full((n, hkv, D), -(2.0 ** power), device=DEV)
        k[torch.from_numpy(half).to(DEV)] *= 0.5
        v = torch.from_numpy(r.normal(size=(n, hkv, D))).to(DEV).to(torch.bfloat16)
        hwkv.prefill_write(cache, 0, b, 0, k.to(torch.bfloat16), v)
        bits = v.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
        held = KF.values(KF.store(bits, "i8"), "i8")
        for h in range(hkv * G):
            seen = half if h % 2 == 0 or n == 1 else ~half
            want[b, h] = held[seen, h // G].mean(axis=0)
    ws = torch.zeros(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    out = torch.full((B, hkv * G, D), float("nan"), device=DEV)
    hwkv.decode_attn(cache, 0, q, 1.0, out, ws)
    # equal weights of one; fp32 sums of at most 6,000 terms below 5: each workgroup
    # adds at most a few hundred, and 2^-24 x 5 x (300 + 300) is 2e-4 of a sum of
    # magnitudes; its mean stays below that
    assert np.abs(out.double().cpu().numpy() - want).max() <= 2e-4
    cache.free()
