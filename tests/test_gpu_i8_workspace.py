"""GPU tests of what int8 decode asks for as workspace: the partials that the
call writes, in the caller's workspace and in the static scratch."""
import math
import re

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


def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _filled(pol, lens, max_ctx, hkv, D, keep):
    cache = hwkv.cache_alloc(pol, len(lens), max_ctx, kv_format="i8")
    g = torch.Generator(device=DEV).manual_seed(5)
    kept = {}
    for b, n in enumerate(lens):
        k, v = (torch.randn((n, hkv, D), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        hwkv.prefill_write(cache, 0, b, 0, k, v)
        if b in keep:
            kept[b] = (_bits(k), _bits(v))
    return cache, kept


def test_noalloc_takes_a_batch_of_many_long_sequences():
    """384 items of 2,560 rows, 256 x 8: as split workgroups about 22 MB of
    partials, more than the 16 MiB scratch; the launch by item that the call runs
    leaves far fewer."""
    B, hkv, G, D, rows = 96, 4, 8, 256, 2560
    pol = hwkv.policy_set(1, hkv, hkv * G, D, 0, [0], [[0] * hkv])
    (one, kept), (two, _) = (_filled(pol, [rows] * B, rows + 64, hkv, D, (0, 95)) for _ in range(2))
    q = torch.randn((B, hkv * G, D), device=DEV).to(torch.bfloat16)
    kn, vn = (torch.randn((B, hkv, D), device=DEV).to(torch.bfloat16) for _ in range(2))
    out, want = (torch.full((B, hkv * G, D), float("nan"), device=DEV) for _ in range(2))
    scale = 1 / math.sqrt(D)
    ws = torch.full((hwkv.decode_workspace_bytes(two),), 0xff, dtype=torch.uint8, device=DEV)
    assert ws.numel() > 16 << 20
    hwkv.append_decode_attn(two, 0, kn, vn, q, scale, want, ws)
    hwkv.append_decode_attn_noalloc(one, 0, kn, vn, q, scale, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and hwkv.cache_seq_len(one, 0, 95) == rows + 1
    for b, (k, v) in kept.items():
        k, v = (np.concatenate([x, _bits(y[b:b + 1])]) for x, y in ((k, kn), (v, vn)))
        kk, vv = (KF.values(KF.store(x, "i8"), "i8") for x in (k, v))
        for h in range(hkv):
            z = q[b, h * G:(h + 1) * G].double().cpu().numpy() @ kk[:, h].T * scale
            p = np.exp(z - z.max(axis=1, keepdims=True))
            ref = p @ vv[:, h] / p.sum(axis=1, keepdims=True)
            # logits below 8 to a few 2^-24 of themselves, fp32 sums of 2,561 terms
            # in parts of a few hundred: below 2e-5 of the largest value (5)
            assert np.abs(out[b, h * G:(h + 1) * G].double().cpu().numpy() - ref).max() <= 1e-4
    one.free()
    two.free()


@pytest.mark.parametrize("lens,hkv,D,G", [
    ([9000], 4, 256, 6),                          # split, one workgroup per CU
    ([7000], 2, 64, 8),                           # split, two
    ([300, 1], 2, 128, 4),                        # by item, no partials
    ([6000] + [50 + i for i in range(23)], 4, 128, 4),      # by item, one sequence split
    ([40 + i for i in range(199)] + [3000], 2, 64, 1),      # two launches by item
])
def test_the_workspace_asked_for_is_what_is_written(lens, hkv, D, G):
    """A workspace of exactly the bytes that a refusal names gives the full one's
    result and writes nothing behind it; a smaller one is refused."""
    pol = hwkv.policy_set(1, hkv, hkv * G, D, 0, [0], [[0] * hkv])
    cache, _ = _filled(pol, lens, max(lens) + 8, hkv, D, ())
    B = len(lens)
    q = torch.randn((B, hkv * G, D), device=DEV).to(torch.bfloat16)
    want, got = (torch.full((B, hkv * G, D), float("nan"), device=DEV) for _ in range(2))
    full = torch.zeros(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    hwkv.decode_attn(cache, 0, q, 0.1, want, full)
    area = torch.full((full.numel() + 4096,), 0x77, dtype=torch.uint8, device=DEV)
    need = 0
    try:
        hwkv.decode_attn(cache, 0, q, 0.1, got, area[:1])
    except hwkv.HwkvError as e:
        assert e.code == hwkv.EINVAL
        need = int(re.search(r"need (\d+) bytes", str(e)).group(1))
        with pytest.raises(hwkv.HwkvError):
            hwkv.decode_attn(cache, 0, q, 0.1, got, area[:need - 1])
    assert 0 <= need <= full.numel() and (max(lens) > 300) == (need > 0)
    got.fill_(float("nan"))
    hwkv.decode_attn(cache, 0, q, 0.1, got, area[:max(need, 1)])
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.isfinite(got).all()
    assert (area[need:] == 0x77).all()
    assert need == 0 or (area[:need] != 0x77).any()
    cache.free()
