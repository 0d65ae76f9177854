"""GPU tests: int8 decode keeps its weights to fp32's last places, in every layout
of the terms' rows (up to 4 heads, 6 and 8), by item, split and merged."""
import numpy as np
import pytest
import torch

from paper_2609_02029_amd import hwkv
from test_host_i8_terms import BOUND, ROUTES, SHAPES, expected, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def _up(x):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)
    assert np.array_equal(t.double().numpy(), x)
    return t.to(DEV)


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("D,G", SHAPES)
@pytest.mark.parametrize("route", ROUTES)
def test_weights_to_the_last_places(D, G, route, fused):
    """Each channel to 24 x 2^-24 of itself (a fused call appends a row of zeros)."""
    k, v, q, scale = values(D, G, route)
    ref, _ = expected(k, v, q, scale, G, more=int(fused))
    lens, hkv = ROUTES[route]
    pol = hwkv.policy_set(1, hkv, hkv * G, D, 0, [0], [[0] * hkv])
    cache = hwkv.cache_alloc(pol, len(lens), max(lens) + 8, kv_format="i8")
    for b in range(len(lens)):
        hwkv.prefill_write(cache, 0, b, 0, _up(k[b]), _up(v[b]))
    ws = torch.zeros(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    out = torch.full(q.shape, float("nan"), device=DEV)
    if fused:
        zero = torch.zeros((len(lens), hkv, D), dtype=torch.bfloat16, device=DEV)
        hwkv.append_decode_attn(cache, 0, zero, zero, _up(q), scale, out, ws)
    else:
        hwkv.decode_attn(cache, 0, _up(q), scale, out, ws)
    err = np.abs(out.double().cpu().numpy() - ref) / ref
    print(f"largest error {float(err.max() * 2 ** 24):.2f} x 2^-24")
    assert err.max() <= BOUND, float(err.max() / BOUND)
    cache.free()
