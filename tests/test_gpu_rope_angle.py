"""GPU tests of the rotation's angles: every frequency that ``rope_set`` takes, at
positions up to the ends of int32, against angles reduced in whole numbers."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2609_02029_amd import hwkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


BITS = 240


def _arctan_inverse(n):
    """arctan(1 / n) in units of 2^-BITS (Machin's series)."""
    t = (1 << BITS) // n
    total, k, sign = t, 3, -1
    while t:
        t //= n * n
        total += sign * (t // k)
        k, sign = k + 2, -sign
    return total


PI = Fraction(4 * (4 * _arctan_inverse(5) - _arctan_inverse(239)), 1 << BITS)


def angle(pos, freq):
    """pos x freq (a double) radians less whole turns, in [-pi, pi]."""
    x = int(pos) * Fraction(float(freq))
    return float(x - round(x / (2 * PI)) * 2 * PI)


def test_pi():
    assert float(PI) == math.pi and abs(float(PI - Fraction(math.pi)) - 1.2246467991473532e-16) < 1e-30


def _positions(n, seed):
    r = np.random.default_rng(seed)
    pos = r.integers(-2 ** 31, 2 ** 31, size=n)
    pos[:8] = [2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, 2 ** 30 + 1, 2 ** 24 + 1, 1, 0, -1]
    return pos


def _expected(x, pos, freq, pairing):
    """x [n, heads, D] turned, in 64 bits from reduced angles."""
    half, out = len(freq), x.copy()
    for i in range(half):
        t = np.array([angle(p, freq[i]) for p in pos])
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        a, b = (i, i + half) if pairing == "half" else (2 * i, 2 * i + 1)
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def _limit(ref, x):
    """Half a bf16 step of the result, and before that rounding, relative to the
    row's largest: the angle in half turns rounds to 2^-24 (pi 2^-24 radians), sine
    and cosine to two last places each, and three fp32 roundings: 16 x 2^-24."""
    return 2.0 ** -8 * np.abs(ref) + 1.01 * np.abs(x).max(axis=-1, keepdims=True) * 16 * 2.0 ** -24 + 2.0 ** -134


# (1e6 is the largest frequency taken)
@pytest.mark.parametrize("pairing", ["half", "pairs"])
@pytest.mark.parametrize("top", [1.0, 3.0, 1e2, 1e4, 1e6])
def test_angles_of_far_positions(top, pairing):
    D, n = 64, 600
    freq = top * np.exp2(-np.arange(32) / 8.0) * np.where(np.arange(32) % 3 == 2, -1, 1)
    rope = hwkv.rope_set(D, freq, pairing=pairing)
    pos = _positions(n, int(top))
    r = np.random.default_rng(1)
    x = r.normal(size=(n, 2, D))
    # one head of pairs (1, 0), whose results are the cosines and sines
    x[:, 1] = 0.0
    x[:, 1, slice(0, 32) if pairing == "half" else slice(0, D, 2)] = 1.0
    q = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    out = torch.empty_like(q)
    hwkv.rope_apply(rope, torch.from_numpy(pos.astype(np.int32)).to(DEV), q, None, out, None)
    x = q.double().cpu().numpy()
    ref = _expected(x, pos, freq, pairing)
    err, lim = np.abs(out.double().cpu().numpy() - ref), _limit(ref, x)
    assert np.all(err <= lim), float((err / lim).max())


def test_append_turns_far_positions_alike():
    """append_rope's queries at the largest frequency are rope_apply's, bit for
    bit, and a bf16 cache holds its keys."""
    D, B = 128, 40
    freq = 1e6 * 0.8 ** np.arange(64)
    rope = hwkv.rope_set(D, freq)
    pol = hwkv.policy_set(1, 2, 4, D, 0, [0], [[0, 0]])
    cache = hwkv.cache_alloc(pol, B, 64)
    pos = torch.from_numpy(_positions(B, 3).astype(np.int32)).to(DEV)
    row = torch.randn((B, 8, D), device=DEV).to(torch.bfloat16)
    q, k, v = row[:, :4], row[:, 4:6], row[:, 6:].contiguous()
    qo, q1, k1 = (torch.empty((B, h, D), dtype=torch.bfloat16, device=DEV) for h in (4, 4, 2))
    hwkv.append_rope(cache, 0, rope, pos, k, v, q, qo)
    hwkv.rope_apply(rope, pos, q, k, q1, k1)
    torch.cuda.synchronize()
    assert torch.equal(qo, q1)
    x = k.double().cpu().numpy()
    ref = _expected(x, pos.cpu().numpy(), freq, "half")
    assert np.all(np.abs(k1.double().cpu().numpy() - ref) <= _limit(ref, x))
    for b in (0, 1, B - 1):
        for h in range(2):
            held = hwkv.cache_read_unit(cache, 0, h, b)[0][0]
            assert np.array_equal(held, k1[b, h].view(torch.int16).cpu().numpy().view(np.uint16))
    cache.free()
