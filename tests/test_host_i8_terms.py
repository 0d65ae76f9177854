"""The accuracy of int8 decode's weights: rows on which the third bf16 term of a
weight shows, the bound that decode keeps on them, and (CPU) that two terms break
it.

Every (sequence, KV head) holds rows whose key and value are zero, which have
logit 0 and, since no logit is above it, weight exactly 1, and three rows of a
negative logit that give each channel to one of them.  A channel's output is then
p v / L: the weight p of one row, with nothing for its rounding to hide in.

What decode may be off by, relative to p v / L, in units of 2^-24: the logit (base
2, at most 1.5) its sum of digits 1, the scale times log2(e) 2, their product 1: 4 x
1.5 x ln 2 = 4.2; the exponential two last places, 4; three terms leave 0.2; the
terms' sum 3; the sum of weights, of which those three rows are at most 3/4, 3/4 of
8.2 and four roundings (lanes, wavefronts, workgroups), 10; the quotient and the
product 2: 24 of them."""
import numpy as np
import pytest

BOUND = 24 * 2.0 ** -24

# (sequence lengths, KV heads): by item in one launch; split, beside items of one
# workgroup; by item, one sequence split and merged
ROUTES = {"item": ([4, 65, 200, 300], 2), "split": ([5000, 70, 9], 2),
          "item merge": ([6000] + [30 + 9 * i for i in range(23)], 4)}
SHAPES = [(64, 1), (64, 6), (128, 2), (128, 8), (256, 4), (256, 6)]


def special(n):
    """The three rows of a sequence of n: in its first tile, its second and about
    the middle, or the first tile where it is short."""
    return [1, 64 + 17 if n > 82 else 2, n // 2 if n > 200 else 3]


def values(D, G, route):
    """Codes / 64 of k, v [n, hkv, D] a sequence, q [B, hq, D] and the logit scale:
    all of them bf16 values, and k and v exact in int8 rows."""
    lens, hkv = ROUTES[route]
    r = np.random.default_rng(D * 10 + G)
    k, v = [], []
    for n in lens:
        kb, vb = np.zeros((n, hkv, D)), np.zeros((n, hkv, D))
        for j, s in enumerate(special(n)):
            low = r.integers(10, 80, size=(hkv, 1))
            kb[s] = -r.integers(low, low + 40, size=(hkv, D)) / 64.0
            kb[s, :, 0] = -127 / 64.0
            vb[s, :, j::3] = r.integers(64, 128, size=(hkv, len(range(j, D, 3)))) / 64.0
        k.append(kb)
        v.append(vb)
    q = r.integers(64, 128, size=(len(lens), hkv * G, D)) / 64.0
    return k, v, q, float(np.float32(0.55 / D / 1.5))


def expected(k, v, q, scale, G, more=0):
    """In 64 bits: the output (with ``more`` rows of zeros behind), and the weights of
    the three rows [3, B, hq]."""
    out, w = np.empty(q.shape), np.empty((3, *q.shape[:2]))
    for b, (kb, vb) in enumerate(zip(k, v)):
        for h in range(q.shape[1]):
            s = special(len(kb))
            p = np.exp(kb[s, h // G] @ q[b, h] * scale)
            w[:, b, h] = p
            out[b, h] = p @ vb[s, h // G] / (p.sum() + len(kb) - 3 + more)
    return out, w


def _bf16(x):
    """Nearest bf16 of fp32, ties to even."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def terms(p, n):
    """The sum of the first n bf16 terms of fp32 weights."""
    rest, total = p.astype(np.float32), np.zeros(p.shape)
    for _ in range(n):
        t = _bf16(rest)
        total, rest = total + t, rest - t
    return total


@pytest.mark.parametrize("D,G", SHAPES)
@pytest.mark.parametrize("route", ROUTES)
def test_two_terms_would_break_the_bound(D, G, route):
    k, v, q, scale = values(D, G, route)
    _, w = expected(k, v, q, scale, G)
    z = np.log2(w)
    assert z.max() < -0.01 and z.min() > -1.5
    two, three = (np.abs(terms(w, n) - w.astype(np.float32)) / w for n in (2, 3))
    assert two.max() > 2 * BOUND and three.max() <= 2.0 ** -26
    # and in every one of the three places
    assert (two.reshape(3, -1).max(axis=1) > BOUND).all()
