"""GPU tests of rotary positions: ``rope_apply`` against 64 bits, and
``append_rope`` against ``rope_apply`` followed by ``append``, bit for bit."""
import math

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


def rotation(D, rot, axes, seed, theta=1e4, pairing="half", magnitude=1.0):
    r = np.random.default_rng(seed)
    freq = theta ** (-2.0 * np.arange(rot // 2) / rot)
    axis = r.integers(0, axes, size=rot // 2)
    return hwkv.rope_set(D, freq, axis, n_axes=axes, pairing=pairing, magnitude=magnitude), freq, axis


def turned(x, pos, freq, axis, pairing, magnitude=1.0):
    """The definition, in 64 bits: x [n, h, D], pos [axes, n]."""
    x, half = x.double().cpu(), len(freq)
    out = x.clone()
    for i in range(half):
        t = pos[int(axis[i])].double().cpu() * float(freq[i])
        c, s = (magnitude * f(t)[:, None] for f in (torch.cos, torch.sin))
        a, b = (i, i + half) if pairing == "half" else (2 * i, 2 * i + 1)
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    return out


def close(got, ref, x, rot, far, magnitude=1.0):
    """Half a bf16 step of the result (2^-8, or 2^-134 where it is subnormal), and
    before that rounding, relative to the largest magnitude of the row: 16 x 2^-24
    for the angle in turns (pi 2^-24), sine and cosine (two last places each) and
    three fp32 roundings, and the angle itself, to 2^-50 of the ``far``thest."""
    got, x = got.double().cpu(), x.double().cpu()
    big = x.abs().amax(dim=-1, keepdim=True) * abs(magnitude)
    lim = 2.0 ** -8 * ref.abs() + 1.01 * big * (16 * 2.0 ** -24 + far * 2.0 ** -50) + 2.0 ** -134
    assert torch.all((got - ref).abs() <= lim), float(((got - ref).abs() / lim).max())
    assert torch.equal(got[..., rot:], x[..., rot:])


CASES = [(64, 64, 1, "half"), (64, 16, 2, "pairs"), (128, 128, 3, "half"), (128, 96, 4, "pairs"), (128, 48, 1, "half"),
         (256, 64, 3, "half"), (256, 256, 8, "pairs"), (256, 176, 2, "half")]


@pytest.mark.parametrize("D,rot,axes,pairing", CASES)
@pytest.mark.parametrize("n,hq,hk", [(1, 8, 2), (77, 6, 1), (1000, 3, 3), (5, 0, 2), (9, 4, 0)])
def test_rope_apply(D, rot, axes, pairing, n, hq, hk):
    far = 1 << 20
    rope, freq, axis = rotation(D, rot, axes, D + rot, pairing=pairing)
    g = torch.Generator(device=DEV).manual_seed(n)
    pos = torch.randint(-far, far, (axes, n), generator=g, device=DEV, dtype=torch.int32)
    x = torch.randn((n, hq + hk, D), generator=g, device=DEV).to(torch.bfloat16)
    q, k = (x[:, :hq].contiguous() if hq else None), (x[:, hq:].contiguous() if hk else None)
    qo, ko = (None if t is None else torch.zeros_like(t) for t in (q, k))
    hwkv.rope_apply(rope, pos, q, k, qo, ko)
    for t, o in ((q, qo), (k, ko)):
        if t is not None:
            close(o, turned(t, pos, freq, axis, pairing), t, rot, far)


@pytest.mark.parametrize("D,rot,pairing", [(64, 64, "half"), (128, 48, "pairs"), (256, 64, "half")])
def test_strided_and_in_place_give_the_same_bits(D, rot, pairing):
    """Slices of a wider row (its other parts stay), in place, and either side
    alone, equal the plain call."""
    n, hq, hk = 131, 6, 2
    rope, _, _ = rotation(D, rot, 2, 3, pairing=pairing)
    pos = torch.randint(0, 5000, (2, n), device=DEV, dtype=torch.int32)
    row = torch.randn((n, hq + 2 * hk + 1, D), device=DEV).to(torch.bfloat16)
    keep = row.clone()
    q, k = row[:, :hq], row[:, hq:hq + hk]
    want = [torch.empty((n, h, D), dtype=torch.bfloat16, device=DEV) for h in (hq, hk)]
    hwkv.rope_apply(rope, pos, q.contiguous(), k.contiguous(), *want)
    got = [torch.empty_like(w) for w in want]
    hwkv.rope_apply(rope, pos, q, k, *got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(row, keep)
    a, b = q.contiguous(), k.contiguous()
    hwkv.rope_apply(rope, pos, a, b, a, b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    only = torch.empty_like(want[1])
    hwkv.rope_apply(rope, pos, None, k, None, only)
    assert torch.equal(only, want[1])


def test_far_positions_frequencies_and_magnitude():
    """Positions up to 2^31 - 1 and down to -2^31, frequencies above one, a
    magnitude, and infinities and NaN in one head of one token only."""
    D, rot, n = 64, 64, 64
    freq = np.array([3.0 ** (1 - i) for i in range(32)])
    axis = np.arange(32) % 2
    rope = hwkv.rope_set(D, freq, axis, n_axes=2, magnitude=-0.75)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, n), device=DEV, dtype=torch.int64).to(torch.int32)
    pos[0, 0], pos[1, 1] = 2 ** 31 - 1, -2 ** 31
    q = torch.randn((n, 3, D), device=DEV).to(torch.bfloat16)
    q[7, 1, 5], q[7, 1, 9] = float("inf"), float("nan")
    out = torch.empty_like(q)
    hwkv.rope_apply(rope, pos, q, None, out, None)
    ref = turned(q, pos, freq, axis, "half", -0.75)
    fine = torch.ones((n, 3), dtype=torch.bool)
    fine[7, 1] = False
    # (both sides round an angle of 2^31 x 3 radians to 2^-52 of itself)
    close(out[fine.to(DEV)], ref[fine], q[fine.to(DEV)], rot, 3.0 * 2 ** 31, -0.75)
    bad = out[7, 1].float().cpu()
    hit = torch.zeros(D, dtype=torch.bool)
    hit[[5, 37, 9, 41]] = True
    assert torch.isfinite(bad[~hit]).all() and not torch.isfinite(bad[hit]).any()


def test_many_heads_no_tokens_and_another_stream():
    rope, freq, axis = rotation(64, 32, 1, 1)
    pos = torch.arange(3, device=DEV, dtype=torch.int32)
    q = torch.randn((3, 300, 64), device=DEV).to(torch.bfloat16)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    hwkv.rope_apply(rope, pos, q, None, out, None, stream=side)
    side.synchronize()
    close(out, turned(q, pos[None], freq, axis, "half"), q, 32, 4)
    none = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    hwkv.rope_apply(rope, pos[:0], none, None, none, None)


def test_more_tokens_than_one_launch():
    """The tokens past the first launch's, which start at neither side's first row,
    of strided q and k in place, with two axes of positions."""
    rope, freq, axis = rotation(64, 16, 2, 4)
    n, cut = 2 ** 22 + 300, 2 ** 22 - 5
    pos = torch.randint(0, 10 ** 6, (2, n), device=DEV, dtype=torch.int32)
    both = torch.randn((n, 2, 64), dtype=torch.bfloat16, device=DEV)
    q, k = both[:, :1], both[:, 1:].contiguous()
    qo, ko = torch.empty((n, 1, 64), dtype=torch.bfloat16, device=DEV), k.clone()
    hwkv.rope_apply(rope, pos, q, ko, qo, ko)
    few = pos[:, cut:].contiguous()
    q2, k2 = (torch.empty((n - cut, 1, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    hwkv.rope_apply(rope, few, q[cut:], k[cut:], q2, k2)
    assert torch.equal(qo[cut:], q2) and torch.equal(ko[cut:], k2)
    close(q2, turned(q[cut:], few, freq, axis, "half"), q[cut:], 16, 1e6)
    close(ko[:50], turned(k[:50], pos[:, :50], freq, axis, "half"), k[:50], 16, 1e6)


FORMATS = ["bf16", "f16", "fp8", "i8"]


def _caches(D, hkv, G, B, fmt, pages, S=3, w=70, max_ctx=900):
    pol = hwkv.policy_set(2, hkv, hkv * G, D, S, [w, 0], [[h % 2 for h in range(hkv)]] * 2)
    kw = dict(k_scale=0.02, v_scale=0.03) if fmt == "fp8" else {}
    need = hwkv.cache_bytes(pol, B, max_ctx, fmt, n_pages=pages)
    bufs = [torch.full((need,), 0x33, dtype=torch.uint8, device=DEV) for _ in range(2)]
    return [hwkv.cache_alloc(pol, B, max_ctx, dev_buf=b, kv_format=fmt, n_pages=pages, **kw) for b in bufs], bufs


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,rot,pairing,hkv,G,B,paged", [
    (64, 64, "half", 2, 4, 3, True), (128, 48, "pairs", 3, 1, 1, False), (256, 64, "half", 4, 6, 5, True),
    (64, 32, "half", 64, 1, 2, False),     # more heads than one launch takes
    (64, 16, "pairs", 2, 2, 200, True),    # more sequences than one launch takes
])
def test_append_rope_is_rope_then_append(fmt, D, rot, pairing, hkv, G, B, paged):
    """The whole cache, byte for byte, and the queries, over steps that wrap
    the window and enter a second page; strided inputs, ragged lengths."""
    pages = B * 2 * hkv * 2 if paged else None
    (one, two), bufs = _caches(D, hkv, G, B, fmt, pages)
    rope, _, _ = rotation(D, rot, 3, 11, pairing=pairing)
    g = torch.Generator(device=DEV).manual_seed(B)
    for b in range(B):
        n = 1 + (b * 37) % 254 if b else 254
        for layer in range(2):
            x = torch.randn((n, 2 * hkv, D), generator=g, device=DEV).to(torch.bfloat16)
            k, v = x[:, :hkv].contiguous(), x[:, hkv:].contiguous()
            for c in (one, two):
                hwkv.prefill_write(c, layer, b, 0, k, v)
    for step in range(6):
        layer = step % 2
        row = torch.randn((B, hkv * (G + 2), D), generator=g, device=DEV).to(torch.bfloat16)
        q, k, v = row[:, :hkv * G], row[:, hkv * G:hkv * (G + 1)], row[:, hkv * (G + 1):]
        pos = torch.randint(0, 1 << 20, (3, B), generator=g, device=DEV, dtype=torch.int32)
        qo, q1 = torch.empty((B, hkv * G, D), dtype=torch.bfloat16, device=DEV), None
        q1, k1 = torch.empty_like(qo), torch.empty((B, hkv, D), dtype=torch.bfloat16, device=DEV)
        if step == 4:                       # without queries
            hwkv.append_rope(one, layer, rope, pos, k, v)
        else:
            hwkv.append_rope(one, layer, rope, pos, k, v, q, qo)
        hwkv.rope_apply(rope, pos, q, k, q1, k1)
        hwkv.append(two, layer, k1, v.contiguous())
        torch.cuda.synchronize()
        assert step == 4 or torch.equal(qo, q1)
        assert torch.equal(bufs[0], bufs[1]), step
        for b in (0, B - 1):
            assert hwkv.cache_seq_len(one, layer, b) == hwkv.cache_seq_len(two, layer, b)
    one.free()
    two.free()


def test_append_rope_where_the_rotation_makes_a_row_infinite():
    """A rotated pair may pass bf16's largest value: an int8 row then reads as
    NaN, like a row that came in so, and the other rows stay."""
    (one, two), bufs = _caches(64, 2, 1, 1, "i8", None)
    rope = hwkv.rope_set(64, [1.0] * 8)
    k = torch.full((1, 2, 64), 1.0, device=DEV).to(torch.bfloat16)
    k[0, 0, 0] = k[0, 0, 8] = 3.3e38
    pos = torch.tensor([2], dtype=torch.int32, device=DEV)          # cos 2 - sin 2 = -1.33
    hwkv.append_rope(one, 0, rope, pos, k, k)
    ks, vs = hwkv.cache_read_scales(one, 0, 0, 0)
    assert ks[0] == 255 and vs[0] == 254
    assert hwkv.cache_read_scales(one, 0, 1, 0)[0][0] < 255
    one.free()
    two.free()


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_prompt_and_its_decoding_together(fmt):
    """The operators as a model's layer runs them: rotate a chunk, attend,
    write; then rotate and append a token and attend -- against 64 bits over
    keys rotated in 64 bits.  Two layers, windows and full units, paged."""
    D, hkv, G, B, P, steps, S, w = 128, 2, 4, 2, 300, 5, 4, 90
    pol = hwkv.policy_set(1, hkv, hkv * G, D, S, [w, 0], [[0, 1]])
    kw = dict(k_scale=0.03, v_scale=0.03) if fmt == "fp8" else {}
    cache = hwkv.cache_alloc(pol, B, 400, kv_format=fmt, n_pages=B * 2, **kw)
    rope, freq, axis = rotation(D, 96, 3, 5)
    g = torch.Generator(device=DEV).manual_seed(1)
    qkv = torch.randn((B, P + steps, hkv * (G + 2), D), generator=g, device=DEV).to(torch.bfloat16)
    pos = torch.randint(0, 4000, (B, 3, P + steps), generator=g, device=DEV, dtype=torch.int32)
    scale, hq = 1 / math.sqrt(D), hkv * G
    ws = torch.empty(max(1, hwkv.prefill_attn_workspace_bytes(cache, P)), dtype=torch.uint8, device=DEV)
    dws = torch.empty(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    got = torch.empty((B, P + steps, hq, D), device=DEV)
    for b in range(B):
        for p0, p1 in ((0, 101), (101, P)):
            x, t = qkv[b, p0:p1], pos[b, :, p0:p1].contiguous()
            q = torch.empty((p1 - p0, hq, D), dtype=torch.bfloat16, device=DEV)
            k = torch.empty((p1 - p0, hkv, D), dtype=torch.bfloat16, device=DEV)
            v = x[:, hq + hkv:].contiguous()
            hwkv.rope_apply(rope, t, x[:, :hq], x[:, hq:hq + hkv], q, k)
            hwkv.prefill_attn(cache, 0, b, p0, q, k, v, scale, got[b, p0:p1], ws=ws)
            hwkv.prefill_write(cache, 0, b, p0, k, v)
    for i in range(P, P + steps):
        x = qkv[:, i]
        q = torch.empty((B, hq, D), dtype=torch.bfloat16, device=DEV)
        out = torch.empty((B, hq, D), device=DEV)
        hwkv.append_rope(cache, 0, rope, pos[:, :, i].T.contiguous(), x[:, hq:hq + hkv], x[:, hq + hkv:],
                         x[:, :hq], q)
        hwkv.decode_attn(cache, 0, q, scale, out, dws)
        got[:, i] = out
    torch.cuda.synchronize()
    for b in range(B):
        x = qkv[b].cpu()
        q = turned(x[:, :hq], pos[b].cpu(), freq, axis, "half")
        k = turned(x[:, hq:hq + hkv], pos[b].cpu(), freq, axis, "half")
        v = x[:, hq + hkv:].double()
        at = torch.arange(P + steps)
        for h, win in ((0, w), (1, 10 ** 6)):
            seen = (at[None] <= at[:, None]) & ((at[None] < S) | (at[None] > at[:, None] - win))
            z = torch.einsum("tgd,sd->gts", q[:, h * G:(h + 1) * G], k[:, h]) * scale
            o = torch.softmax(z.masked_fill(~seen, -math.inf), dim=-1) @ v[:, h]
            d = (got[b, :, h * G:(h + 1) * G].permute(1, 0, 2).cpu().double() - o)
            # relative, in norm: half a bf16 step (2^-8) of q, of k and of prefill's
            # weights; and of K and V each what the format takes: half a step of f16
            # (2^-11) or fp8 (2^-4), or of an int8 row's power of two: 2^-7 / sqrt(3)
            # of its largest, which is at most 4 standard deviations here
            stored = {"bf16": 0.0, "f16": 2.0 ** -11, "fp8": 2.0 ** -4, "i8": 2.3 * 2.0 ** -7}[fmt]
            norm = d.norm() / o.norm()
            assert norm <= 3 * 2.0 ** -8 + 2 * stored, (fmt, h, float(norm))
    cache.free()


def test_capture_and_replay():
    """A captured rotation follows its inputs; the eager calls between the
    replays do not disturb it."""
    rope, freq, axis = rotation(128, 128, 1, 2)
    pos = torch.zeros(50, dtype=torch.int32, device=DEV)
    q = torch.zeros((50, 4, 128), dtype=torch.bfloat16, device=DEV)
    out, want = torch.empty_like(q), torch.empty_like(q)
    hwkv.rope_apply(rope, pos, q, None, out, None)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hwkv.rope_apply(rope, pos, q, None, out, None)
    for i in range(4):
        pos.copy_(torch.randint(0, 9999, (50,), device=DEV, dtype=torch.int32))
        q.copy_(torch.randn((50, 4, 128), device=DEV))
        hwkv.rope_apply(rope, pos, q, None, want, None)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
