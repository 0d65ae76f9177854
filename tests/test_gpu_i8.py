"""GPU tests of int8 caches (rows with a scale of their own): what the write
paths store, bit for bit against the oracle's encoding, and decode attention,
prefill attention and the calibration replay over it against 64 bits."""
import math

import numpy as np
import pytest
import torch

import oracle
import workloads as W
from hwkv_harness import Run, log, up
from oracle import kvformat as KF
from paper_2609_02029_amd import hwkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


class Run8(Run):
    """``Run`` over an int8 cache: codes and scale bytes are both checked."""

    def __init__(self, cfg, **kw):
        super().__init__(cfg, kv_format="i8", **kw)

    def check_unit(self, layer, h, b, hist=None):
        tab = oracle.UnitTable(self.S, self.windows[layer][h], self.max_ctx)
        if self.n[layer, b] > 0:
            tab.prefill(0, int(self.n[layer, b]))
        nv = tab.n_valid
        hk, hv = (self.kh[layer][b], self.vh[layer][b]) if hist is None else hist
        same_rows(self.cache, layer, h, b, nv, hk[tab.table[:nv], h], hv[tab.table[:nv], h])


def same_rows(cache, layer, h, b, nv, k_bits, v_bits):
    """The unit holds exactly the oracle's encoding of these bf16 rows."""
    k, v, n = hwkv.cache_read_unit(cache, layer, h, b)
    ks, vs = hwkv.cache_read_scales(cache, layer, h, b)
    assert n == nv and k.dtype == np.int8
    for got, sc, bits, what in ((k, ks, k_bits, "K"), (v, vs, v_bits, "V")):
        exp = KF.store(bits, "i8")
        assert np.array_equal(sc[:nv], exp["scale"][:, 0]), f"{what} scales, head {h} seq {b}"
        assert np.array_equal(got[:nv], exp["code"]), f"{what} codes, head {h} seq {b}"


def mini(**kw):
    c = dict(name="mini", seed=41, n_layers=1, batch=1, n_q_heads=8, n_kv_heads=2, head_dim=64,
             n_sinks=4, level_windows=[256, 0], levels=[[0, 1]], prompt=[300], steps=4, max_ctx=400)
    c.update(kw)
    return c


# ---------------------------------------------------------------------------
# what is stored
# ---------------------------------------------------------------------------
def _odd_rows(D, n, seed):
    """bf16 rows where the format can go wrong: every magnitude, one loud
    channel, ties at half steps, the clamp, zeros, subnormals, infinities, NaN."""
    r = np.random.default_rng(seed)
    x = (r.normal(size=(n, D)) * np.exp2(r.integers(-120, 120, size=(n, 1)))).astype(np.float32)
    bits = (x.view(np.uint32) >> 16).astype(np.uint16)
    for i in range(n):
        kind = i % 12
        if kind == 1:
            bits[i] = r.integers(0, 65536, size=D)          # any pattern: mostly not finite
        elif kind == 2:
            bits[i] = r.integers(0, 0x7f80, size=D) | (r.integers(0, 2, size=D) << 15)   # finite
        elif kind == 3:
            bits[i] = 0
        elif kind == 4:
            bits[i] = r.integers(0, 0x80, size=D) | (r.integers(0, 2, size=D) << 15)     # subnormal
        elif kind == 5:                                      # whole and half steps under 1.x
            v = (r.integers(-255, 256, size=D) / 128.0).astype(np.float32)
            v[0] = 1.9921875                                 # 127.5 steps: clamped
            bits[i] = (v.view(np.uint32) >> 16).astype(np.uint16)
        elif kind == 6:
            bits[i, r.integers(D)] = 0x7f80                  # one infinity
        elif kind == 7:
            bits[i, r.integers(D)] = 0xffc1                  # one NaN
        elif kind == 8:
            bits[i] = 0
            bits[i, r.integers(D)] = 0x8001                  # the smallest, negative
        elif kind == 9:
            bits[i, r.integers(D)] = 0x7f7f                  # the largest
        elif kind == 10:
            bits[i, -1] = 0xc47a                             # loud last channel
    return bits


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("paged", [False, True])
def test_rows_are_stored_as_the_format_says(D, paged):
    """Prefill in ragged chunks, append and the fused append, over a window
    that wraps and a full unit (of several pages)."""
    S, w, P, steps, B = 3, 150, 523, 9, 2
    pol = hwkv.policy_set(1, 2, 4, D, S, [w, 0], [[0, 1]])
    cache = hwkv.cache_alloc(pol, B, 700, kv_format="i8", n_pages=B * 3 if paged else None)
    k = np.stack([_odd_rows(D, (P + steps) * 2, 7 + b).reshape(-1, 2, D) for b in range(B)])
    v = np.stack([_odd_rows(D, (P + steps) * 2, 17 + b).reshape(-1, 2, D) for b in range(B)])
    for b in range(B):
        for p0, p1 in ((0, 1), (1, 64), (64, 300), (300, 301), (301, P)):
            hwkv.prefill_write(cache, 0, b, p0, up(k[b, p0:p1], DEV), up(v[b, p0:p1], DEV))
    ws = torch.zeros(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    q = torch.randn((B, 4, D), device=DEV).to(torch.bfloat16)
    out = torch.empty((B, 4, D), device=DEV)
    for i in range(steps):
        kn, vn = up(k[:, P + i], DEV), up(v[:, P + i], DEV)
        if i % 2:
            hwkv.append(cache, 0, kn, vn)
        else:
            hwkv.append_decode_attn(cache, 0, kn, vn, q, 0.1, out, ws)
    n = P + steps
    for b in range(B):
        for h, win in ((0, w), (1, 0)):
            tab = oracle.UnitTable(S, win, 700)
            tab.prefill(0, n)
            at = tab.table[:tab.n_valid]
            same_rows(cache, 0, h, b, tab.n_valid, k[b][at, h], v[b][at, h])
    cache.free()


def test_rows_beyond_the_written_ones_stay():
    """A chunk writes its own slots' codes and scale bytes and no others."""
    D = 64
    pol = hwkv.policy_set(1, 1, 1, D, 0, [0], [[0]])
    need = hwkv.cache_bytes(pol, 2, 256, "i8")
    assert need == 2 * 256 * (2 * D + 2)
    buf = torch.full((need,), 0x5a, dtype=torch.uint8, device=DEV)
    cache = hwkv.cache_alloc(pol, 2, 256, dev_buf=buf, kv_format="i8")
    x = W.normal_bf16((70, 1, D), 3, 0, W.K, 0)
    hwkv.prefill_write(cache, 0, 1, 0, up(x, DEV), up(x, DEV))
    got = buf.cpu().numpy()
    codes, pairs = got[:2 * 2 * 256 * D].reshape(2, 2, 256 * D), got[2 * 2 * 256 * D:].reshape(2, 256, 2)
    assert (codes[:, 0] == 0x5a).all() and (pairs[0] == 0x5a).all()      # the other sequence
    assert (pairs[1, 70:] == 0x5a).all() and (codes[1, 1].reshape(256, D)[70:] == 0x5a).all()
    kt = codes[0, 1].reshape(4, D // 8, 64, 8)
    assert (kt[1, :, 6:] == 0x5a).all() and (kt[2:] == 0x5a).all()
    cache.free()


# ---------------------------------------------------------------------------
# decode attention
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("D,G", [(d, g) for d in (64, 128, 256) for g in (1, 2, 4, 6, 8)])
def test_decode_every_head_dim_and_group(D, G):
    """Fused and separate steps over prompts of 1 to several hundred tokens, a
    window that wraps and a full unit."""
    c = mini(batch=4, head_dim=D, n_q_heads=2 * G, prompt=[1, 63, 64, 333], n_sinks=3, level_windows=[100, 0])
    r = Run8(c)
    for b in range(r.B):
        r.prefill(0, b, chunks=[5, 129] if r.prompts[b] > 129 else None)
    for st in range(4):
        qa, out = r.step(0, fused=st % 2 == 0)
        r.check_out(0, qa, out, f"D={D} G={G} step {st}")
    r.check_layer(0)
    r.free()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("D,G,lens", [(256, 6, [9000, 1, 2500]), (128, 4, [12001, 64, 700]), (64, 8, [16000, 17, 129])])
def test_decode_long_and_ragged(D, G, lens, paged):
    """Every split workgroup walks several tiles; the ends of tiles and pages."""
    c = mini(batch=3, head_dim=D, n_q_heads=4 * G, n_kv_heads=4, prompt=lens, max_ctx=17000,
             level_windows=[300, 5000, 0], levels=[[0, 1, 2, 2]], outliers=True)
    pages = 2 * sum((n + 10 + 255) // 256 for n in lens) if paged else None
    r = Run8(c, n_pages=pages)
    for b in range(r.B):
        r.prefill(0, b)
    for st in range(3):
        qa, out = r.step(0, fused=st != 1)
        r.check_out(0, qa, out, f"D={D} paged={paged} step {st}")
    r.check_layer(0)
    r.free()


@pytest.mark.parametrize("batch", [1, 20, 200])
def test_decode_batches(batch):
    """Batches of fewer and more sequences than a launch holds, ragged."""
    rng = np.random.default_rng(batch)
    c = mini(batch=batch, head_dim=64, n_q_heads=8, n_kv_heads=4, levels=[[0, 1, 1, 0]],
             prompt=[int(x) for x in rng.integers(1, 500, size=batch)], max_ctx=600)
    r = Run8(c)
    for b in range(batch):
        r.prefill(0, b)
    for st in range(2):
        qa, out = r.step(0, fused=st == 1)
        r.check_out(0, qa, out, f"batch {batch} step {st}")
    for b in (0, batch // 2, batch - 1):
        for h in range(4):
            r.check_unit(0, h, b)
    r.free()


def _one_unit(k, v, D, G=2, S=0, window=0, max_ctx=600):
    """A one-head int8 cache filled with bf16 bit rows k, v [n, D]."""
    pol = hwkv.policy_set(1, 1, G, D, S, [window], [[0]])
    cache = hwkv.cache_alloc(pol, 1, max_ctx, kv_format="i8")
    hwkv.prefill_write(cache, 0, 0, 0, up(k[:, None], DEV), up(v[:, None], DEV))
    ws = torch.zeros(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    return cache, ws


def _decode(cache, ws, q_bits, scale):
    q = up(q_bits[None], DEV)
    out = torch.full(q.shape, float("nan"), device=DEV)
    hwkv.decode_attn(cache, 0, q, scale, out, ws)
    return out.cpu().numpy()[0].astype(np.float64)


def _reference(q_bits, k, v, scale):
    return KF.attend_values(KF.bf16_values(q_bits)[None], [KF.values(KF.store(k, "i8"), "i8")[:, None]],
                            [KF.values(KF.store(v, "i8"), "i8")[:, None]], [len(k) - 1], 0, [0], scale)[0]


@pytest.mark.parametrize("spread", [0, 8, 40])
def test_decode_rows_of_unlike_scales(spread):
    """Rows whose magnitudes differ by up to 2^spread, in K (the softmax is
    nearly hard) and in V (the weights meet scales far apart)."""
    D, n = 128, 500
    r = np.random.default_rng(spread)
    bits = lambda x: (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)
    k = bits(r.normal(size=(n, D)) * np.exp2(r.integers(-spread, 1, size=(n, 1)) / 4.0))
    v = bits(r.normal(size=(n, D)) * np.exp2(r.integers(-spread, spread + 1, size=(n, 1))))
    q = bits(r.normal(size=(2, D)))
    cache, ws = _one_unit(k, v, D)
    got, ref = _decode(cache, ws, q, 1 / math.sqrt(D)), _reference(q, k, v, 1 / math.sqrt(D))
    # the weights to 2^-16 of themselves, logits and sums in 32 bits: relative to
    # the sum of the terms' magnitudes, 2^-16 + 2e-5
    kk, vv = KF.values(KF.store(k, "i8"), "i8"), KF.values(KF.store(v, "i8"), "i8")
    z = KF.bf16_values(q) @ kk.T / math.sqrt(D)
    p = np.exp(z - z.max(axis=1, keepdims=True))
    lim = (2.0 ** -16 + 2e-5) * (p @ np.abs(vv)) / p.sum(axis=1, keepdims=True)
    assert np.all(np.abs(got - ref) <= lim), float((np.abs(got - ref) / lim).max())
    cache.free()


def test_decode_large_and_small_queries():
    """Queries of any magnitude, and one whose components span 2^20: what is
    below 2^-14 of the largest enters to 2^-22 of it."""
    D, n = 64, 200
    r = np.random.default_rng(5)
    bits = lambda x: (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)
    k, v = bits(r.normal(size=(n, D))), bits(r.normal(size=(n, D)))
    cache, ws = _one_unit(k, v, D)
    kk = np.abs(KF.values(KF.store(k, "i8"), "i8")).sum(axis=1).max()
    for mag in (2.0 ** -90, 2.0 ** -20, 1.0, 2.0 ** 20, 2.0 ** 90):
        x = r.normal(size=(2, D)) * mag
        x[1] *= np.exp2(r.integers(-20, 1, size=D))
        q = bits(x)
        scale = float(np.float32(0.125 / mag))
        got, ref = _decode(cache, ws, q, scale), _reference(q, k, v, scale)
        top = np.abs(KF.bf16_values(q)).max()
        dz = 2.0 ** -23 * top * kk * scale + 1e-5       # error of a logit
        lim = (2 * dz + 2.0 ** -16 + 2e-5) * np.abs(KF.values(KF.store(v, "i8"), "i8")).max()
        assert np.abs(got - ref).max() <= lim, mag
    zero = np.zeros((2, D), dtype=np.uint16)            # equal weights
    assert np.abs(_decode(cache, ws, zero, 0.125) - _reference(zero, k, v, 0.125)).max() < 1e-5
    cache.free()


def test_decode_keys_of_any_magnitude():
    """Keys near the ends of the range, under a scale that makes the logits
    ordinary; values of 2^-100 and 2^100."""
    D, n = 64, 300
    r = np.random.default_rng(8)
    bits = lambda x: (np.ascontiguousarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)
    for km, vm, qm in ((2.0 ** 110, 2.0 ** 100, 2.0 ** -50), (2.0 ** -110, 2.0 ** -100, 2.0 ** 50), (1.0, 2.0 ** 115, 1.0)):
        k, v, q = bits(r.normal(size=(n, D)) * km), bits(r.normal(size=(n, D)) * vm), bits(r.normal(size=(2, D)) * qm)
        cache, ws = _one_unit(k, v, D)
        scale = float(np.float32(0.125 / (km * qm)))
        got, ref = _decode(cache, ws, q, scale) / vm, _reference(q, k, v, scale) / vm
        # as test_decode_large_and_small_queries: logits to 1e-5, weights to 2^-16
        assert np.abs(got - ref).max() <= (2e-5 + 2.0 ** -16 + 2e-5) * 4.0 and np.abs(ref).max() > 1e-2
        cache.free()


def test_decode_one_long_sequence_among_many_short():
    """More items than a split launch takes, one of them of hundreds of tiles:
    its splits meet in the merge, the others stay whole."""
    c = mini(batch=24, head_dim=128, n_q_heads=16, n_kv_heads=4, levels=[[0, 1, 1, 0]], level_windows=[3000, 0],
             prompt=[37 + 11 * i for i in range(23)] + [20001], max_ctx=20100)
    r = Run8(c)
    for b in range(24):
        r.prefill(0, b)
    for st in range(2):
        qa, out = r.step(0, fused=st == 1)
        r.check_out(0, qa, out, f"step {st}")
    for b in (0, 22, 23):
        for h in range(4):
            r.check_unit(0, h, b)
    r.free()


@pytest.mark.parametrize("paged", [False, True])
def test_decode_past_four_gigabytes(paged):
    """Rows, scale pairs and pages whose offsets pass 2^32: keys of zero give
    every row the same weight, a loud key at the very end takes all of it."""
    D, H, n, step = 64, 4, 17_000_000, 1_000_000
    pol = hwkv.policy_set(1, H, H, D, 0, [0], [[0] * H])
    cache = hwkv.cache_alloc(pol, 1, n, kv_format="i8", n_pages=H * -(-n // 256) if paged else None)
    assert hwkv.cache_bytes(pol, 1, n, "i8") > 2 * 2 ** 32
    total = torch.zeros((H, D), dtype=torch.float64, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(3)
    for p0 in range(0, n, step):
        log(f"rows {p0}")
        k = torch.zeros((step, H, D), dtype=torch.bfloat16, device=DEV)
        # rows whose codes are exact: multiples of 1/64 below 2, the first 1
        v = (torch.randint(-100, 101, (step, H, D), generator=g, device=DEV).float() / 64).to(torch.bfloat16)
        v[:, :, 0] = 1.0
        v = v.clamp(-1.5, 1.5)
        if p0 + step == n:
            k[-1] = 8.0
            last = v[-1].double()
        total += v.double().sum(dim=0)
        hwkv.prefill_write(cache, 0, 0, p0, k, v)
    ws = torch.empty(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
    out = torch.empty((1, H, D), device=DEV)
    hwkv.decode_attn(cache, 0, torch.zeros((1, H, D), dtype=torch.bfloat16, device=DEV), 1.0, out, ws)
    # fp32 sums of 17M terms in thousands of parts: far below 1e-4 of a row's largest
    assert (out[0].double() - total / n).abs().max() < 1e-4
    hwkv.decode_attn(cache, 0, torch.full((1, H, D), 2.0, device=DEV).to(torch.bfloat16), 1.0, out, ws)
    assert (out[0].double() - last).abs().max() < 1e-5        # e^-1024 is zero
    cache.free()


def test_two_streams_at_once():
    """Calls on two caches and two streams, each with its own workspace, give
    what they give alone."""
    runs = [Run8(mini(seed=50 + i, batch=3, head_dim=128, n_q_heads=16, n_kv_heads=4, levels=[[0, 1, 1, 0]],
                      prompt=[3000, 500, 77], max_ctx=3200)) for i in range(2)]
    qs, alone = [], []
    for i, r in enumerate(runs):
        for b in range(3):
            r.prefill(0, b)
        qs.append(up(W.normal_bf16((3, 16, 128), 60 + i, 0, W.Q, 0), DEV))
        alone.append(torch.empty((3, 16, 128), device=DEV))
        hwkv.decode_attn(r.cache, 0, qs[i], r.scale, alone[i], r.ws)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in runs], [torch.zeros_like(a) for a in alone]
    for _ in range(20):
        for i, r in enumerate(runs):
            hwkv.decode_attn(r.cache, 0, qs[i], r.scale, outs[i], r.ws, stream=streams[i])
    torch.cuda.synchronize()
    for i, r in enumerate(runs):
        assert torch.equal(outs[i], alone[i])
        r.free()


@pytest.mark.parametrize("where", ["k", "v"])
def test_decode_a_row_that_is_not_finite_poisons_only_what_sees_it(where):
    D, n = 64, 300
    x = {"k": W.normal_bf16((n, 2, D), 9, 0, W.K, 0), "v": W.normal_bf16((n, 2, D), 9, 0, W.V, 0)}
    x[where][137, 1, 5] = 0x7f80
    # KV head 0 sees everything finite; head 1 holds the row, until its window moves on
    pol = hwkv.policy_set(1, 2, 4, D, 0, [0, 100], [[0, 1]])
    for n_now, seen in ((200, True), (300, False)):
        cache = hwkv.cache_alloc(pol, 1, 400, kv_format="i8")
        hwkv.prefill_write(cache, 0, 0, 0, up(x["k"][:n_now], DEV), up(x["v"][:n_now], DEV))
        ws = torch.zeros(hwkv.decode_workspace_bytes(cache), dtype=torch.uint8, device=DEV)
        q = torch.randn((1, 4, D), device=DEV).to(torch.bfloat16)
        out = torch.zeros((1, 4, D), device=DEV)
        hwkv.decode_attn(cache, 0, q, 0.125, out, ws)
        o = out.cpu().numpy()[0]
        assert np.isfinite(o[:2]).all()
        assert np.isnan(o[2:]).all() if seen else np.isfinite(o[2:]).all()
        cache.free()


def test_decode_ignores_what_lies_behind_the_last_row():
    """Codes and scale bytes past the last row may hold anything (255, an
    infinite scale, among it)."""
    D, n = 128, 70
    k, v = W.normal_bf16((n, 1, D), 2, 0, W.K, 0), W.normal_bf16((n, 1, D), 2, 0, W.V, 0)
    pol = hwkv.policy_set(1, 1, 4, D, 0, [0], [[0]])
    outs = []
    for fill in (0x00, 0xff, 0x80):
        buf = torch.full((hwkv.cache_bytes(pol, 1, 200, "i8"),), fill, dtype=torch.uint8, device=DEV)
        cache = hwkv.cache_alloc(pol, 1, 200, dev_buf=buf, kv_format="i8")
        hwkv.prefill_write(cache, 0, 0, 0, up(k, DEV), up(v, DEV))
        ws = torch.full((hwkv.decode_workspace_bytes(cache),), 0xff, dtype=torch.uint8, device=DEV)
        q = up(W.normal_bf16((1, 4, D), 2, 0, W.Q, 0), DEV)
        out = torch.empty((1, 4, D), device=DEV)
        hwkv.decode_attn(cache, 0, q, 0.1, out, ws)
        outs.append(out.cpu())
        cache.free()
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_decode_noalloc_other_stream_and_capture():
    """The allocation-free call, a call on a stream of its own, and a captured
    and replayed decode_attn give the plain call's bits."""
    c = mini(batch=2, head_dim=128, n_q_heads=8, n_kv_heads=2, prompt=[900, 333], max_ctx=1200)
    r = Run8(c)
    for b in range(2):
        r.prefill(0, b)
    q = up(W.normal_bf16((2, 8, 128), 1, 0, W.Q, 0), DEV)
    want = torch.empty((2, 8, 128), device=DEV)
    hwkv.decode_attn(r.cache, 0, q, r.scale, want, r.ws)
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), torch.zeros_like(want)
    hwkv.decode_attn(r.cache, 0, q, r.scale, got, r.ws, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    got.zero_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        hwkv.decode_attn(r.cache, 0, q, r.scale, got, r.ws)
    for i in range(4):
        q.copy_(up(W.normal_bf16((2, 8, 128), 1, 0, W.Q, i), DEV))
        got.zero_()
        hwkv.decode_attn(r.cache, 0, q, r.scale, want, r.ws)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
    kn, vn = (up(W.normal_bf16((2, 2, 128), 1, 0, kind, 9), DEV) for kind in (W.K, W.V))
    # (a fused call takes the new token's tile first, so it is compared with the
    # fused call on a cache of the same rows, not with decode_attn)
    twin = Run8(c)
    for b in range(2):
        twin.prefill(0, b)
    hwkv.append_decode_attn_noalloc(r.cache, 0, kn, vn, q, r.scale, got)
    hwkv.append_decode_attn(twin.cache, 0, kn, vn, q, r.scale, want, twin.ws)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    r.free()
    twin.free()


def test_paged_and_reserved_rows_give_the_same_bits():
    c = mini(batch=2, head_dim=128, n_q_heads=16, n_kv_heads=4, prompt=[700, 300], max_ctx=1000,
             levels=[[0, 1, 1, 0]])
    outs = []
    for pages in (None, 2 * 2 * 4):
        r = Run8(c, n_pages=pages)
        for b in range(2):
            r.prefill(0, b, chunks=[100])
        outs.append([r.step(0)[1].cpu() for _ in range(3)])
        r.check_layer(0)
        r.free()
    for x, y in zip(*outs):
        assert torch.equal(x, y)


# ---------------------------------------------------------------------------
# prefill attention and the calibration replay
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("D,G,P,chunks", [(64, 1, 500, [77, 78]), (128, 4, 700, [300, 512]), (256, 6, 400, [1, 129])])
@pytest.mark.parametrize("paged", [False, True])
def test_prefill_attention(D, G, P, chunks, paged):
    """Every row within the weight-rounding bound of prefill attention: the
    weights enter rounded to bf16, |o - ref| <= (2^-8 + 2e-5) max |v|."""
    c = mini(head_dim=D, n_q_heads=2 * G, prompt=[P], max_ctx=P + 8, n_sinks=4, level_windows=[90, 0])
    r = Run8(c, n_pages=4 if paged else None)
    q, qh, out = r.prefill_with_attn(0, 0, chunks=chunks, check_untouched=True)
    torch.cuda.synchronize()
    rows = np.arange(P)
    ref = r.oracle_rows(0, 0, rows, qh)
    got = out.cpu().numpy().astype(np.float64)
    kv, vv = r.stored_values(0, r.kh[0][0][:P], r.vh[0][0][:P])
    for h in range(2):
        for t in rows:
            pos = KF.retained_positions(int(t), r.S, r.windows[0][h])
            lim = (2.0 ** -8 + 2e-5) * np.abs(vv[pos, h]).max(axis=0)
            err = np.abs(got[t, h * G:(h + 1) * G] - ref[t, h * G:(h + 1) * G])
            assert np.all(err <= lim), (h, t, float((err / lim).max()))
    r.check_layer(0)
    qa, o = r.step(0)
    r.check_out(0, qa, o, "first decode step")
    r.free()


@pytest.mark.parametrize("split", [False, True])
def test_prefill_ignores_what_lies_behind_the_last_row(split):
    """The buffer, the workspace and the partials may hold anything; the keys split
    or not."""
    D, G, n0, n = 128, 4, 650, 40
    x = {kind: up(W.normal_bf16((n0 + n, 2, D), 3, 0, kind, 0), DEV) for kind in (W.K, W.V)}
    k, v = x[W.K], x[W.V]
    q = up(W.normal_bf16((n, 2 * G, D), 3, 0, W.Q, 0), DEV)
    pol = hwkv.policy_set(1, 2, 2 * G, D, 3, [70, 0], [[0, 1]])
    outs = []
    for fill in (0x00, 0xff, 0x80):
        buf = torch.full((hwkv.cache_bytes(pol, 1, 800, "i8"),), fill, dtype=torch.uint8, device=DEV)
        cache = hwkv.cache_alloc(pol, 1, 800, dev_buf=buf, kv_format="i8")
        hwkv.prefill_write(cache, 0, 0, 0, k[:n0], v[:n0])
        ws = torch.full((hwkv.prefill_attn_workspace_bytes(cache, n),), fill, dtype=torch.uint8, device=DEV)
        size = hwkv.prefill_attn_split_bytes(cache, 0, n0, n) if split else 0
        parts = torch.full((max(size, 16),), fill, dtype=torch.uint8, device=DEV)
        out = torch.empty((n, 2 * G, D), device=DEV)
        hwkv.prefill_attn(cache, 0, 0, n0, q, k[n0:], v[n0:], 0.1, out, ws=ws, parts=parts)
        outs.append(out.cpu())
        cache.free()
    assert torch.isfinite(outs[0]).all() and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_a_released_sequence_leaves_nothing_behind():
    """Pages of a released sequence, whose rows were not finite, taken by others."""
    c = mini(batch=3, head_dim=64, prompt=[700, 300, 520], max_ctx=800)
    r = Run8(c, n_pages=3 + 2 + 3 + 1)
    for b in range(3):
        r.prefill(0, b)
    bad = torch.full((700, 2, 64), float("inf"), dtype=torch.bfloat16, device=DEV)
    hwkv.cache_reset_seq(r.cache, 0)
    hwkv.prefill_write(r.cache, 0, 0, 0, bad, bad)
    r.reset(0)
    r.prefill(0, 0, P=130)           # into the first of its pages
    r.reset(2)
    r.prefill(0, 2, P=777)           # its own, and one of those
    for st in range(2):
        qa, out = r.step(0, fused=st == 1)
        r.check_out(0, qa, out, f"step {st}")
    r.check_layer(0)
    r.free()


@pytest.mark.parametrize("batch", [2, 24])
def test_timed_steps_and_two_graphs(batch):
    """Timing events around both ways of launching, and two captured calls, of
    different layers, that share a workspace on one stream."""
    c = mini(batch=batch, n_layers=2, head_dim=64, n_q_heads=8, n_kv_heads=4, levels=[[0, 1, 1, 0], [1, 1, 0, 0]],
             prompt=[400 + 31 * i for i in range(batch)], max_ctx=1300)
    r = Run8(c)
    for layer in range(2):
        for b in range(batch):
            r.prefill(layer, b)
    q = up(W.normal_bf16((batch, 8, 64), 1, 0, W.Q, 0), DEV)
    want = [torch.empty((batch, 8, 64), device=DEV) for _ in range(2)]
    got = [torch.zeros_like(want[0]) for _ in range(2)]
    hwkv.decode_timing(r.cache, True)
    for layer in range(2):
        hwkv.decode_attn(r.cache, layer, q, r.scale, want[layer], r.ws)
    split_ms, merge_ms, launches = hwkv.decode_timing_read(r.cache)
    hwkv.decode_timing(r.cache, False)
    assert split_ms > 0 and merge_ms >= 0 and launches >= 2
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for layer, g in enumerate(graphs):
        with torch.cuda.graph(g):
            hwkv.decode_attn(r.cache, layer, q, r.scale, got[layer], r.ws)
    for i in range(3):
        q.copy_(up(W.normal_bf16((batch, 8, 64), 1, 0, W.Q, i), DEV))
        for layer in range(2):
            got[layer].zero_()
            hwkv.decode_attn(r.cache, layer, q, r.scale, want[layer], r.ws)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
    r.free()


def test_prefill_refuses_a_cache_without_workspace():
    r = Run8(mini())
    x = torch.zeros((4, 8, 64), dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(hwkv.HwkvError):
        hwkv.prefill_attn(r.cache, 0, 0, 0, x, kv, kv, 0.1, torch.empty((4, 8, 64), device=DEV))
    r.free()


@pytest.mark.parametrize("D,G", [(64, 4), (256, 6)])
def test_calibration_replay(D, G):
    """Every candidate attends over the trace as an int8 cache stores it."""
    hkv, hist, S, windows = 2, 3001, 4, [50, 700]
    rows = np.array([0, 31, 900, 1777, 2500, 3000])
    k, v = W.normal_bf16((hist, hkv, D), 6, 0, W.K, 0), W.normal_bf16((hist, hkv, D), 6, 0, W.V, 0)
    q = W.normal_bf16((len(rows), hkv * G, D), 6, 0, W.Q, 0)
    need = hwkv.calib_workspace_bytes(hkv * G, D, S, hist, len(rows), n_kv_heads=hkv, kv_format="i8")
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    outs = torch.empty((3, len(rows), hkv * G, D), device=DEV)
    scores = torch.empty((2, len(rows), hkv * G), device=DEV)
    means = torch.empty((2, hkv), device=DEV)
    scale = 1 / math.sqrt(D)
    hwkv.calib_replay(up(k, DEV), up(v, DEV), rows, up(q, DEV), windows, S, scale, outs, scores, means, ws,
                      kv_format="i8")
    kv, vv = KF.values(KF.store(k, "i8"), "i8"), KF.values(KF.store(v, "i8"), "i8")
    ref = KF.replay_outputs_values(KF.bf16_values(q), kv, vv, rows, S, windows + [0], scale)
    lim = (2.0 ** -8 + 2e-5) * np.abs(vv).max()
    assert np.abs(outs.cpu().numpy() - ref).max() <= lim
    with pytest.raises(hwkv.HwkvError):
        hwkv.calib_replay(up(k, DEV), up(v, DEV), rows, up(q, DEV), windows, S, scale, outs, scores, means, ws,
                          kv_format="i8", k_scale=1.0)
