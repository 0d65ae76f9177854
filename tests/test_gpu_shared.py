"""GPU tests of decode attention over shared pages, against 64-bit attention over
what the cache holds.

Outputs: fp32 sums over exact products, the exponentials' rounding, and weights kept
to 2^-22 or better: 2e-5 of the largest value that the row sees, the bound of the
other decode kernels' tests."""
import math

import numpy as np
import pytest
import torch

from paper_2609_02029_amd import hwkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PT = hwkv.PAGE_TOKENS


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def values(cache, layer, h, b):
    """K and V rows of a unit as 64-bit values, in slot order."""
    k, v, n = hwkv.cache_read_unit(cache, layer, h, b)
    fmt, ks, vs = hwkv.cache_format(cache)
    out = []
    for i, (x, s) in enumerate(((k[:n], ks[layer, h]), (v[:n], vs[layer, h]))):
        if fmt == "i8":
            e = hwkv.cache_read_scales(cache, layer, h, b)[i][:n].astype(np.float64)
            y = x.astype(np.float64) * np.exp2(e - 133.0)[:, None]
            y[e == 255] = np.nan
        elif fmt == "fp8":
            y = torch.from_numpy(x.copy()).view(torch.float8_e4m3fn).double().numpy() * np.float64(s)
        else:
            y = torch.from_numpy(x.copy().view(np.int16)).view(torch.float16 if fmt == "f16" else torch.bfloat16).double().numpy()
        out.append(y)
    return out


def check(cache, layer, q, scale, out, seqs=None, heads=None):
    torch.cuda.synchronize()
    G = cache.n_q_heads // cache.n_kv_heads
    q, out = q.double().cpu().numpy(), out.double().cpu().numpy()
    worst = 0.0
    for b in range(cache.batch) if seqs is None else seqs:
        for h in range(cache.n_kv_heads) if heads is None else heads:
            k, v = values(cache, layer, h, b)
            for g in range(h * G, h * G + G):
                z = (k @ q[b, g]) * scale
                p = np.exp(z - z.max())
                ref = p @ v / p.sum()
                off = np.abs(out[b, g] - ref).max() / np.abs(v).max()
                assert off <= 2e-5, (b, h, g, off)
                worst = max(worst, off)
    return worst


class Forked:
    """A cache of one layer: prompts prefilled, forked, and given tails of their own."""

    def __init__(self, D, G, prompts, tails, levels=(1, 0), book=(70, 0), S=4, fmt="bf16", paged=True, seed=0, spread=1.0,
                 max_ctx=None):
        """prompts: (length, its sequences); tails: tokens behind, per sequence."""
        self.H, self.D, self.G = len(levels), D, G
        self.B = sum(n for _, n in prompts)
        max_ctx = max_ctx or max(p for p, _ in prompts) + max(tails) + 300
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.spread = spread
        kw = dict(k_scale=0.03, v_scale=0.02) if fmt == "fp8" else {}
        pages = self.B * len(levels) * -(-max_ctx // PT) if paged else None
        self.pol = hwkv.policy_set(1, self.H, self.H * G, D, S, list(book), [list(levels)])
        self.cache = hwkv.cache_alloc(self.pol, self.B, max_ctx, kv_format=fmt, n_pages=pages, **kw)
        parents, b = [], 0
        for n, count in prompts:
            hwkv.prefill_write(self.cache, 0, b, 0, *self.rows(n))
            parents += [b] * count
            b += count
        hwkv.cache_reorder(self.cache, parents)
        for b, t in enumerate(tails):
            self.write(b, t)
        self.ws = torch.full((hwkv.decode_shared_workspace_bytes(self.cache),), 0xff, dtype=torch.uint8, device=DEV)
        self.q = torch.randn((self.B, self.H * G, D), generator=self.gen, device=DEV).to(torch.bfloat16)
        self.scale = 1 / math.sqrt(D)

    def rows(self, n):
        return [(torch.randn((n, self.H, self.D), generator=self.gen, device=DEV) * self.spread).to(torch.bfloat16) for _ in range(2)]

    def write(self, b, n):
        if n:
            hwkv.prefill_write(self.cache, 0, b, hwkv.cache_seq_len(self.cache, 0, b), *self.rows(n))

    def run(self, q=None, **kw):
        q = self.q if q is None else q
        out = torch.full(q.shape, float("nan"), device=DEV)
        hwkv.decode_attn_shared(self.cache, 0, q, self.scale, out, self.ws, **kw)
        return out

    def check(self, **kw):
        return check(self.cache, 0, self.q, self.scale, self.run(), **kw)


@pytest.mark.parametrize("fmt", ["bf16", "f16", "fp8", "i8"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("G", [1, 2, 4, 6, 8])
def test_every_head_dim_group_and_format(fmt, D, G):
    for prompts, tails in ((((700, 2),), (9, 300)), (((1200, 9), (300, 3), (5, 1)), [1, 0, 70, 255, 256, 2, 3, 4, 513, 0, 1, 2, 60])):
        Forked(D, G, prompts, tails, fmt=fmt, seed=D + G).check()


@pytest.mark.parametrize("fmt", ["bf16", "i8"])
def test_many_samples_of_one_prompt(fmt):
    """More columns than a block has, tails that are empty, or whole pages; more
    sequences than a launch takes."""
    Forked(128, 8, ((1024, 20),), [i % 3 * 128 for i in range(20)], fmt=fmt).check()
    Forked(64, 1, ((800, 100), (300, 30)), [i % 5 for i in range(130)], fmt=fmt).check()
    Forked(64, 4, ((512, 17), (512, 17)), [0] * 34, fmt=fmt).check()


def test_nothing_is_shared():
    """Unpaged caches, sequences of their own, a batch of one, lengths from one token."""
    Forked(128, 4, ((300, 2), (1, 1), (64, 1)), [3, 4, 0, 1], paged=False).check()
    Forked(64, 2, tuple((n, 1) for n in (1, 2, 63, 64, 65, 255, 256, 257)), [0] * 8).check()
    Forked(256, 6, ((4000, 1),), [1]).check()
    Forked(64, 8, ((1, 1),), [0]).check()


def test_windows_alone_and_many_heads():
    Forked(64, 2, ((500, 4),), [1, 2, 3, 4], levels=(0, 0, 0), book=(70, 0)).check()
    Forked(64, 1, ((400, 3),), [1, 2, 3], levels=[i % 2 for i in range(40)]).check()


def test_long_shared_prompts():
    """Several tiles for every workgroup, and as many parts to merge."""
    r = Forked(256, 6, ((40000, 8),), [17 * i for i in range(8)], levels=(2, 0, 1), book=(2048, 8192, 0)[0:2] + (0,))
    assert r.check(seqs=(0, 7)) < 5e-6
    r = Forked(128, 4, ((20000, 4), (9000, 4)), [100 * i for i in range(8)], fmt="f16")
    r.check(seqs=(0, 3, 4, 7))


@pytest.mark.parametrize("count,G", [(2, 4), (6, 8)])
def test_many_tiles_a_workgroup(count, G):
    """More than the 64 tiles whose pages a workgroup looks up at once, in workgroups of
    one column group and of three."""
    r = Forked(64, G, ((70000, count),), [9 * i for i in range(count)], levels=(1,) * 32, max_ctx=70200)
    r.check(seqs=(0, count - 1), heads=(0, 13, 31))


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_blocks_of_unequal_widths(fmt):
    """Blocks of one to five column groups in one launch, beside sequences of none."""
    Forked(64, 8, ((600, 10), (300, 2), (512, 5), (260, 3), (90, 2), (1024, 1)), [3 * i for i in range(23)], fmt=fmt).check()
    Forked(128, 1, ((600, 50), (300, 17), (256, 2)), [i % 4 for i in range(69)], fmt=fmt).check()


def test_families_within_a_prompt():
    """Forks of forks: a short prefix that all share and longer ones that some do;
    sequences that were moved and dropped; a moved cache."""
    r = Forked(64, 4, ((300, 8),), [0, 600, 0, 0, 700, 0, 0, 20])
    hwkv.cache_reorder(r.cache, [0, 1, 1, 1, 4, 4, 6, 7])
    for b in range(8):
        r.write(b, 5 + b)
    r.check()
    hwkv.cache_reorder(r.cache, [4, 1, 5, 1, 0, 6, 3, 2])
    r.check()
    hwkv.cache_move(r.cache, 60)
    r.check()
    hwkv.cache_reset_seq(r.cache, 3)
    hwkv.prefill_write(r.cache, 0, 3, 0, *r.rows(77))
    r.check()


def test_as_decode_attn_and_equal_bits():
    """The same attention as decode_attn's, from run to run with the same bits, and
    whether the pages are shared or not."""
    for fmt in ("bf16", "f16", "fp8", "i8"):
        r = Forked(128, 4, ((3000, 6),), [11 * i for i in range(6)], fmt=fmt)
        first = r.run()
        other = torch.empty_like(first)
        hwkv.decode_attn(r.cache, 0, r.q, r.scale, other, torch.empty(hwkv.decode_workspace_bytes(r.cache), dtype=torch.uint8, device=DEV))
        # (each within 2e-5 of the largest value, about 5)
        assert (first - other).abs().max() <= 2e-4
        for _ in range(3):
            assert torch.equal(first, r.run())


def test_logits_and_values_of_any_size():
    """Near one-hot weights, large and small queries, logits far below zero, a scale of
    zero and a negative one."""
    for fmt in ("bf16", "f16", "fp8", "i8"):
        r = Forked(64, 2, ((600, 3),), [1, 2, 3], fmt=fmt)
        for factor, scale in ((50.0, 0.125), (2.0 ** -20, 0.125), (1.0, 0.0), (1.0, -0.5), (1.0, 300.0)):
            r.q, r.scale = (r.q.float() * factor).to(torch.bfloat16), scale
            # (logits of thousands: an fp32 sum's error, 2^-22 of them, moves the weights by as much)
            if factor * abs(scale) < 10:
                r.check()
            else:
                assert torch.isfinite(r.run()).all()
            r.q = torch.randn(r.q.shape, generator=r.gen, device=DEV).to(torch.bfloat16)
    r = Forked(128, 4, ((600, 3),), [1, 2, 3], spread=2.0 ** 30)
    r.q, r.scale = (r.q.float() * 2.0 ** -40).to(torch.bfloat16), 1.0
    r.check()


@pytest.mark.parametrize("fmt", ["bf16", "f16", "i8"])
def test_a_row_that_is_not_finite_reaches_only_those_that_see_it(fmt):
    r = Forked(64, 2, ((512, 3), (300, 1)), [0, 0, 0, 0], fmt=fmt, levels=(1, 1))
    k, v = r.rows(10)
    v[4, 0, 7] = torch.inf
    hwkv.prefill_write(r.cache, 0, 1, 512, k, v)
    for b in (0, 2, 3):
        r.write(b, 3)
    out = r.run()
    bad = ~torch.isfinite(out)
    assert bad[1, :2].any() and not bad[1, 2:].any() and not bad[[0, 2, 3]].any()
    keep = [0, 2, 3]
    check(r.cache, 0, r.q, r.scale, out, seqs=keep)


def test_junk_behind_the_last_row_is_not_seen():
    """Pages and regions are full of NaN before they are written."""
    for fmt in ("bf16", "f16", "fp8", "i8"):
        D, G, B = 128, 2, 3
        pol = hwkv.policy_set(1, 2, 2 * G, D, 4, [70, 0], [[0, 1]])
        n = hwkv.cache_bytes(pol, B, 900, fmt, 12)
        buf = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
        kw = dict(k_scale=0.03, v_scale=0.02) if fmt == "fp8" else {}
        cache = hwkv.cache_alloc(pol, B, 900, dev_buf=buf, kv_format=fmt, n_pages=12, **kw)
        g = torch.Generator(device=DEV).manual_seed(4)
        rows = lambda n: [torch.randn((n, 2, D), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2)]   # noqa: E731
        hwkv.prefill_write(cache, 0, 0, 0, *rows(290))
        hwkv.cache_reorder(cache, [0, 0, 0])
        for b in range(B):
            hwkv.prefill_write(cache, 0, b, 290, *rows(1 + 40 * b))
        q = torch.randn((B, 2 * G, D), generator=g, device=DEV).to(torch.bfloat16)
        out = torch.full(q.shape, float("nan"), device=DEV)
        ws = torch.full((hwkv.decode_shared_workspace_bytes(cache),), 0xff, dtype=torch.uint8, device=DEV)
        hwkv.decode_attn_shared(cache, 0, q, 0.1, out, ws)
        check(cache, 0, q, 0.1, out)


def test_captured_on_another_stream_and_a_shared_workspace():
    r = Forked(128, 4, ((1500, 4), (700, 2)), [9, 8, 7, 6, 5, 4])
    o = Forked(64, 2, ((900, 3),), [30, 20, 10], fmt="i8", seed=3)
    ws = torch.full((max(r.ws.numel(), o.ws.numel()),), 0xff, dtype=torch.uint8, device=DEV)
    r.ws = o.ws = ws
    want = [x.run().clone() for x in (r, o)]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = r.run()
    s.synchronize()
    assert torch.equal(got, want[0])
    graphs, outs = [], [torch.empty_like(w) for w in want]
    for x, out in zip((r, o), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            hwkv.decode_attn_shared(x.cache, 0, x.q, x.scale, out, ws)
        graphs.append(g)
    for turn in range(4):
        for x, out, w, g in zip((r, o), outs, want, graphs):
            x.q.copy_(x.q.roll(1, 0))
            out.fill_(7.0)
            g.replay()
        for x, out in zip((r, o), outs):
            torch.cuda.synchronize()
            assert torch.equal(out, x.run())
            check(x.cache, 0, x.q, x.scale, out)


def test_refusals():
    r = Forked(64, 2, ((300, 2),), [1, 2])
    out = torch.empty(r.q.shape, device=DEV)
    with pytest.raises(hwkv.HwkvError, match="workspace"):
        hwkv.decode_attn_shared(r.cache, 0, r.q, 0.1, out, r.ws[:64])
    with pytest.raises(hwkv.HwkvError, match="layer"):
        hwkv.decode_attn_shared(r.cache, 1, r.q, 0.1, out, r.ws)
    with pytest.raises(hwkv.HwkvError, match="finite"):
        hwkv.decode_attn_shared(r.cache, 0, r.q, math.inf, out, r.ws)
    with pytest.raises(hwkv.HwkvError, match="aligned"):
        hwkv.decode_attn_shared(r.cache, 0, r.q, 0.1, out, torch.empty(r.ws.numel() + 8, dtype=torch.uint8, device=DEV)[8:])
    with pytest.raises(ValueError, match="batch"):
        hwkv.decode_attn_shared(r.cache, 0, r.q[:1], 0.1, out[:1], r.ws)
    hwkv.cache_reset_seq(r.cache, 0)
    with pytest.raises(hwkv.HwkvError, match="empty"):
        hwkv.decode_attn_shared(r.cache, 0, r.q, 0.1, out, r.ws)
