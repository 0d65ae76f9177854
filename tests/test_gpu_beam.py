"""GPU tests of beam selection against scores formed in 64 bits on the host.

Scores are 64-bit sums rounded once to fp32: off by half a step, 2^-24 of the
value, by the error of lse (5.5e-11 a term, so at most 1e-10 in all), and in rows far
from zero by the reference's own rounding of lse (half a step of 2^-52 of it, and as
much again in x - lse)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_02029_amd import hwkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)


def reference(x, s, n):
    """(scores in 64 bits, parents, tokens) of logits x [groups, beams, vocab]
    and running scores s, numpy float64."""
    G, B, V = x.shape
    val = np.full((G, n), -np.inf)
    par, tok = np.full((G, n), -1), np.full((G, n), -1)
    for g in range(G):
        sc = np.full((B, V), -np.inf)
        for b in range(B):
            row = x[g, b]
            if not np.isfinite(s[g, b]) or np.isnan(row).any() or (row == np.inf).any() or row.max() == -np.inf:
                continue
            top = row.max()
            lse = top + np.log(np.exp(row - top).sum())
            sc[b] = s[g, b] + (row - lse)
        flat = sc.ravel()
        order = np.argsort(-flat, kind="stable")[:n]
        order = order[flat[order] > -np.inf]
        val[g, :len(order)] = flat[order]
        par[g, :len(order)] = g * B + order // V
        tok[g, :len(order)] = order % V
    return val, par, tok


def outputs(G, n):
    return (torch.full((G, n), 7.0, device=DEV), torch.full((G, n), 7, dtype=torch.int32, device=DEV),
            torch.full((G, n), 7, dtype=torch.int32, device=DEV))


def select(x, s, n, **kw):
    out = outputs(x.shape[0], n)
    ws = torch.full((hwkv.beam_workspace_bytes(x, n),), 0xff, dtype=torch.uint8, device=DEV)
    hwkv.beam_select(x, s, *out, ws, **kw)
    return out


def check(out, x, s, n):
    torch.cuda.synchronize()
    val, par, tok = reference(x.double().cpu().numpy(), s.double().cpu().numpy(), n)
    got = [t.cpu().numpy() for t in out]
    assert np.array_equal(got[1], par) and np.array_equal(got[2], tok)
    some = par >= 0
    assert np.array_equal(got[0] == -np.inf, ~some)
    ref = val[some]
    far = np.nan_to_num(np.abs(x.double().cpu().numpy()), posinf=0.0, neginf=0.0).max()
    assert np.all(np.abs(got[0][some] - ref) <= 2.0 ** -24 * np.abs(ref) + 1e-10 + 2.0 ** -52 * far)


def inputs(G, B, V, t, seed=0, spread=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed + V)
    x = (torch.randn((G, B, V), generator=g, device=DEV) * spread).to(TYPES[t])
    return x, -torch.rand((G, B), generator=g, device=DEV) * 9


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 255, 256, 257, 511, 512, 513, 2049, 16385, 50257])
def test_sizes(t, V):
    for G, B, n in ((1, 1, 1), (2, 3, 6), (1, 4, 64), (3, 5, 10)):
        x, s = inputs(G, B, V, t)
        check(select(x, s, n), x, s, n)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_many_beams_and_groups(t):
    for G, B, V, n in ((70, 4, 3001, 8), (1, 64, 40001, 64), (300, 8, 130, 16), (1, 1, 600001, 5),
                       (2, 16, 1100, 30), (9, 16, 1500, 64), (3, 8, 1000, 16)):
        x, s = inputs(G, B, V, t, seed=3)
        check(select(x, s, n), x, s, n)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_more_blocks_than_fit_a_workgroup(t):
    """Searches whose maxima stay in memory, also where they are all alike."""
    G, B, V, n = 1, 5, (1 << 22) + 3, 20
    x, s = inputs(G, B, V, t, seed=6)
    check(select(x, s, n), x, s, n)
    x.fill_(0.5)
    x[0, 3, 4000000:] = 0.75
    out = select(x, s.zero_(), n)
    lse = [math.log(V) + 0.5] * 5
    lse[3] = math.log(4000000 * math.exp(0.5) + (V - 4000000) * math.exp(0.75))
    assert out[1].tolist() == [[3] * n] and out[2].tolist() == [list(range(4000000, 4000000 + n))]
    assert (out[0].double() - (0.75 - lse[3])).abs().max() < 2.0 ** -20    # fp32 of about 15
    x.fill_(0.5)                                  # every score is -log V
    out = select(x, s, n)
    assert out[1].tolist() == [[0] * n] and out[2].tolist() == [list(range(n))]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_rows_apart_and_anywhere(t):
    """Rows of an odd length, apart, and starting at every element of 16 bytes;
    what lies between them is not read."""
    G, B, V = 2, 3, 4099
    x, s = inputs(G, B, V, t)
    for stride, at in ((V + 5, 1), (V + 1, 2), (V, 3), (V + 2, 5), (V + 3, 7)):
        buf = torch.full((at + G * B * stride,), float("nan"), dtype=TYPES[t], device=DEV)
        rows = buf[at:].view(G, B, stride)[:, :, :V]
        rows.copy_(x)
        assert rows.data_ptr() % 16 or at == 0
        check(select(rows, s, 8), x, s, 8)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_ties_go_to_the_lowest(t):
    V = 5003
    x = torch.zeros((2, 3, V), dtype=TYPES[t], device=DEV)
    s = torch.zeros((2, 3), device=DEV)
    out = select(x, s, 20)                        # every score is -log V
    check(out, x, s, 20)
    assert out[1].tolist() == [[0] * 20, [3] * 20] and out[2].tolist() == [list(range(20))] * 2
    s[:, 0] = -1.0
    x[1, 2, 77], x[1, 1, 4000] = 3.0, 3.0         # equal rows but for the places of their largest
    check(select(x, s, 64), x, s, 64)
    few = torch.randint(0, 4, (2, 4, V), device=DEV).to(TYPES[t])   # long runs of ties
    s = torch.tensor([[0.0, 0.0, -1.0, 0.0]] * 2, device=DEV)
    few[:, 1] = few[:, 0]
    check(select(few, s, 33), few, s, 33)


def test_rising_logits():
    """The n largest lie in one block, and whole blocks above the next ones'."""
    for V in (700, 9000, 66000):
        x = (torch.arange(V, device=DEV, dtype=torch.float32) / 1024).repeat(1, 3, 1)
        s = torch.tensor([[0.0, -0.25, 0.125]], device=DEV)
        check(select(x, s, 64), x, s, 64)
        check(select(-x, s, 64), -x, s, 64)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_masked_logits(t):
    G, B, V, n = 4, 4, 3001, 9
    x, s = inputs(G, B, V, t, seed=8)
    x[torch.rand(x.shape, device=DEV) < 0.99] = -torch.inf
    x[0] = -torch.inf                             # nothing is allowed
    x[1] = -torch.inf
    x[1, 2, 2999], x[1, 3, 5] = -4.0, 2.0         # two are
    x[2, :3] = -torch.inf                         # one beam
    s[3, :] = -torch.inf
    s[3, 2] = 0.0                                 # a first step: one beam is alive
    out = select(x, s, n)
    check(out, x, s, n)
    # (a row's only token has the probability 1, so that its score is the row's own)
    by = [6, 7] if s[1, 2] >= s[1, 3] else [7, 6]
    assert out[1][0].tolist() == [-1] * n and out[1][1].tolist() == by + [-1] * 7


def test_rows_without_a_sum():
    """A NaN or +infinity takes its row out, and no other; so does a score that is
    not finite."""
    x, s = inputs(1, 8, 2777, "f32", seed=4)
    x[0, 1, 2776] = torch.nan
    x[0, 2, 0] = torch.inf
    x[0, 3, 100], x[0, 3, 101] = torch.inf, -torch.inf
    s[0, 4], s[0, 5], s[0, 6] = torch.nan, torch.inf, -torch.inf
    out = select(x, s, 40)
    check(out, x, s, 40)
    assert set(out[1].flatten().tolist()) <= {0, 7}
    y = x.to(torch.bfloat16)
    check(select(y, s, 40), y, s, 40)


def test_logits_of_any_magnitude():
    """Sums whose terms lie far apart, and rows far from zero (a row's logits all
    lie within fp32's range; scores are then large, and their order is by them)."""
    V = 2100
    g = torch.Generator(device=DEV).manual_seed(2)
    base = torch.randn((1, 1, V), generator=g, device=DEV)
    for shift, spread in ((0.0, 300.0), (1e6, 1.0), (-1e6, 5.0), (3e7, 64.0), (1e30, 1e28), (-1e30, 1e28), (0.0, 1e37),
                          (0.0, 1e-30)):
        x = (base * spread + shift).repeat(1, 2, 1)
        x[0, 1] = x[0, 1].flip(0)
        s = torch.tensor([[0.0, -0.5]], device=DEV)
        check(select(x, s, 12), x, s, 12)
    # one logit far above the blocks before it, and far below
    x = base.clone() * 2
    x[0, 0, 2050], x[0, 0, 700] = 5000.0, -3e38
    check(select(x, torch.zeros((1, 1), device=DEV), 6), x, torch.zeros((1, 1), device=DEV), 6)
    x = base.clone() - 3e6
    x[0, 0, 1500] = 10.0
    check(select(x, torch.zeros((1, 1), device=DEV), 6), x, torch.zeros((1, 1), device=DEV), 6)


def test_the_order_is_that_of_64_bits():
    """Two beams with the same largest logit, whose running scores differ by what
    their sums do, but for 1e-9: fp32 sums could not tell them apart."""
    V = 40000
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn((1, 2, V), generator=g, device=DEV)
    x[0, :, 11] = 30.0                            # (its share of the sum is near 1: lse is near 30)
    lse = torch.logsumexp(x.double(), dim=2)
    d = (lse[0, 1] - lse[0, 0]).item()
    for eps in (1e-9, -1e-9):
        s = torch.tensor([[0.0, d + eps]], device=DEV)          # |d| is small: fp32 holds it to 1e-15
        check(select(x, s, 4), x, s, 4)


def test_nothing_else_is_written():
    x, s = inputs(2, 2, 999, "bf16")
    n = 5
    ws = torch.full((hwkv.beam_workspace_bytes(x, n) + 64,), 0x5a, dtype=torch.uint8, device=DEV)
    bufs = [torch.full((2 * n + 8,), 7, dtype=d, device=DEV) for d in (torch.float32, torch.int32, torch.int32)]
    hwkv.beam_select(x, s, *(b[4:4 + 2 * n].view(2, n) for b in bufs), ws[:-64])
    check([b[4:4 + 2 * n].view(2, n) for b in bufs], x, s, n)
    assert all((b[:4] == 7).all() and (b[-4:] == 7).all() for b in bufs) and (ws[-64:] == 0x5a).all()
    empty = torch.empty((0, 2, 999), dtype=torch.bfloat16, device=DEV)
    hwkv.beam_select(empty, torch.empty((0, 2), device=DEV), *outputs(0, n), ws)


def test_captured_and_on_two_streams():
    """Two captured selections that share a workspace, replayed in turn, and two
    selections at once on streams of their own."""
    sets = [inputs(3, 4, 20011, t, seed=9 + i) for i, t in enumerate(("bf16", "f32"))]
    ws = torch.empty(max(hwkv.beam_workspace_bytes(x, 8) for x, _ in sets), dtype=torch.uint8, device=DEV)
    outs, graphs = [outputs(3, 8) for _ in sets], []
    torch.cuda.synchronize()
    for (x, s), out in zip(sets, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            hwkv.beam_select(x, s, *out, ws)
        graphs.append(g)
    for turn in range(4):
        for (x, s), out, g in zip(sets, outs, graphs):
            x.copy_(x.roll(turn + 1, 2))
            s.sub_(0.5 * turn)
            out[1].fill_(7)
            g.replay()
        for (x, s), out in zip(sets, outs):
            check(out, x, s, 8)
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for (x, s), st in zip(sets, streams):
        with torch.cuda.stream(st):
            got.append([select(x, s, 8) for _ in range(5)])
    torch.cuda.synchronize()
    for (x, s), outs in zip(sets, got):
        for out in outs:
            check(out, x, s, 8)


def test_equal_calls_give_equal_bits():
    x, s = inputs(8, 4, 70001, "f16", seed=5)
    first = [t.clone() for t in select(x, s, 16)]
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, select(x, s, 16)))
