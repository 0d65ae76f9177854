"""GPU test of random runs of calls on one cache (chunks, appends, forks, permutations,
drops, resets and moves, over a pool that runs out at times) against a list of the rows
that each sequence should hold: stored bits, pages, and decoding through the device's
page table.  Bounds of outputs: test_gpu_shared."""
import random

import pytest
import torch

from paper_2609_02029_amd import hwkv
from test_gpu_shared import DEV, _gpu, check  # noqa: F401

pytestmark = pytest.mark.gpu
PT = hwkv.PAGE_TOKENS


class Walk:
    def __init__(self, seed, D, G, levels, fmt, B, max_ctx, pages, S=3, w=50):
        self.rng, self.D, self.L, self.H, self.B, self.S, self.w = random.Random(seed), D, len(levels), len(levels[0]), B, S, w
        self.levels, self.max_ctx, self.pages, self.fmt = levels, max_ctx, pages, fmt
        self.full = sum(x == 1 for row in levels for x in row)
        self.pol = hwkv.policy_set(self.L, self.H, self.H * G, D, S, [w, 0], levels)
        self.cache = hwkv.cache_alloc(self.pol, B, max_ctx, kv_format=fmt, n_pages=pages)
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.G = G
        # per sequence: k and v rows [tokens][layers][heads][D], and the names of its pages
        self.k = [torch.empty((0, self.L, self.H, D), dtype=torch.bfloat16, device=DEV) for _ in range(B)]
        self.v = [x.clone() for x in self.k]
        self.chain, self.names = [[] for _ in range(B)], 0

    def rows(self, n):
        return [torch.randn((n, self.L, self.H, self.D), generator=self.gen, device=DEV).to(torch.bfloat16) for _ in range(2)]

    def used(self, chains):
        return self.full * len({p for c in chains for p in c})

    def grown(self, b, n):
        chain = list(self.chain[b])
        while len(chain) < -(-n // PT):
            self.names += 1
            chain.append(self.names)
        return chain

    def chunk(self):
        b, n = self.rng.randrange(self.B), self.rng.choice([1, 5, 70, 256, 300, 600])
        n = min(n, self.max_ctx - len(self.k[b]))
        chain = self.grown(b, len(self.k[b]) + n)
        if n == 0 or self.used(self.chain[:b] + [chain] + self.chain[b + 1:]) > self.pages:
            return
        k, v = self.rows(n)
        for layer in range(self.L):
            hwkv.prefill_write(self.cache, layer, b, len(self.k[b]), k[:, layer].contiguous(), v[:, layer].contiguous())
        self.k[b], self.v[b], self.chain[b] = torch.cat([self.k[b], k]), torch.cat([self.v[b], v]), chain

    def append(self):
        if any(len(x) == self.max_ctx for x in self.k):
            return
        chains = [self.grown(b, len(self.k[b]) + 1) for b in range(self.B)]
        if self.used(chains) > self.pages:
            return
        k, v = self.rows(self.B)
        for layer in range(self.L):
            hwkv.append(self.cache, layer, k[:, layer].contiguous(), v[:, layer].contiguous())
        for b in range(self.B):
            self.k[b], self.v[b] = torch.cat([self.k[b], k[b:b + 1]]), torch.cat([self.v[b], v[b:b + 1]])
        self.chain = chains

    def reorder(self):
        B, r = self.B, self.rng
        how = r.randrange(4)
        parents = list(range(B))
        if how == 0:
            r.shuffle(parents)
        elif how == 1:
            parents = [r.randrange(-1, B) for _ in range(B)]
        elif how == 2:
            for _ in range(r.randint(1, 3)):
                parents[r.randrange(B)] = r.randrange(B)
        else:
            ring = r.sample(range(B), r.randint(2, B))
            for x, y in zip(ring, ring[1:] + ring[:1]):
                parents[x] = y
        chains, kept = [], set()
        heir = {p: p if parents[p] == p else parents.index(p) for p in parents if p >= 0}
        for b, p in enumerate(parents):
            chain = [] if p < 0 else list(self.chain[p])
            if p >= 0 and len(self.k[p]) % PT and heir[p] != b:
                self.names += 1
                chain[-1] = self.names
            chains.append(chain)
            kept.add(p)
        if self.used(chains) > self.pages:
            with pytest.raises(hwkv.HwkvError, match="pages needed"):
                hwkv.cache_reorder(self.cache, parents)
            return
        hwkv.cache_reorder(self.cache, parents)
        self.chain = chains
        self.k = [self.k[p] if p >= 0 else self.k[0][:0] for p in parents]
        self.v = [self.v[p] if p >= 0 else self.v[0][:0] for p in parents]

    def reset(self):
        b = self.rng.randrange(self.B)
        hwkv.cache_reset_seq(self.cache, b)
        self.k[b], self.v[b], self.chain[b] = self.k[b][:0], self.v[b][:0], []

    def move(self):
        used = self.used(self.chain)
        pages = self.rng.choice([used + 3, used + 40, used + 200])
        buf = None
        if self.rng.random() < 0.5:
            buf = torch.full((hwkv.cache_bytes(self.pol, self.B, self.max_ctx, self.fmt, pages),), 0xff, dtype=torch.uint8, device=DEV)
        if used > 0:
            with pytest.raises(hwkv.HwkvError, match="pages in use"):
                hwkv.cache_move(self.cache, used - 1, buf)
        hwkv.cache_move(self.cache, pages, buf)
        self.pages = pages

    def check(self):
        assert hwkv.cache_pages(self.cache) == (self.pages, self.pages - self.used(self.chain))
        for b in range(self.B):
            n = len(self.k[b])
            for layer in range(self.L):
                assert hwkv.cache_seq_len(self.cache, layer, b) == n
                for h in range(self.H):
                    at = list(range(n))
                    if self.levels[layer][h] == 0:
                        at = at[:self.S] + at[max(self.S, n - self.w):]
                        at.sort(key=lambda p: p if p < self.S else self.S + (p - self.S) % self.w)
                    k, v, held = hwkv.cache_read_unit(self.cache, layer, h, b)
                    assert held == len(at)
                    if self.fmt != "bf16":
                        continue
                    for x, y in ((k, self.k), (v, self.v)):
                        x = torch.from_numpy(x[:held].astype("int32")).to(torch.int16)
                        assert torch.equal(x, y[b][at, layer, h].view(torch.int16).cpu()), (b, layer, h)
        live = [b for b in range(self.B) if len(self.k[b])]
        if len(live) < self.B:
            return
        q = torch.randn((self.B, self.H * self.G, self.D), generator=self.gen, device=DEV).to(torch.bfloat16)
        for call, size in ((hwkv.decode_attn, hwkv.decode_workspace_bytes),
                           (hwkv.decode_attn_shared, hwkv.decode_shared_workspace_bytes)):
            ws = torch.full((size(self.cache),), 0xff, dtype=torch.uint8, device=DEV)
            for layer in range(self.L):
                out = torch.full(q.shape, float("nan"), device=DEV)
                call(self.cache, layer, q, self.D ** -0.5, out, ws)
                check(self.cache, layer, q, self.D ** -0.5, out, seqs=self.rng.sample(live, 4))


@pytest.mark.parametrize("seed,D,G,fmt", [(1, 64, 1, "bf16"), (2, 64, 4, "bf16"), (3, 128, 2, "i8"), (4, 128, 8, "fp8"), (5, 64, 6, "f16")])
def test_a_random_run(seed, D, G, fmt):
    r = Walk(seed, D, G, [[0, 1, 1], [1, 0, 1]], fmt, 23, 2000, 4 * 60)
    for step in range(160):
        r.rng.choice([r.chunk, r.chunk, r.append, r.append, r.reorder, r.reorder, r.reorder, r.reset if step % 3 == 0 else r.append,
                      r.move if step % 2 == 0 else r.chunk])()
        if step % 8 == 7:
            for b in range(r.B):               # (decode takes no empty sequence)
                if len(r.k[b]) == 0 and r.used(r.chain) + r.full <= r.pages:
                    k, v = r.rows(9)
                    for layer in range(r.L):
                        hwkv.prefill_write(r.cache, layer, b, 0, k[:, layer].contiguous(), v[:, layer].contiguous())
                    r.k[b], r.v[b], r.chain[b] = k, v, r.grown(b, 9)
            r.check()
