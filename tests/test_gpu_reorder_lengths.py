"""GPU test of a reorder of sequences whose lengths differ from layer to layer: a layer
of windows alone may be longer than the cache's max_ctx, which bounds full units."""
import numpy as np
import pytest
import torch

from paper_2609_02029_amd import hwkv
from test_gpu_reorder import DEV, Held, _gpu, reference  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("parents", [[0] * 10, [9, 8, 7, 6, 5, 4, 3, 2, 1, 0], [1, 2, 3, 4, 5, 6, 7, 8, 9, 0],
                                     [3, 3, 3, 3, -1, 5, 5, 7, 8, 8]])
def test_layers_of_unequal_lengths(parents):
    """Stored rows follow their parents, and the kernels see the new chains (an output's
    bound: test_gpu_reorder.test_long_page_tables)."""
    B, H, max_ctx = 10, 6, 2800
    r = Held([[1] * H, [0] * H], [0] * B, max_ctx=max_ctx, pages=1000, seed=4)
    for b in range(B):
        for layer, n in ((0, max_ctx - 9 - b), (1, 9000 + b)):
            hwkv.prefill_write(r.cache, layer, b, 0, *r.rows(n))
    was = r.read()
    hwkv.cache_reorder(r.cache, parents)
    now = r.read()
    for (layer, h, b), rows in now.items():
        p = parents[b]
        assert hwkv.cache_seq_len(r.cache, layer, b) == (0 if p < 0 else (max_ctx - 9 - p, 9000 + p)[layer])
        if p >= 0:
            assert all(np.array_equal(x, y) for x, y in zip(was[layer, h, p], rows)), (layer, h, b)
    for b in range(B):                       # (decode takes no empty sequence)
        if parents[b] < 0:
            for layer in range(2):
                hwkv.prefill_write(r.cache, layer, b, 0, *r.rows(300))
    q = torch.randn((B, H, 64), generator=r.gen, device=DEV).to(torch.bfloat16)
    out = torch.empty((B, H, 64), dtype=torch.float32, device=DEV)
    ws = torch.empty(hwkv.decode_workspace_bytes(r.cache), dtype=torch.uint8, device=DEV)
    for _ in range(2):
        for layer in range(2):
            hwkv.append(r.cache, layer, *r.rows(B))
    want = torch.stack([reference(r, b, q[b]) for b in range(B)])
    for layer in range(2):
        hwkv.decode_attn(r.cache, layer, q, 0.125, out, ws)
        assert (out.cpu().double() - want[:, layer]).abs().max() < 1.4e-4
