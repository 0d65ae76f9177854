"""GPU tests of caches that move out of buffers which nobody else holds."""
import pytest
import torch

from paper_2609_02029_amd import hwkv
from test_gpu_reorder import DEV, Held, _gpu, same  # noqa: F401

pytestmark = pytest.mark.gpu


def held():
    """A cache in a buffer of torch's that only the cache refers to, and its bytes."""
    pol = hwkv.policy_set(1, 2, 2, 64, 4, [70, 0], [[0, 1]])
    need = hwkv.cache_bytes(pol, 3, 1400, "bf16", 40)
    r = Held([[0, 1]], [600, 30, 300], pages=40, dev_buf=torch.empty(need, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    return r, need


def test_on_a_stream_that_is_not_the_buffers():
    r, need = held()
    was, s = r.read(), torch.cuda.Stream()
    target = torch.empty(need, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)         # the move begins later than what follows
        hwkv.cache_move(r.cache, 40, target)
    junk = [torch.full((need,), 0xff, dtype=torch.uint8, device=DEV) for _ in range(4)]
    torch.cuda.synchronize()
    same(was, r.read())
    assert len(junk) == 4


def test_captured_and_replayed():
    r, need = held()
    was = r.read()
    target = torch.zeros(need, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hwkv.cache_move(r.cache, 40, target)
    for _ in range(3):
        target.fill_(0xff)
        junk = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)
        graph.replay()
        torch.cuda.synchronize()
        same(was, r.read())
        del junk
