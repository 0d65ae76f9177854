"""CPU tests of beam selection, reordering and moving: every refusal that comes
before device work, over device pointers that are never dereferenced."""
import ctypes

import pytest

FAKE = 0x7f0000000000


@pytest.fixture(scope="module")
def hw():
    from paper_2609_02029_amd import hwkv
    return hwkv


@pytest.fixture(scope="module")
def cache(hw):
    pol = hw.policy_set(2, 2, 4, 64, 4, [128, 0], [[0, 1], [1, 1]])
    h = ctypes.c_void_p()
    assert hw._lib.hwkv_cache_alloc_paged(ctypes.byref(h), pol.handle, 3, 1000, 0, None, None, 10, FAKE, 1 << 40) == hw.OK
    return hw.Cache(h, 2, 2, 4, 64, 3)


def select(hw, groups=2, beams=3, vocab=1000, logits=FAKE, type=0, stride=1000, scores=FAKE + (1 << 30), n_out=6,
           outs=(FAKE + (2 << 30), FAKE + (3 << 30), FAKE + (4 << 30)), ws=FAKE + (5 << 30), ws_bytes=1 << 30):
    return hw._lib.hwkv_beam_select(groups, beams, vocab, logits, type, stride, scores, n_out, *outs, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [
    dict(beams=0), dict(beams=65), dict(n_out=0), dict(n_out=65), dict(vocab=0), dict(vocab=(1 << 24) + 1, stride=1 << 25),
    dict(groups=-1), dict(groups=(1 << 20) // 3 + 1), dict(type=3), dict(type=-1), dict(logits=None), dict(scores=None),
    dict(outs=(None, FAKE, FAKE)), dict(outs=(FAKE + (2 << 30), None, FAKE + (4 << 30))),
    dict(outs=(FAKE + (2 << 30), FAKE + (3 << 30), None)), dict(stride=999), dict(stride=(1 << 31) + 1),
    dict(logits=FAKE + 1), dict(type=2, logits=FAKE + 2), dict(scores=FAKE + (1 << 30) + 2), dict(ws=None), dict(ws_bytes=8),
    dict(ws=FAKE + (5 << 30) + 8), dict(outs=(FAKE + 400, FAKE + (3 << 30), FAKE + (4 << 30))),
    dict(outs=(FAKE + (2 << 30), FAKE + (2 << 30) + 44, FAKE + (4 << 30))), dict(ws=FAKE + 64, ws_bytes=1 << 20),
    dict(scores=FAKE + (2 << 30) + 16),
])
def test_selection_refuses(hw, bad):
    assert select(hw, **bad) == hw.EINVAL and hw.last_error()


def test_selection_of_no_groups_and_its_workspace(hw):
    assert select(hw, groups=0, logits=None, ws=None) == hw.OK
    n = ctypes.c_size_t()
    f = hw._lib.hwkv_beam_workspace_bytes
    assert f(1, 4, 32000, 0, 8, ctypes.byref(n)) == hw.OK
    # 63 blocks of 512 logits: 16 workgroups a row with 16 bytes, and 4 bytes a block (and
    # one more, whole fours)
    assert n.value == 4 * (16 * 16 + 64 * 4)
    assert f(0, 4, 32000, 0, 8, ctypes.byref(n)) == hw.OK and n.value == 0
    assert f(1, 4, 32000, 0, 8, None) == hw.EINVAL
    assert f(1, 4, 32000, 7, 8, ctypes.byref(n)) == hw.EINVAL
    assert f(1, 0, 32000, 0, 8, ctypes.byref(n)) == hw.EINVAL


def test_binding_refuses_shapes(hw):
    import torch
    x = torch.zeros((2, 3, 9))
    with pytest.raises(ValueError, match="device"):
        hw.beam_workspace_bytes(x, 4)


def test_reorder_refuses(hw, cache):
    f = hw._lib.hwkv_cache_reorder
    arr = lambda *p: (ctypes.c_int32 * 3)(*p)   # noqa: E731
    assert f(None, arr(0, 1, 2), None) == hw.EINVAL
    assert f(cache.handle, None, None) == hw.EINVAL
    for bad in ((0, 1, 3), (-2, 1, 2), (0, 1 << 30, 2)):
        assert f(cache.handle, arr(*bad), None) == hw.EINVAL
    assert f(cache.handle, arr(0, 1, 2), None) == hw.OK           # nothing to do
    with pytest.raises(ValueError, match="per sequence"):
        hw.cache_reorder(cache, [0, 1], stream=0)
    # empty sequences: host bookkeeping alone
    hw.cache_reorder(cache, [2, -1, 0], stream=0)
    assert [hw.cache_seq_len(cache, 1, b) for b in range(3)] == [0, 0, 0]
    assert hw.cache_pages(cache) == (10, 10)


def test_reorder_refuses_a_long_cycle(hw):
    pol = hw.policy_set(1, 1, 1, 64, 0, [16], [[0]])
    h = ctypes.c_void_p()
    assert hw._lib.hwkv_cache_alloc_format(ctypes.byref(h), pol.handle, 300, 64, 0, None, None, FAKE, 1 << 40) == hw.OK
    ring = list(range(1, 192)) + [0] + list(range(192, 300))
    assert hw._lib.hwkv_cache_reorder(h, (ctypes.c_int32 * 300)(*ring), None) == hw.EINVAL
    assert "cycle of 192" in hw.last_error()
    hw._lib.hwkv_cache_free(h)


def test_move_refuses(hw, cache):
    f = hw._lib.hwkv_cache_move
    need = hw.cache_bytes(hw.policy_set(2, 2, 4, 64, 4, [128, 0], [[0, 1], [1, 1]]), 3, 1000, "bf16", 20)
    there = FAKE + (1 << 41)
    assert f(None, 20, there, need, None) == hw.EINVAL
    assert f(cache.handle, -1, there, need, None) == hw.EINVAL
    assert f(cache.handle, 20, there, need - 1, None) == hw.ENOMEM
    assert f(cache.handle, 20, there + 8, need, None) == hw.EINVAL
    assert f(cache.handle, 20, FAKE + 64, need, None) == hw.EINVAL and "overlaps" in hw.last_error()
    assert hw.cache_pages(cache) == (10, 10)
    assert f(cache.handle, 20, there, need, None) == hw.OK         # nothing to copy
    assert hw.cache_pages(cache) == (20, 20)
    pol = hw.policy_set(1, 1, 1, 64, 0, [16], [[0]])
    h = ctypes.c_void_p()
    assert hw._lib.hwkv_cache_alloc_format(ctypes.byref(h), pol.handle, 2, 64, 0, None, None, FAKE, 1 << 40) == hw.OK
    assert f(h, 1, there, need, None) == hw.EINVAL
    assert f(h, 0, there, need, None) == hw.OK
    hw._lib.hwkv_cache_free(h)


def test_batches_that_moves_cannot_name(hw):
    """Sequences are named in 16 bits, and one name is taken."""
    pol = hw.policy_set(1, 1, 1, 64, 0, [16], [[0]])
    for batch, ok in ((65534, True), (65535, False)):
        h = ctypes.c_void_p()
        assert hw._lib.hwkv_cache_alloc_format(ctypes.byref(h), pol.handle, batch, 64, 0, None, None, FAKE, 1 << 42) == hw.OK
        need = hw.cache_bytes(pol, batch, 64, "bf16")
        parents = (ctypes.c_int32 * batch)(*range(1, batch), -1)
        assert hw._lib.hwkv_cache_reorder(h, (ctypes.c_int32 * batch)(*range(batch)), None) == (hw.OK if ok else hw.EINVAL)
        if not ok:
            assert hw._lib.hwkv_cache_reorder(h, parents, None) == hw.EINVAL and "65534" in hw.last_error()
        assert hw._lib.hwkv_cache_move(h, 0, FAKE + (1 << 43), need, None) == (hw.OK if ok else hw.EINVAL)
        hw._lib.hwkv_cache_free(h)


def test_shared_decode_refuses(hw, cache):
    f = hw._lib.hwkv_decode_attn_shared
    scale = ctypes.c_float(0.125)
    q, out, ws = FAKE + (1 << 42), FAKE + (2 << 42), FAKE + (3 << 42)
    assert f(None, 0, q, scale, out, ws, 1 << 30, None) == hw.EINVAL
    for layer in (-1, 2):
        assert f(cache.handle, layer, q, scale, out, ws, 1 << 30, None) == hw.EINVAL and "layer" in hw.last_error()
    for a in ((None, out, ws), (q, None, ws)):
        assert f(cache.handle, 0, a[0], scale, a[1], a[2], 1 << 30, None) == hw.EINVAL and "null" in hw.last_error()
    for a in ((q + 8, out, ws), (q, out + 8, ws), (q, out, ws + 8)):
        assert f(cache.handle, 0, a[0], scale, a[1], a[2], 1 << 30, None) == hw.EINVAL and "aligned" in hw.last_error()
    for bad in (float("inf"), float("nan")):
        assert f(cache.handle, 0, q, ctypes.c_float(bad), out, ws, 1 << 30, None) == hw.EINVAL and "finite" in hw.last_error()
    assert f(cache.handle, 0, q, scale, out, ws, 1 << 30, None) == hw.EINVAL and "empty" in hw.last_error()


def test_shared_decode_workspace(hw, cache):
    f = hw._lib.hwkv_decode_shared_workspace_bytes
    n = ctypes.c_size_t()
    assert f(None, ctypes.byref(n)) == hw.EINVAL and f(cache.handle, None) == hw.EINVAL
    assert f(cache.handle, ctypes.byref(n)) == hw.OK
    assert n.value > 0 and n.value % 4 == 0
    # a cache that shares nothing has no parts of blocks
    pol = hw.policy_set(2, 2, 4, 64, 4, [128, 0], [[0, 1], [1, 1]])
    h = ctypes.c_void_p()
    assert hw._lib.hwkv_cache_alloc_format(ctypes.byref(h), pol.handle, 3, 1000, 0, None, None, FAKE, 1 << 40) == hw.OK
    m = ctypes.c_size_t()
    assert f(h, ctypes.byref(m)) == hw.OK and 0 < m.value < n.value
    hw._lib.hwkv_cache_free(h)
