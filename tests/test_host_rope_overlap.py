"""CPU tests: an output in place of its own input is refused where another input
starts at the same address (the kernel would read rows as it turns them)."""
import ctypes

import pytest

FAKE = 0x7f0000000000


@pytest.fixture(scope="module")
def hw():
    from paper_2609_02029_amd import hwkv
    return hwkv


@pytest.mark.parametrize("hq,hk", [(2, 2), (4, 2), (2, 4)])
@pytest.mark.parametrize("side", ["q", "k", "both"])
def test_rope_apply_of_one_buffer_as_both_inputs(hw, hq, hk, side):
    rope = hw.rope_set(64, [1.0] * 16)
    x, far = FAKE + (1 << 20), FAKE + (8 << 20)
    qo = x if side in ("q", "both") else far
    ko = x if side in ("k", "both") else far
    # (contiguous rows: each side alone may be turned in place)
    rc = hw._lib.hwkv_rope_apply(rope.handle, 10, hq, hk, FAKE, x, hq * 64, x, hk * 64, qo, ko, None)
    assert rc == hw.EINVAL and "overlap" in hw.last_error()


@pytest.mark.parametrize("which", ["k_new", "v_new"])
def test_append_rope_of_queries_where_a_new_row_starts(hw, which):
    p = hw.policy_set(1, 2, 4, 64, 4, [256, 0], [[0, 1]])
    h, nb = ctypes.c_void_p(), hw.cache_bytes(p, 2, 300, "bf16")
    assert hw._lib.hwkv_cache_alloc_format(ctypes.byref(h), p.handle, 2, 300, 0, None, None, FAKE, nb) == hw.OK
    rope = hw.rope_set(64, [1.0] * 16)
    far = FAKE + (1 << 40)
    x, y = far + (1 << 20), far + (2 << 20)
    k, v = (x, y) if which == "k_new" else (y, x)
    rc = hw._lib.hwkv_append_rope(h, 0, rope.handle, far, k, 256, v, 256, x, 256, x, None)
    assert rc == hw.EINVAL and "overlap" in hw.last_error()
    n = ctypes.c_int64()
    assert hw._lib.hwkv_cache_seq_len(h, 0, 0, ctypes.byref(n)) == hw.OK and n.value == 0
    hw._lib.hwkv_cache_free(h)
