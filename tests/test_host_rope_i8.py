"""CPU tests of the rotation and of int8 caches: the oracle's encoding on
hand-worked rows, sizes, and every refusal that comes before device work (over
a device pointer that is never dereferenced)."""
import ctypes

import numpy as np
import pytest

from oracle import kvformat as KF

FAKE = 0x7f0000000000


@pytest.fixture(scope="module")
def hw():
    from paper_2609_02029_amd import hwkv
    return hwkv


# ---------------------------------------------------------------------------
# the oracle's int8 rows
# ---------------------------------------------------------------------------
def test_i8_rows_by_hand():
    # largest 1.5 in [2^0, 2^1): steps of 2^-6, scale byte 127
    r = KF.i8_rows([1.5, -1.0, 0.0078125, 0.0234375, -0.0390625, 0.0])
    assert r["scale"].tolist() == [127] * 6
    # 96, -64, 0.5 -> 0 (even), 1.5 -> 2, -2.5 -> -2 (even), 0
    assert r["code"].tolist() == [96, -64, 0, 2, -2, 0]
    assert KF.i8_values(r).tolist() == [1.5, -1.0, 0.0, 0.03125, -0.03125, 0.0]
    # 1.9921875 is 127.5 steps: clamped to 127, not 128
    assert KF.i8_rows([1.9921875, -1.9921875])["code"].tolist() == [127, -127]
    # a power of two: code 64 of its own scale
    r = KF.i8_rows([2.0 ** 100, 2.0 ** 94])
    assert r["scale"][0] == 227 and r["code"].tolist() == [64, 1]
    # zeros and subnormals: the smallest scale, steps of 2^-132
    assert KF.i8_rows([0.0, -0.0])["scale"].tolist() == [1, 1]
    r = KF.i8_rows([2.0 ** -126 - 2.0 ** -133, 2.0 ** -133, 3 * 2.0 ** -133])
    assert r["scale"][0] == 1 and r["code"].tolist() == [64, 0, 2]
    # not finite: 255 and zeros, all NaN
    for bad in (np.inf, -np.inf, np.nan):
        r = KF.i8_rows([1.0, bad])
        assert r["scale"].tolist() == [255, 255] and r["code"].tolist() == [0, 0]
        assert np.isnan(KF.i8_values(r)).all()


def test_i8_rows_error_and_exactness():
    """At most half a step (2^-7 of the row's power of two; a whole one at the
    clamp), and every value is a bf16 value."""
    x = np.random.default_rng(0).normal(size=(200, 64)).astype(np.float32)
    x = (x.view(np.uint32) & 0xffff0000).view(np.float32).astype(np.float64)
    r = KF.i8_rows(x)
    v = KF.i8_values(r)
    unit = np.exp2(r["scale"].astype(np.float64) - 127)
    assert np.all(np.abs(v - x) <= unit * np.where(np.abs(r["code"]) == 127, 2.0 ** -6, 2.0 ** -7))
    assert np.array_equal((v.astype(np.float32).view(np.uint32) & 0xffff), np.zeros(v.shape, dtype=np.uint32))
    assert np.all(np.abs(x).max(axis=1) < 2 * unit[:, 0]) and np.all(np.abs(x).max(axis=1) >= unit[:, 0])


# ---------------------------------------------------------------------------
# sizes and caches
# ---------------------------------------------------------------------------
def _pol(hw, **kw):
    a = dict(n_layers=2, n_kv_heads=2, n_q_heads=8, head_dim=64, n_sinks=4, level_window=[256, 0],
             level_of_unit=[[0, 1], [1, 0]])
    a.update(kw)
    return hw.policy_set(**a)


def test_i8_sizes(hw):
    p = _pol(hw)
    for D in (64, 128, 256):
        p = _pol(hw, head_dim=D)
        # 2 x 260 (320 rows padded) and 2 x 1000 (1024): codes and 2 scale bytes a row
        assert hw.cache_bytes(p, 3, 1000, "i8") == 3 * 2 * (320 + 1024) * (2 * D + 2)
        assert hw.policy_bytes(p, 1000, "i8") == 2 * (260 + 1000) * (2 * D + 2)
        fin = 3 * 2 * 320 * (2 * D + 2)
        pool = (fin + 255) // 256 * 256 + 7 * 256 * (2 * D + 2)
        assert hw.cache_bytes(p, 3, 1000, "i8", n_pages=7) == (pool + 255) // 256 * 256 + 2 * 3 * 4 * 4
    n = (1 << 24) + 1                     # as fp8: twice the tokens of a 16-bit format
    p = _pol(hw)
    assert hw.cache_bytes(p, 1, n, "i8") > 0
    with pytest.raises(hw.HwkvError):
        hw.cache_bytes(p, 1, 2 * n, "i8")


def _cache(hw, p, fmt, B=2, max_ctx=300, n_pages=None):
    h = ctypes.c_void_p()
    nb = hw.cache_bytes(p, B, max_ctx, {v[0]: k for k, v in hw.KV_FORMATS.items()}[fmt], n_pages=n_pages)
    if n_pages is None:
        rc = hw._lib.hwkv_cache_alloc_format(ctypes.byref(h), p.handle, B, max_ctx, fmt, None, None, FAKE, nb)
    else:
        rc = hw._lib.hwkv_cache_alloc_paged(ctypes.byref(h), p.handle, B, max_ctx, fmt, None, None, n_pages, FAKE, nb)
    assert rc == hw.OK, hw.last_error()
    return h


def test_i8_alloc_and_refusals(hw):
    p, L = _pol(hw), hw._lib
    h = ctypes.c_void_p()
    one = np.ones((2, 2), dtype=np.float32)
    nb = hw.cache_bytes(p, 2, 300, "i8")
    for ks, vs in ((one, None), (None, one)):      # the rows carry their scales
        rc = L.hwkv_cache_alloc_format(ctypes.byref(h), p.handle, 2, 300, 4,
                                       *(None if s is None else s.ctypes.data for s in (ks, vs)), FAKE, nb)
        assert rc == hw.EINVAL and not h.value
    rc = L.hwkv_cache_alloc_format(ctypes.byref(h), p.handle, 2, 300, 4, None, None, FAKE, nb - 1)
    assert rc == hw.ENOMEM and not h.value
    h = _cache(hw, p, 4)
    code, ks, vs = ctypes.c_int32(), np.zeros((2, 2), np.float32), np.zeros((2, 2), np.float32)
    assert L.hwkv_cache_format(h, ctypes.byref(code), ks.ctypes.data, vs.ctypes.data) == hw.OK
    assert code.value == 4 and np.all(ks == 1) and np.all(vs == 1)
    # prefill attention needs its workspace
    f = ctypes.c_float(0.1)
    assert L.hwkv_prefill_attn(h, 0, 0, 0, 4, FAKE, FAKE, FAKE, f, FAKE, None) == hw.EINVAL
    need = ctypes.c_size_t()
    assert L.hwkv_prefill_attn_workspace_bytes(h, 4, ctypes.byref(need)) == hw.OK
    assert need.value == 2 * 2 * (320 + 320) * 64 + 2 * 4 * 2 * 64 * 2    # two padded units' K and V, the chunk's
    assert L.hwkv_prefill_attn_ws(h, 0, 0, 0, 4, FAKE, FAKE, FAKE, f, FAKE, FAKE, need.value - 1, None) == hw.EINVAL
    out = np.zeros(300, dtype=np.uint8)
    assert L.hwkv_cache_read_scales(h, 2, 0, 0, out.ctypes.data, out.ctypes.data) == hw.EINVAL
    assert L.hwkv_cache_read_scales(h, 0, 0, 0, None, out.ctypes.data) == hw.EINVAL
    assert L.hwkv_cache_read_scales(None, 0, 0, 0, out.ctypes.data, out.ctypes.data) == hw.EINVAL
    L.hwkv_cache_free(h)
    h = _cache(hw, p, 2)
    assert L.hwkv_cache_read_scales(h, 0, 0, 0, out.ctypes.data, out.ctypes.data) == hw.EINVAL
    assert "int8" in hw.last_error()
    L.hwkv_cache_free(h)


def test_i8_replay_workspace(hw):
    a = hw.calib_workspace_bytes(8, 64, 4, 1000, 5, n_kv_heads=2, kv_format="fp8")
    assert hw.calib_workspace_bytes(8, 64, 4, 1000, 5, n_kv_heads=2, kv_format="i8") == a


# ---------------------------------------------------------------------------
# the rotation
# ---------------------------------------------------------------------------
def test_rope_set_refusals(hw):
    good = dict(head_dim=128, freq=[1.0] * 32, axis=[0] * 32, n_axes=2)
    hw.rope_free(hw.rope_set(**good))
    bad = [dict(head_dim=96), dict(head_dim=512), dict(freq=[1.0] * 72, axis=None), dict(freq=[], axis=None),
           dict(freq=[1.0] * 31, axis=None), dict(freq=[1.0] * 4, axis=None), dict(axis=[0] * 31 + [2]),
           dict(axis=[-1] + [0] * 31), dict(n_axes=0), dict(n_axes=9), dict(freq=[float("nan")] + [1.0] * 31),
           dict(freq=[float("inf")] + [1.0] * 31), dict(freq=[2e6] + [1.0] * 31), dict(magnitude=float("nan")),
           dict(magnitude=float("inf"))]
    for kw in bad:
        with pytest.raises(hw.HwkvError) as e:
            hw.rope_set(**{**good, **kw})
        assert e.value.code == hw.EINVAL, kw
    for kw in (dict(pairing="odd"), dict(axis=[0] * 3)):
        with pytest.raises(ValueError):
            hw.rope_set(**{**good, **kw})
    f = np.ones(8)
    h = ctypes.c_void_p()
    one = ctypes.c_float(1.0)
    assert hw._lib.hwkv_rope_set(None, 64, 16, 0, 1, f.ctypes.data, None, one) == hw.EINVAL
    assert hw._lib.hwkv_rope_set(ctypes.byref(h), 64, 16, 0, 1, None, None, one) == hw.EINVAL
    assert hw._lib.hwkv_rope_set(ctypes.byref(h), 64, 16, 2, 1, f.ctypes.data, None, one) == hw.EINVAL
    assert hw._lib.hwkv_rope_free(None) == hw.OK


def test_rope_apply_refusals(hw):
    rope = hw.rope_set(64, [1.0] * 16, n_axes=3)
    L, base, n = hw._lib, FAKE, 10

    def call(r=rope.handle, n=n, hq=4, hk=2, pos=base, q=base + (1 << 20), qs=256, k=base + (2 << 20), ks=128,
             qo=base + (3 << 20), ko=base + (4 << 20)):
        return L.hwkv_rope_apply(r, n, hq, hk, pos, q, qs, k, ks, qo, ko, None)

    assert call(n=0) == hw.OK and call(n=0, pos=None, q=None) == hw.OK and call(hq=0, hk=0) == hw.OK
    size = n * 256 * 2
    for kw in (dict(r=None), dict(n=-1), dict(n=1 << 29), dict(hq=-1), dict(hk=-1), dict(hq=70000), dict(pos=None),
               dict(pos=base + 2), dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(q=base + (1 << 20) + 8),
               dict(ko=base + (4 << 20) + 2), dict(qs=255), dict(qs=248), dict(qs=260), dict(ks=120),
               dict(qs=(1 << 31) + 8),
               dict(qo=base + (1 << 20) + 16),                     # shifted in place
               dict(qo=base + (1 << 20), qs=512),                  # in place, but apart
               dict(qo=base + (2 << 20)), dict(ko=base + (1 << 20) + size - 16),     # over the other input
               dict(qo=base + (2 << 20) - size + 16), dict(ko=base + (3 << 20)),     # over the other output
               dict(qo=base)):                                     # over the positions
        assert call(**kw) == hw.EINVAL, kw
        assert hw.last_error()


def test_append_rope_refusals(hw):
    p, L = _pol(hw), hw._lib
    rope, wide = hw.rope_set(64, [1.0] * 16), hw.rope_set(128, [1.0] * 16)
    h = _cache(hw, p, 0)
    far = FAKE + (1 << 40)

    def call(c=h, layer=0, r=rope.handle, pos=far, k=far + (1 << 20), ks=128, v=far + (2 << 20), vs=128,
             q=far + (3 << 20), qs=512, qo=far + (4 << 20)):
        return L.hwkv_append_rope(c, layer, r, pos, k, ks, v, vs, q, qs, qo, None)

    for kw in (dict(c=None), dict(r=None), dict(r=wide.handle), dict(layer=-1), dict(layer=2), dict(pos=None),
               dict(pos=far + 1), dict(k=None), dict(v=None), dict(q=None), dict(qo=None), dict(k=far + (1 << 20) + 8),
               dict(v=far + 2), dict(ks=127), dict(ks=120), dict(vs=0), dict(qs=504), dict(qo=far + (3 << 20) + 16),
               dict(qo=far + (1 << 20)), dict(qo=far), dict(qo=FAKE)):
        assert call(**kw) == hw.EINVAL, kw
    n = ctypes.c_int64()
    assert L.hwkv_cache_seq_len(h, 0, 0, ctypes.byref(n)) == hw.OK and n.value == 0
    L.hwkv_cache_free(h)
    # a pool without pages: refused before any launch, nothing changed
    h = _cache(hw, p, 4, n_pages=1)
    assert call(c=h) == hw.ENOMEM and "page" in hw.last_error()
    assert L.hwkv_cache_seq_len(h, 0, 0, ctypes.byref(n)) == hw.OK and n.value == 0
    L.hwkv_cache_free(h)


def test_binding_checks(hw):
    import torch
    rope = hw.rope_set(64, [1.0] * 16)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        hw.rope_apply(rope, pos, x, None, x, None)              # host tensors
    with pytest.raises(ValueError):
        hw.rope_apply(rope, pos, None, None, None, None)
    with pytest.raises(ValueError):
        hw.rope_apply(rope, pos, x, None, None, None)


# ---------------------------------------------------------------------------
# the kernels' registers
# ---------------------------------------------------------------------------
def test_kernels_are_present_within_their_registers(tmp_path):
    """Two wavefronts per SIMD for int8 decode (256 registers); none of them, nor
    the rotation's, uses scratch."""
    import os

    from paper_2609_02029_amd import build
    from test_kernel_resources import _compile, _kernels
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not found")
    # head_dims x groups x (split, by item), and the merge; head_dims x (1 + formats)
    for src, count in (("decode_i8.hip", 3 * 5 * 3), ("rope_kernels.hip", 3 * (1 + 4))):
        kernels = _kernels(_compile(src, str(tmp_path)))
        assert len(kernels) == count, (src, [name for name, _, _ in kernels])
        for name, vgprs, scratch in kernels:
            assert vgprs <= 256 and scratch == 0, (src, name, vgprs, scratch)
