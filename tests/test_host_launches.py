"""CPU tests of what the host hands to the kernels of shared decode and reordering: the
library as it is, in a process whose kernel launches are looked at and not made
(``launch_shim.cpp``), so that caches can be filled, forked and decoded without a GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    from paper_2609_02029_amd import build
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not found")
    so = str(tmp_path_factory.mktemp("shim") / "launch_shim.so")
    r = subprocess.run([build.HIPCC, "--offload-host-only", "-x", "hip", "-std=c++17", "-O1", "-fPIC", "-shared",
                        f"-I{build.INCLUDE}", f"-I{build.CSRC}", os.path.join(ROOT, "tests", "launch_shim.cpp"),
                        "-o", so, "-ldl"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]

    def go(what):
        preload = " ".join([so] + [x for x in [os.environ.get("LD_PRELOAD")] if x])
        env = dict(os.environ, LD_PRELOAD=preload, HIP_VISIBLE_DEVICES="", SHIM=so)
        r = subprocess.run([sys.executable, os.path.abspath(__file__), what], cwd=ROOT, env=env, capture_output=True,
                           text=True, timeout=600)
        assert r.returncode == 0, (r.stdout + r.stderr)[-6000:]
    return go


def test_shared_decode_takes_no_more_than_its_workspace(run):
    run("workspace")


def test_a_reorder_moves_no_more_entries_than_a_table_row_has(run):
    run("table")


# ---- in the process of the shim
FAKE, BUF = 0x7f0000000000, 1 << 42


class Filled:
    """A paged cache of one layer over memory that is never touched."""

    def __init__(self, hw, H, G, D, fmt, families, prompt, tails, levels=None, pages=None):
        import ctypes
        self.hw, self.lib = hw, hw._lib
        self.B = sum(families)
        max_ctx = max(prompt) + max(tails) + 1
        self.pol = hw.policy_set(1, H, H * G, D, 4, [100, 0], [levels or [1] * H])
        self.h = ctypes.c_void_p()
        n = pages or H * self.B * -(-max_ctx // 256)
        assert self.lib.hwkv_cache_alloc_paged(ctypes.byref(self.h), self.pol.handle, self.B, max_ctx, hw.KV_FORMATS[fmt][0],
                                               None, None, n, FAKE, BUF) == hw.OK, hw.last_error()
        parents, b = [], 0
        for i, count in enumerate(families):
            self.write(b, 0, prompt[i % len(prompt)])
            parents += [b] * count
            b += count
        self.reorder(parents)
        self.len = [prompt[i % len(prompt)] for i, count in enumerate(families) for _ in range(count)]
        for b in range(self.B):
            self.write(b, self.len[b], tails[b % len(tails)])

    def write(self, b, at, n):
        assert self.lib.hwkv_prefill_write(self.h, 0, b, at, n, FAKE + 2 * BUF, FAKE + 3 * BUF, None) == self.hw.OK, self.hw.last_error()

    def reorder(self, parents):
        import ctypes
        rc = self.lib.hwkv_cache_reorder(self.h, (ctypes.c_int32 * self.B)(*parents), None)
        assert rc == self.hw.OK, self.hw.last_error()

    def decode(self):
        import ctypes
        n = ctypes.c_size_t()
        assert self.lib.hwkv_decode_shared_workspace_bytes(self.h, ctypes.byref(n)) == self.hw.OK
        at = [FAKE + i * BUF for i in (2, 3, 4)]
        rc = self.lib.hwkv_decode_attn_shared(self.h, 0, at[0], 0.125, at[1], at[2], n.value, None)
        assert rc == self.hw.OK, self.hw.last_error()

    def free(self):
        self.lib.hwkv_cache_free(self.h)


def workspace(hw, shim):
    """Families of unequal sizes, in as many heads as fill the card and more, that
    share from a page to five; tails that are empty, short, or of several pages."""
    import random
    made = shim.shim_launches(b"decode_shared")
    cases = [(8, 4, 64, "bf16", [9] + [2] * 43, [300], [20]), (32, 4, 128, "bf16", [9] + [2] * 9, [300], [20]),
             (16, 2, 128, "f16", [20] + [2] * 14, [300], [20]), (8, 4, 256, "bf16", [9] + [2] * 31, [800], [20]),
             (8, 4, 128, "bf16", [12] + [2] * 42, [356], [0])]
    rng = random.Random(5)
    for i in range(600):
        families, left = [], rng.choice([4, 30, 60, 96, 96, 200])
        if i % 2:                      # one wide family, and pairs
            families = [rng.randint(3, 24)]
            left = max(2, left - families[0]) // 2 * 2
            families += [2] * (left // 2)
            left = 0
        while left > 0:
            families.append(min(left, rng.choice([1, 2, 2, 2, 3, 5, 9, 12, 17, 40])))
            left -= families[-1]
        H = rng.choice([1, 2, 8, 16, 32, 40, 64])
        cases.append((H, rng.choice([1, 2, 4, 6, 8]), rng.choice([64, 128, 256]), rng.choice(["bf16", "f16", "fp8", "i8"]),
                      families, [rng.randint(1, 1400) for _ in range(1 if i % 2 else rng.randint(1, 3))],
                      [rng.randint(0, rng.choice([1, 30, 600])) for _ in range(rng.randint(1, 5))],
                      [rng.randint(0, 1) for _ in range(H)] if rng.random() < 0.3 else None))
    short = []
    for c in cases:
        r = Filled(hw, *c)
        try:
            r.decode()
        except AssertionError as e:
            short.append((c, str(e)))
        r.free()
    assert not short, (len(short), short[:3])
    assert shim.shim_launches(b"decode_shared") >= made + len(cases)


def table(hw, shim):
    """Sequences that are longer in a layer of windows alone than any full unit may be:
    forked and permuted, with more table entries than lists of them hold."""
    import ctypes
    L, H, B, max_ctx = 2, 6, 10, 2800
    pol = hw.policy_set(L, H, H, 64, 4, [100, 0], [[1] * H, [0] * H])
    for parents in ([0] * B, [B - 1 - b for b in range(B)], [(b + 1) % B for b in range(B)]):
        h, made = ctypes.c_void_p(), shim.shim_launches(b"table_move")
        assert hw._lib.hwkv_cache_alloc_paged(ctypes.byref(h), pol.handle, B, max_ctx, 0, None, None, 1000, FAKE, BUF) == hw.OK
        for b in range(B):
            for layer, n in ((0, max_ctx - b), (1, 9000 + b)):
                assert hw._lib.hwkv_prefill_write(h, layer, b, 0, n, FAKE + 2 * BUF, FAKE + 3 * BUF, None) == hw.OK
        assert hw._lib.hwkv_cache_reorder(h, (ctypes.c_int32 * B)(*parents), None) == hw.OK, hw.last_error()
        assert shim.shim_launches(b"table_move") > made
        assert shim.shim_fault() == b"", shim.shim_fault()
        hw._lib.hwkv_cache_free(h)


if __name__ == "__main__":
    import ctypes
    sys.path.insert(0, ROOT)
    shim = ctypes.CDLL(os.environ["SHIM"])
    shim.shim_fault.restype = ctypes.c_char_p
    from paper_2609_02029_amd import hwkv
    {"workspace": workspace, "table": table}[sys.argv[1]](hwkv, shim)
