"""Registers and LDS of the kernels of beam selection, reordering and shared decode (no
GPU needed): what their launch shapes count on to have two workgroups on a CU, or one."""
import concurrent.futures as cf
import os
import re

import pytest

from paper_2609_02029_amd import build
from test_kernel_resources import _compile

FORMATS = {"bf16": 0, "f16": 1, "fp8": 2, "i8": 4}


def _short(name):
    """kernel<integers>, or as it is mangled where a type is among its arguments."""
    base = re.sub(r"^_ZN4hwkv12_GLOBAL__N_1\d+", "", name)
    m = re.match(r"([a-z_]+)I((?:L[ib]\d+E)+)E", base)
    return f"{m.group(1)}<{', '.join(re.findall(r'L[ib]([0-9]+)E', m.group(2)))}>" if m else base


@pytest.fixture(scope="module")
def table(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not found")
    d = str(tmp_path_factory.mktemp("asm"))
    srcs = ["beam_kernels.hip", "reorder_kernels.hip", "decode_shared_merge.hip"] + [f"decode_shared_{f}.hip" for f in FORMATS]
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs), os.cpu_count() or 1)) as ex:
        paths = list(ex.map(lambda s: _compile(s, d), srcs))
    out = {}
    for p in paths:
        text = open(p).read()
        for block in re.split(r"\n  - \.", text[text.index("amdhsa.kernels:"):])[1:]:
            at = [re.search(rf"\.{key}:\s+(\S+)", block) for key in
                  ("name", "vgpr_count", "private_segment_fixed_size", "group_segment_fixed_size")]
            if all(at):
                name, *sizes = (m.group(1) for m in at)
                out[_short(name)] = tuple(int(x) for x in sizes)
    return out


def test_shared_decode(table):
    for D in (64, 128, 256):
        for f in FORMATS.values():
            for n in (1, 2, 3):
                vg, scratch, lds = table[f"decode_shared<{D}, {f}, {n}>"]
                assert scratch == 0
                # two workgroups of four wavefronts a CU, or one
                assert vg <= (256 if n == 1 else 512)
                assert lds <= (80 if n == 1 else 160) * 1024
        assert table[f"shared_merge<{D}>"][1] == 0


def test_beam_selection(table):
    for t in (0, 1, 2):
        for held, most in ((8192, 80), (32768, 160)):
            vg, scratch, lds = table[f"beam_pick<{t}, {held}>"]
            assert scratch == 0 and vg <= 128 and lds <= most * 1024
        scan = [x for name, x in table.items() if name.startswith(f"beam_scan<{t}, ")]
        assert len(scan) == 1
        # six workgroups a CU
        assert scan[0][0] <= 80 and scan[0][1] == 0


def test_copies(table):
    names = [n for n in table if re.match("move_rows|table_move|page_copy|page_move|few", n)]
    assert len(names) == 9, names
    for n in names:
        assert table[n][1] == 0, n
