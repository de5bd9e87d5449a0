"""Several axes, page tables and the four-bit cache: what the compiler made of the kernels, and which kernels a call takes (see test_operator_kernels.py and test_hazards.py)."""
import json
import os
import re
import subprocess
import sys

import pytest

import test_hazards as hazards
from test_operator_kernels import NONE, ROOT


@pytest.fixture(scope="module")
def functions():
    """{name: lines} of the kernels of attention over the four-bit cache"""
    out, name = {}, None
    for line in hazards.assembly("sb_cache4_attn.hip"):
        m = re.match(r"(_Z[\w.$]+):", line)
        if m:
            name = m[1]
        if name:
            out.setdefault(name, []).append(line)
    return out


def test_waits_of_the_chunks(functions):
    """Their tiles' rows go through the packed batches' code, whose inline assembly reads results of matrix instructions."""
    seen = 0
    for name, lines in functions.items():
        if "chunk" in name:
            (_, code, labels), = hazards.kernels(lines)
            bad = hazards.hazards(code, labels)
            assert not bad, (name, bad[:3])
            assert not [x.text for x in code if x.op.startswith("scratch_")], name
            seen += 1
    assert seen == 4


def test_loads_of_the_strips(functions):
    """An asynchronous load's place is set right in front of it, five wait states before it; what does not fit the registers is kept in memory outside the loop over strips only."""
    seen = 0
    for name, lines in functions.items():
        if "split" not in name:
            continue
        text = [l.split(";")[0].strip() for l in lines]
        text = [l for l in text if l and not l.startswith(".")] 
        loads = [i for i, l in enumerate(text) if l.startswith("global_load_lds")]
        assert len(loads) >= 6
        for i in loads:
            assert text[i - 1] == "s_nop 4" and text[i - 2].startswith("s_mov_b32 m0"), text[i - 3: i + 1]
        products = [i for i, l in enumerate(text) if l.startswith("v_mfma")]
        spills = [i for i, l in enumerate(text) if l.startswith("scratch_")]
        # (loads of spilled numbers would be waited for together with the strips': none between a strip's first product and its last)
        assert len(spills) <= 24 and not [i for i in spills if products[0] < i < products[-1]], name
        seen += 1
    assert seen == 12


CALLS = """
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
shim.recorded_kernel.restype = C.c_char_p
import numpy as np
from paper_2604_13847_amd import binding as sb
kind, a = json.loads(sys.argv[2])
b, z, lib = C.c_void_p(4096), C.c_int64(0), sb.lib()
if kind == "tables":
    S, total = a
    p = sb.sb_page_pool(S, 100, 1000, 16, 4096, 4096, 4096, 4096)
    sb._check(lib.sb_cache_tables(C.byref(p), b, b, total, b, b, b, b, None))
else:
    S, total, most, length, Hq, Hkv, D, dtype, window = a
    c = sb.sb_cache4(1 << 20, 64, Hkv, D, dtype, length // 64 + 1, 4096, 4096, 4096, 4096, 4096)
    n = sb.sb_chunk(S, Hq, total, most, length, 0.0, 4096, 4096)
    if kind == "append":
        sb._check(lib.sb_cache4_append(C.byref(c), C.byref(n), sb.Rope(D).ref(), None, None, b, z, b, z, b, z, C.c_void_p(1 << 50), None, None, None))
    else:
        sb._check(lib.sb_cache4_attn(C.byref(c), C.byref(n), window, 0, b, b, b, b, None))
out = np.zeros((256, 6), dtype=np.uint32)
for i in range(shim.recorded_launches(out.ctypes.data_as(C.c_void_p))):
    print("kernel", shim.recorded_kernel(i).decode(), out[i][0], out[i][1], out[i][3])
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    shim = str(tmp_path_factory.mktemp("launch") / "record_launches.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "launch", "record_launches.c")], check=True)

    def of(kind, *a):
        r = subprocess.run([sys.executable, "-c", CALLS, shim, json.dumps([kind, a])], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout[-3000:]
        lines = [l.split() for l in r.stdout.splitlines() if l.startswith("kernel ")]
        return [(re.search(r"\d+((?:cache|page|token)\w+?_kernel)", l[1])[1], int(l[2]), int(l[3])) for l in lines]

    return of


def test_launches_of_few_rows(launches):
    # as many workgroups as the chip holds, or as there are strips at most, and their parts joined four rows a workgroup
    assert launches("attn", 1, 1, 1, 4098, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 264, 1), ("cache4_join_kernel", 264, 1)]  # 8 items of 33 strips a wavefront
    assert launches("attn", 64, 64, 1, 32769, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 1024, 1), ("cache4_join_kernel", 1024, 1)]
    assert launches("attn", 64, 128, 2, 32769, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 768, 1), ("cache4_join_kernel", 768, 2)]       # 8 rows
    assert launches("attn", 64, 64, 1, 32769, 16, 1, 128, 0, NONE) == [("cache4_split_kernel", 512, 1), ("cache4_join_kernel", 512, 4)]         # 16
    assert launches("attn", 64, 512, 8, 32769, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 512, 1), ("cache4_join_kernel", 512, 8)]        # 32
    assert launches("attn", 64, 320, 5, 32769, 28, 4, 128, 0, NONE) == [("cache4_split_kernel", 512, 1), ("cache4_join_kernel", 512, 4)]        # 35: three tiles of 16
    assert launches("attn", 64, 64, 1, 32769, 32, 8, 64, 0, NONE) == [("cache4_split_kernel", 1280, 1), ("cache4_join_kernel", 1280, 2)]
    assert launches("attn", 64, 64, 1, 32769, 32, 8, 64, 1, NONE) == [("cache4_split_kernel", 1024, 1), ("cache4_join_kernel", 1024, 2)]
    # eight strips a wavefront, a window of that, or sixteen where items are many: whole items, nothing to join
    assert launches("attn", 1, 1, 1, 1024, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 8, 1)]
    assert launches("attn", 32, 32, 1, 2048, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 256, 1)]
    assert len(launches("attn", 31, 31, 1, 2048, 32, 8, 128, 0, NONE)) == len(launches("attn", 32, 32, 1, 2049, 32, 8, 128, 0, NONE)) == 2
    assert launches("attn", 64, 64, 1, 256, 32, 8, 128, 0, NONE) == [("cache4_split_kernel", 512, 1)]
    assert launches("attn", 64, 64, 1, 1 << 20, 32, 8, 128, 0, 100) == [("cache4_split_kernel", 512, 1)]
    # float32 prompts: tiles of 16 rows, whole where there are many
    assert launches("attn", 1, 4000, 4000, 4000, 32, 8, 128, 1, NONE) == [("cache4_split_kernel", 8 * 1000, 1)]
    assert launches("attn", 1, 100, 100, 4000, 32, 8, 128, 1, NONE)[0] == ("cache4_split_kernel", 512, 1)


def test_launches_of_chunks(launches):
    names = lambda *a: [k for k, _, _ in launches("attn", *a)]
    assert launches("attn", 1, 6001, 6001, 6001, 32, 8, 128, 0, NONE) == [("cache4_chunk_kernel", 8 * 94, 1)]
    assert names(1, 200, 200, 30000, 32, 8, 128, 0, NONE) == ["cache4_chunk_kernel", "cache_merge_kernel"]
    assert names(1, 1000, 1000, 1000, 32, 8, 128, 0, NONE) == ["cache4_chunk_kernel"]
    # mostly cached keys: equal shares; a batch of several may have sequences of few rows besides
    assert launches("attn", 1, 1000, 1000, 20000, 32, 8, 128, 0, NONE) == [("cache4_chunk_stream_kernel", 256, 1), ("cache4_join_kernel", 256, 16)]
    assert names(2, 4000, 2000, 30000, 28, 4, 128, 0, 8192) == ["cache4_chunk_stream_kernel", "cache4_join_kernel", "cache4_split_kernel", "cache4_join_kernel"]
    # rows that a tile's shares never cut: 131072 new tokens are one launch
    assert names(1, 131072, 131072, 131072, 32, 8, 128, 0, NONE) == ["cache4_chunk_kernel"]


def test_launches_of_the_others(launches):
    assert launches("tables", 64, 256) == [("page_tables_kernel", 1, 1)]
    assert launches("tables", 64, 4096) == [("page_tables_kernel", 1, 1)]
    assert launches("tables", 64, 4097) == [("page_tables_kernel", 1, 1), ("token_slots_kernel", 17, 1)]
    assert launches("append", 64, 64, 1, 2000, 32, 8, 128, 0, 1) == [("cache4_append_kernel", 64, 1)]
    assert launches("append", 2, 8192, 4096, 9000, 32, 8, 128, 0, 1) == [("cache4_append_kernel", 1024, 1)]
    # a launch has fewer than 2^32 threads
    (_, n, _), = launches("append", 1, 2 ** 31 - 1, 2 ** 31 - 1, 1 << 20, 1, 1, 64, 0, 1)
    assert n * 256 < 2 ** 32
