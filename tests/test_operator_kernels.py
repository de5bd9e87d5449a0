"""What the compiler made of the kernels of window attention and of the paged cache (see test_hazards.py, whose scan this uses), and which kernels a call takes."""
import json
import os
import re
import subprocess
import sys

import pytest

import test_hazards as hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def without_float32(lines):
    """The float32 kernels, whose matrix instructions take another time, use none from inline assembly."""
    keep = True
    for l in lines:
        m = re.match(r"(_Z[\w.$]+):", l)
        if m:
            keep = "f32_kernel" not in m[1]
        if keep:
            yield l


@pytest.mark.parametrize("source,least", [("sb_window.hip", 12), ("sb_cache_attn.hip", 6)])
def test_waits_and_spills(source, least):
    lines = hazards.assembly(source)
    seen = products = loads = 0
    for name, code, labels in hazards.kernels(list(without_float32(lines))):
        seen += 1
        loads += sum(bool(re.match(r"(buffer_load\S* .* lds$|global_load_lds)", x.text)) for x in code)
        products += sum(x.matrix for x in code)
        bad = hazards.hazards(code, labels)
        assert not bad, (name, bad[:3])
        # a spilled register in these loops would also make the compiler wait for all loads in flight
        assert not [x.text for x in code if x.op.startswith("scratch_")], name
    assert seen >= least and loads >= 16 and products >= 24


CALLS = """
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
shim.recorded_kernel.restype = C.c_char_p
import numpy as np
from paper_2604_13847_amd import binding as sb
kind, a = json.loads(sys.argv[2])
b, lib = C.c_void_p(4096), sb.lib()
if kind == "window":
    lens, Hq, Hkv, D, dtype, window, sinks = a
    pb = sb.Problem(np.concatenate([[0], np.cumsum(lens)]), [1] * len(lens), Hq, Hkv, D, dtype=dtype)
    pb.c.cu_seqlens_dev = 4096
    sb._check(lib.sb_window_attn_fwd(pb.ref(), window, sinks, b, b, b, b, b, b, None))
    sb._check(lib.sb_window_attn_bwd(pb.ref(), window, sinks, b, b, b, b, b, b, b, b, b, b, None))
else:
    S, total, most, length, Hq, Hkv, D, dtype, window = a
    c = sb.sb_cache(1 << 20, 64, Hkv, D, dtype, length // 64 + 1, 4096, 4096, 4096)
    n = sb.sb_chunk(S, Hq, total, most, length, 0.0, 4096, 4096)
    sb._check(lib.sb_cache_attn(C.byref(c), C.byref(n), window, 0, b, b, b, b, None))
out = np.zeros((256, 6), dtype=np.uint32)
for i in range(shim.recorded_launches(out.ctypes.data_as(C.c_void_p))):
    print("kernel", shim.recorded_kernel(i).decode(), out[i][0])
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    shim = str(tmp_path_factory.mktemp("launch") / "record_launches.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "launch", "record_launches.c")], check=True)

    def of(kind, *a):
        r = subprocess.run([sys.executable, "-c", CALLS, shim, json.dumps([kind, a])], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout[-3000:]
        return [(re.search(r"(window_\w+?_kernel|cache_\w+?_kernel)(?:I(.*?)EEv)?", l.split()[1]), int(l.split()[2])) for l in r.stdout.splitlines() if l.startswith("kernel ")]

    return lambda *a: [(m[1], m[2] or "", n) for m, n in of(*a)]


NONE = 2 ** 31 - 1


def test_forms_of_the_backward(launches):
    form = lambda x: [re.search(r"DkvModeE(\d)", t)[1] for k, t, _ in x if k == "window_dkv_kernel"]
    # (0 whole items, 1 far rows, 2 parts, 3 their join)
    x = launches("window", [20000], 32, 8, 128, 0, 1000, 4)
    assert [k for k, _, _ in x] == ["window_fwd_kernel", "window_dq_kernel", "window_dkv_kernel", "window_dkv_kernel"] and form(x) == ["1", "0"]
    # the far items that the workspace was sized by: one block of 4 sinks, 64 runs of the rows behind the first 1000, by KV head
    assert x[2][2] == 8 * -(-(20000 - 1000) // 320) and x[3][2] == 8 * 157
    assert form(launches("window", [20000], 32, 8, 128, 0, 1000, 0)) == ["0"]        # no sinks
    assert form(launches("window", [20000], 32, 8, 128, 0, 1000, 600)) == ["0"]      # so many that their tiles take all rows
    assert form(launches("window", [20000], 32, 8, 128, 0, NONE, 4)) == ["0"]
    assert form(launches("window", [600, 400], 8, 2, 64, 0, 512, 4)) == ["2", "3"]
    assert form(launches("window", [3000], 4, 1, 128, 0, 256, 4)) == ["1", "2", "3"]
    assert form(launches("window", [1, 1], 8, 2, 64, 0, 512, 4)) == ["0"]
    assert [k for k, _, _ in launches("window", [300], 2, 1, 64, 1, 50, 4)] == ["window_fwd_f32_kernel", "window_delta_kernel", "window_dq_f32_kernel", "window_dkv_f32_kernel"]


def test_forms_of_a_chunk(launches):
    names = lambda *a: [k for k, _, _ in launches("cache", *a)]
    assert names(1, 1, 1, 4098, 32, 8, 128, 0, NONE) == ["cache_split_kernel", "cache_merge_kernel"]
    assert names(64, 64, 1, 100, 32, 8, 128, 0, NONE) == ["cache_split_kernel"]
    assert names(1, 3000, 3000, 3000, 32, 8, 128, 0, NONE) == ["window_fwd_kernel"]
    assert names(1, 100, 100, 30000, 4, 1, 128, 0, NONE) == ["window_fwd_kernel", "cache_merge_kernel"]
    assert names(10, 3000, 2000, 30000, 32, 8, 64, 0, NONE) == ["window_fwd_kernel", "cache_split_kernel", "cache_merge_kernel"]
    assert names(1, 1, 1, 20000, 4, 1, 64, 1, NONE) == ["window_fwd_f32_kernel", "cache_merge_kernel"]
    # 131072 new tokens of 32 heads are a launch, though as many workgroups that join runs would not be
    assert names(1, 131072, 131072, 131072, 32, 8, 128, 0, NONE) == ["window_fwd_kernel"]
    # runs of 128 keys for one sequence, of 1024 for 64; no more than two strips are one run
    assert launches("cache", 1, 1, 1, 4098, 32, 8, 128, 0, NONE)[0][2] == 8 * 33
    assert launches("cache", 64, 64, 1, 32769, 32, 8, 128, 0, NONE)[0][2] == 64 * 8 * 33
    assert names(1, 1, 1, 64, 32, 8, 128, 0, NONE) == ["cache_split_kernel"]
    # a window bounds the runs, whatever the length
    assert launches("cache", 64, 64, 1, 1 << 20, 32, 8, 128, 0, 1000)[0][2] <= 64 * 8 * 2


def test_forms_of_the_float32_backward(launches):
    of = lambda *a: [(k, n) for k, _, n in launches("window", *a) if "dkv" in k]
    assert of([1024], 1, 1, 64, 1, 200, 4) == [("window_dkv_f32_kernel", 32 * 4), ("window_dkv_f32_join_kernel", 32)]  # 32 strips of eight wavefronts
    assert of([1024], 1, 1, 64, 1, 200, 0) == [("window_dkv_f32_kernel", 32)]      # 7 strips without sinks
    assert of([1000, 24], 1, 1, 64, 1, 200, 4) == [("window_dkv_f32_kernel", 33)]  # 31
    assert of([1000, 24], 2, 1, 128, 1, NONE, 0) == [("window_dkv_f32_kernel", 33 * 7), ("window_dkv_f32_join_kernel", 33)]
    assert of([4096], 2, 1, 128, 1, NONE, 0) == [("window_dkv_f32_kernel", 128 * 2), ("window_dkv_f32_join_kernel", 128)]
    assert of([4097], 2, 1, 128, 1, NONE, 0) == [("window_dkv_f32_kernel", 129)]   # items enough to be one round by themselves
