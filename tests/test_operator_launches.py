"""Which launches the calls of window attention and of the paged cache take, and which of them are refused, at sizes that no test runs (see test_operator_kernels.py)."""
import ctypes as C
import os
import subprocess
import sys

from paper_2604_13847_amd import binding as sb
from test_operator_kernels import NONE, ROOT, launches  # noqa: F401 (the fixture)


def test_the_largest_backward(launches):  # noqa: F811
    # 4.3 million tokens of 32 heads, 138 million rows: a bfloat16 backward has no launch that would be too large
    x = launches("window", [1000000] * 4 + [300000], 32, 8, 128, 0, 1000, 0)
    assert [k for k, _, _ in x] == ["window_fwd_kernel", "window_dq_kernel", "window_dkv_kernel"]


def serving(S, total, most, length, Hq=32, Hkv=8, D=128, page=64, pages=None):
    c = sb.sb_cache(1 << 20, page, Hkv, D, sb.SB_BF16, -(-length // page) if pages is None else pages, 4096, 4096, 4096)
    return c, sb.sb_chunk(S, Hq, total, most, length, 0.0, 4096, 4096)


def ws_bytes(c, n, window=NONE):
    out = C.c_int64()
    sb._check(sb.lib().sb_cache_attn_ws_bytes(C.byref(c), C.byref(n), window, 0, C.byref(out)))
    return out.value


def test_a_prompt_beside_single_tokens_asks_for_no_sums_of_its_own():
    """What the joined runs take is counted in the rows of sequences that have runs, not in the prompt's."""
    alone = ws_bytes(*serving(64, 64, 1, 32768))
    assert alone == 64 * 32 * 32 * (4 + 4 * 128)                                       # 32 runs of 64 rows of 32 heads
    # with up to 16 rows (64 of a group of four) of 64 sequences
    assert ws_bytes(*serving(64, 8192 + 63, 8192, 32768)) <= 16 * alone
    assert ws_bytes(*serving(64, 65536 + 63, 65536, 131072)) <= 4 * 16 * alone
    assert ws_bytes(*serving(64, 100, 37, 32768)) <= alone * 100 // 64 + 512           # fewer tokens in all than that


def test_a_length_that_the_table_cannot_hold():
    """max_length is about how long a sequence gets, whatever the caller knows of that; keys behind the page table do not exist."""
    assert ws_bytes(*serving(64, 64, 1, NONE, pages=512)) == ws_bytes(*serving(64, 64, 1, 32768))
    assert ws_bytes(*serving(2, 300, 200, NONE, pages=512)) == ws_bytes(*serving(2, 300, 200, 32768))
    assert ws_bytes(*serving(1, 1, 1, NONE, pages=1)) == ws_bytes(*serving(1, 1, 1, NONE, pages=0)) == 0


ROTATIONS = """
import ctypes as C, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
shim.recorded_kernel.restype = C.c_char_p
import numpy as np
from paper_2604_13847_amd import binding as sb
T = int(sys.argv[2])
cu, b, z = np.array([0, T], dtype=np.int32), C.c_void_p(4096), C.c_int64(0)
pb = sb.Problem([0, 100], [1], 1, 1, 64)
pb.c.total_tokens, pb.c.cu_seqlens_host, pb.c.cu_seqlens_dev = T, cu.ctypes.data, 4096
sb._check(sb.lib().sb_rope_apply(pb.ref(), sb.Rope(64).ref(), None, None, z, b, z, None, b, 0, None))
out = np.zeros((256, 6), dtype=np.uint32)
assert shim.recorded_launches(out.ctypes.data_as(C.c_void_p)) == 1
print("launch", *out[0])
"""


def test_rotations_of_very_many_tokens(tmp_path):
    """A launch has fewer than 2^32 threads; 2^29 tokens and more, at one a wavefront or eight, would take as many."""
    shim = str(tmp_path / "record_launches.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "launch", "record_launches.c")], check=True)
    for T, workgroups in ((2039, 510), (65536, 2048), (1 << 28, 1 << 23), (1 << 30, 1 << 23), (2 ** 31 - 1, (1 << 23) + (1 << 18))):
        r = subprocess.run([sys.executable, "-c", ROTATIONS, shim, str(T)], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout[-2000:]
        x, y, z, threads, _, _ = (int(n) for n in r.stdout.split("launch")[1].split())
        assert (y, z, threads) == (1, 1, 256) and x <= workgroups and x * threads < 1 << 32, (T, x)


def test_single_tokens_of_very_many_sequences(launches):  # noqa: F811
    # 65536 sequences, 8 KV heads, 32 runs of keys: 2^24 workgroups of two wavefronts
    x = launches("cache", 65536, 65536, 1, 32700, 32, 8, 128, 0, NONE)
    assert [k for k, _, _ in x] == ["cache_split_kernel", "cache_merge_kernel"] and x[0][2] == 65536 * 8 * 32
