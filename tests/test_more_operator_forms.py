"""Which kernels the calls of cache4_forms.py take, so that a change of the rules does not leave forms of the four-bit cache's attention without a test of their values; and what the
compiler made of the loops over strips."""
import json
import os
import re
import subprocess
import sys

import pytest

import cache4_forms as forms
from test_more_operator_kernels import functions, launches  # noqa: F401 (fixtures)
from test_operator_kernels import ROOT

CALLS = """
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
shim.recorded_kernel.restype = C.c_char_p
import numpy as np
from paper_2604_13847_amd import binding as sb
b, lib, at = C.c_void_p(4096), sb.lib(), 0
for have, new, Hq, Hkv, D, page, window, sinks, dtype, extra in json.loads(sys.argv[2]):
    need = [-(-(a + n) // page) for a, n in zip(have, new)]
    c = sb.sb_cache4(sum(need) + 2, page, Hkv, D, dtype, max(need) + extra, *[4096] * 5)
    n = sb.sb_chunk(len(have), Hq, sum(new), max(new), max(a + m for a, m in zip(have, new)), 0.0, 4096, 4096)
    sb._check(lib.sb_cache4_attn(C.byref(c), C.byref(n), window, sinks, b, b, b, b, None))
    count = shim.recorded_launches(np.zeros((256, 6), dtype=np.uint32).ctypes.data_as(C.c_void_p))
    print("call", *[shim.recorded_kernel(i).decode() for i in range(at, count)])
    at = count
"""


@pytest.fixture(scope="module")
def taken(tmp_path_factory):
    shim = str(tmp_path_factory.mktemp("launch") / "record_launches.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "launch", "record_launches.c")], check=True)

    def of(calls):
        r = subprocess.run([sys.executable, "-c", CALLS, shim, json.dumps(calls)], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout[-3000:]
        # (name, template arguments)
        names = lambda l: [(m[1], [a or b for a, b in re.findall(r"L[ij](\d+)E|(?<=I)(f|DF16b)(?=L)", k)]) for k in l.split()[1:] for m in [re.search(r"\d+((?:cache)\w+?_kernel)", k)]]
        out = [names(l) for l in r.stdout.splitlines() if l.startswith("call")]
        assert len(out) == len(calls)
        return out

    return of


def test_chunks_in_equal_shares(taken):
    calls = [(*c, 0, 0) for c in forms.SHARED_CHUNKS]
    for call, got in zip(calls, taken(calls)):
        D = str(call[4])
        assert got[:2] == [("cache4_chunk_stream_kernel", [D]), ("cache4_join_kernel", ["DF16b", D, "256"])], (call, got)


def test_few_rows_in_equal_shares(taken):
    for dtype, name in ((0, "DF16b"), (1, "f")):
        calls = [(*c, dtype, 0) for _, c in forms.SHARED_ROWS]
        for (rows, call), got in zip(forms.SHARED_ROWS, taken(calls)):
            rows = min(rows, 16) if dtype else rows
            D, (split, join) = str(call[4]), got
            parts, tiles = 16 // min(rows, 16), max(rows // 16, 1)
            assert split == ("cache4_split_kernel", [name, D, str(parts), str(tiles), "3" if dtype else "1"]), (call, got)
            assert join == ("cache4_join_kernel", [name, D, str(rows)]), (call, got)


def test_float32_chunks(taken):
    for calls, join in ((forms.WHOLE_FLOATS, False), (forms.SHARED_FLOATS, True)):
        calls = [(*c, 1, 0) for c in calls]
        for call, got in zip(calls, taken(calls)):
            D = str(call[4])
            assert got == [("cache4_split_kernel", ["f", D, "1", "1", "3"]), ("cache4_join_kernel", ["f", D, "16"])][: 1 + join], (call, got)


def test_whole_items_of_float32_chunks(launches):  # noqa: F811
    """From 1280 items of 16 rows on, which is where they even out by themselves, both sides measured."""
    assert launches("attn", 1, 700, 700, 8700, 32, 8, 128, 1, forms.NONE) == [("cache4_split_kernel", 8 * 175, 1)]
    assert launches("attn", 1, 2000, 2000, 22000, 32, 8, 128, 1, forms.NONE) == [("cache4_split_kernel", 8 * 500, 1)]
    assert launches("attn", 1, 300, 300, 8300, 32, 8, 128, 1, forms.NONE) == [("cache4_split_kernel", 512, 1), ("cache4_join_kernel", 512, 4)]


@pytest.mark.parametrize("dtype,total,workgroups", [(0, 2048, 512), (0, 4096, 1024), (0, 4097, 1025), (0, 6000, 1500), (0, 7680, 1920), (0, 8193, 2049), (0, 10000, 2500), (0, 16384, 4096),
                                                    (0, 100000, 25000), (1, 4097, 1025), (1, 8192, 2048), (1, 8193, 2049)])
def test_append_of_many_tokens_fills_the_chip(launches, dtype, total, workgroups):  # noqa: F811
    """A token more never makes much fewer wavefronts than the 4096 that fill the chip: four to a workgroup, a token each."""
    assert launches("append", 2, total, total, 9000, 32, 8, 128, dtype, 1) == [("cache4_append_kernel", workgroups, 1)]


def loops(lines):
    """Bodies of a function's natural loops, smallest first."""
    code, labels = [], {}
    for line in (l.split(";")[0].strip() for l in lines):
        m = re.match(r"([\w.$]+):$", line)
        if m:
            labels[m[1]] = len(code)
        elif line and line[0] != ".":
            code.append(line)
    after, before = [[] for _ in code], [[] for _ in code]
    for i, x in enumerate(code):
        words = x.split()
        if words[0].startswith(("s_branch", "s_cbranch")):
            after[i].append(labels[words[1]])
        if words[0] not in ("s_branch", "s_endpgm") and i + 1 < len(code):
            after[i].append(i + 1)
    for i, targets in enumerate(after):
        for j in targets:
            before[j].append(i)

    def reached(i, without):
        """Whether the start leads to i on a way round `without`: a branch there is no loop then."""
        seen, todo = {without}, [0]
        while todo:
            n = todo.pop()
            if n not in seen:
                seen.add(n)
                todo += after[n]
        return i in seen and i != without

    found = []
    for i, targets in enumerate(after):
        for head in (j for j in targets if j <= i and not reached(i, j)):
            body, todo = {head, i}, [i]
            while todo:
                n = todo.pop()
                for j in before[n] if n != head else ():
                    if j not in body:
                        body.add(j)
                        todo.append(j)
            found.append([code[n] for n in sorted(body)])
    return sorted(found, key=len)


def test_loops():
    """Of two loops, one in the other, where the inner one's body goes on behind the outer one's end."""
    outer, inner = loops(["a:", "v_x", "b:", "v_y", "s_cbranch_scc1 c", "d:", "v_z", "s_cbranch_scc0 b", "s_cbranch_scc1 a", "s_endpgm", "c:", "v_w", "s_branch d"])[::-1]
    assert [x.split()[0] for x in inner] == ["v_y", "s_cbranch_scc1", "v_z", "s_cbranch_scc0", "v_w", "s_branch"] and "v_x" in outer and len(outer) == 8


def test_nothing_is_spilled_in_the_loop_over_strips(functions):  # noqa: F811
    """From the loop's head, where the next strip's loads are issued, to its end: a spilled number there would be waited for together with the strips."""
    seen = 0
    for name, lines in functions.items():
        if "split" not in name:
            continue
        body = next(b for b in loops(lines) if any(x.startswith("v_mfma") for x in b))
        assert sum(x.startswith("global_load_lds") for x in body) == (6 if "Li128E" in name else 3), name
        assert sum(x.startswith("v_mfma") for x in body) == sum(x.split()[0].startswith("v_mfma") for l in lines for x in [l.strip()] if x), name  # all products of a strip
        assert not [x for x in body if x.startswith("scratch_")], name
        seen += 1
    assert seen == 12
