"""Rotary positions, window attention and the paged cache on the CPU: frequencies against their formulas, and every refusal (a refused call
enqueues nothing and reads none of its buffers, so their addresses do not matter)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2604_13847_amd import binding as sb

BUF = C.c_void_p(4096)


def plain(rot, base=10000.0):
    return [base ** (-2.0 * i / rot) for i in range(rot // 2)]


def test_frequencies():
    f = plain(64)
    turns = lambda **kw: [2 * math.pi * x for x in sb.Rope(64, **kw).c.turns[:32]]
    assert np.allclose(turns(), f, rtol=1e-14)
    assert np.allclose(turns(base=500000.0), plain(64, 500000.0), rtol=1e-14)
    assert np.allclose(turns(scaling=sb.SB_ROPE_LINEAR, factor=8.0), [x / 8 for x in f], rtol=1e-14)
    assert np.allclose(turns(scaling=sb.SB_ROPE_NTK, factor=8.0), plain(64, 10000.0 * 8 ** (64 / 62)), rtol=1e-13)
    # by parts: the fast pairs as they were, the slow ones divided, in between falling
    for scaling, high in ((sb.SB_ROPE_YARN, 32.0), (sb.SB_ROPE_BANDS, 4.0)):
        got = turns(scaling=scaling, factor=8.0, original_length=4096.0)
        ratio = [a / b for a, b in zip(got, f)]
        assert all(b <= a + 1e-12 for a, b in zip(ratio, ratio[1:]))
        for x, r in zip(f, ratio):
            n = x * 4096 / (2 * math.pi)
            if n > 1.5 * high:
                assert abs(r - 1) < 1e-12
            if n < 0.6:
                assert abs(r - 1 / 8) < 1e-12
        mid = [i for i, r in enumerate(ratio) if 0.126 < r < 0.999]
        assert len(mid) >= 3
        if scaling == sb.SB_ROPE_BANDS:   # linear in the number of turns
            want = [1 / 8 + 7 / 8 * (f[i] * 4096 / (2 * math.pi) - 1) / 3 for i in mid]
        else:                             # linear in the pair's index, between the whole pairs around 32 turns and one
            pair = lambda n: 64 * math.log(4096 / (n * 2 * math.pi)) / (2 * math.log(10000.0))
            lo, hi = math.floor(pair(32.0)), math.ceil(pair(1.0))
            want = [1 - 7 / 8 * (i - lo) / (hi - lo) for i in mid]
        assert np.allclose([ratio[i] for i in mid], want, rtol=1e-12)
    assert sb.Rope(64, scaling=sb.SB_ROPE_YARN, factor=8.0, original_length=4096.0).c.amplitude == np.float32(0.1 * math.log(8) + 1)
    assert sb.Rope(64, scaling=sb.SB_ROPE_BANDS, factor=8.0, original_length=4096.0).c.amplitude == 1.0
    # a factor of one changes nothing
    for scaling in range(5):
        assert np.allclose(turns(scaling=scaling, factor=1.0, original_length=4096.0), f, rtol=1e-14)


@pytest.mark.parametrize("kw", [
    dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=130), dict(rot_dim=-2), dict(rot_dim=64, layout=2), dict(rot_dim=64, scaling=5), dict(rot_dim=64, scaling=-1),
    dict(rot_dim=64, base=1.0), dict(rot_dim=64, base=float("nan")), dict(rot_dim=64, base=float("inf")), dict(rot_dim=64, scaling=1, factor=0.5),
    dict(rot_dim=64, scaling=1, factor=float("nan")), dict(rot_dim=2, scaling=2, factor=2.0), dict(rot_dim=64, scaling=3, factor=2.0),
    dict(rot_dim=64, scaling=4, factor=2.0, original_length=-1.0), dict(rot_dim=64, scaling=4, factor=2.0, original_length=100.0, low=5.0, high=4.0)])
def test_bad_frequencies_are_refused(kw):
    with pytest.raises(sb.SparseBalError, match="error -1:"):
        sb.Rope(**kw)


def refused(rc, code, text):
    assert rc == code and text in sb.lib().sb_last_error().decode(), (rc, sb.lib().sb_last_error())


def problem(**kw):
    pb = sb.Problem([0, 40, 100], [1, 1], 4, 2, 64)
    pb.c.cu_seqlens_dev = 4096
    for k, v in kw.items():
        setattr(pb.c, k, v)
    return pb


def rope_call(pb, r, *, pos=None, q=BUF, qp=0, k=BUF, kp=0, qo=C.c_void_p(8192), ko=C.c_void_p(8192), direction=0):
    return sb.lib().sb_rope_apply(pb.ref(), r, pos, q, C.c_int64(qp), k, C.c_int64(kp), qo, ko, direction, None)


def test_rope_refusals():
    r = sb.Rope(64)
    refused(rope_call(problem(), None), -1, "null rope")
    refused(rope_call(problem(), sb.Rope(128).ref()), -1, "rot_dim")
    refused(rope_call(problem(), r.ref(), direction=2), -1, "direction")
    refused(rope_call(problem(), r.ref(), qp=4 * 64 - 1), -1, "q_pitch")
    refused(rope_call(problem(), r.ref(), kp=-5), -1, "k_pitch")
    refused(rope_call(problem(), r.ref(), qo=None), -1, "without its output")
    refused(rope_call(problem(), r.ref(), k=None), -1, "without its output")
    refused(rope_call(problem(), r.ref(), qp=4 * 64 + 8, qo=BUF), -1, "in place")
    refused(rope_call(problem(cu_seqlens_dev=None), r.ref()), -1, "cu_seqlens_dev")
    refused(rope_call(problem(dtype=3), r.ref()), -1, "dtype")
    assert rope_call(problem(), r.ref(), q=None, qo=None, k=None, ko=None) == 0
    bad = sb.Rope(64)
    bad.c.rot_dim = 33
    refused(rope_call(problem(), bad.ref()), -1, "rot_dim")


BAD_PROBLEMS = [(dict(num_q_heads=3), -1, "multiple"), (dict(head_dim=96), -2, "head_dim"), (dict(dtype=9), -1, "dtype"), (dict(num_seqs=-1), -1, "negative"),
                (dict(total_tokens=99), -1, "cu_seqlens must"), (dict(cu_seqlens_host=None), -1, "cu_seqlens_host"), (dict(num_seqs=0), -1, "S == 0"),
                (dict(cu_seqlens_dev=None), -1, "cu_seqlens_dev")]


@pytest.mark.parametrize("fields,code,text", BAD_PROBLEMS)
def test_window_refuses_bad_problems(fields, code, text):
    pb, L = problem(**fields), sb.lib()
    refused(L.sb_window_attn_fwd(pb.ref(), 8, 2, BUF, BUF, BUF, BUF, BUF, BUF, None), code, text)
    refused(L.sb_window_attn_bwd(pb.ref(), 8, 2, BUF, BUF, BUF, BUF, BUF, BUF, BUF, BUF, BUF, BUF, None), code, text)
    if "cu_seqlens_dev" not in fields:
        refused(L.sb_window_ws_bytes(pb.ref(), 8, 2, None, None), code, text)


def test_window_refusals():
    pb, L = problem(), sb.lib()
    for w, s in ((0, 0), (-3, 1), (5, -1)):
        refused(L.sb_window_attn_fwd(pb.ref(), w, s, BUF, BUF, BUF, BUF, BUF, BUF, None), -1, "window")
        with pytest.raises(sb.SparseBalError, match="window"):
            sb.sb_window_ws_bytes(pb, w, s)
    for w, s in ((2 ** 32 + 5, 0), (2 ** 31, 0), (5, 2 ** 32)):  # would arrive as another number
        with pytest.raises(sb.SparseBalError, match="window"):
            sb.sb_window_ws_bytes(pb, w, s)
    for missing in range(5):
        a = [BUF] * 5
        a[missing] = None
        refused(L.sb_window_attn_fwd(pb.ref(), 8, 2, *a, BUF, None), -1, "null argument")
    for missing in range(10):
        a = [BUF] * 10
        a[missing] = None
        refused(L.sb_window_attn_bwd(pb.ref(), 8, 2, *a, None), -1, "null argument")
    for odd in (0, 1, 2, 3):
        a = [BUF] * 5
        a[odd] = C.c_void_p(4096 + 8)
        refused(L.sb_window_attn_fwd(pb.ref(), 8, 2, *a, BUF, None), -1, "16 bytes")
    for odd in (0, 1, 2, 3, 5, 6, 7, 8, 9):
        a = [BUF] * 10
        a[odd] = C.c_void_p(4096 + 2)
        refused(L.sb_window_attn_bwd(pb.ref(), 8, 2, *a, None), -1, "16 bytes")
    # flattened rows pass 32 bits: 2^26 tokens, 64 query heads on one KV head
    cu = np.array([0, 1 << 26], dtype=np.int32)
    refused(L.sb_window_attn_fwd(problem(total_tokens=1 << 26, num_seqs=1, cu_seqlens_host=cu.ctypes.data, num_q_heads=64, num_kv_heads=1).ref(), 8, 2, BUF, BUF, BUF, BUF, BUF, BUF,
                                 None), -2, "32 bits")
    # budgets and blocks are not read
    pb = problem(topk_host=None, topk_dev=None, block_size=7, select_mode=9)
    assert sb.sb_window_ws_bytes(pb, 8, 2)[1] > 0
    # nothing to do: no launch, whatever the pointers
    empty = sb.Problem([0, 0], [1], 4, 2, 64)
    assert L.sb_window_attn_fwd(empty.ref(), 8, 2, None, None, None, None, None, None, None) == 0
    assert L.sb_window_attn_bwd(empty.ref(), 8, 2, *[None] * 10, None) == 0


def serving(cache=(), chunk=()):
    c = sb.sb_cache(10, 64, 2, 128, sb.SB_BF16, 4, 4096, 4096, 4096)
    n = sb.sb_chunk(3, 4, 20, 9, 200, 0.0, 4096, 4096)
    for k, v in dict(cache).items():
        setattr(c, k, v)
    for k, v in dict(chunk).items():
        setattr(n, k, v)
    return C.byref(c), C.byref(n)


@pytest.mark.parametrize("cache,chunk,code,text", [
    (dict(dtype=2), {}, -1, "dtype"), (dict(head_dim=80), {}, -2, "head_dim"), (dict(page_size=8), {}, -2, "page_size"), (dict(page_size=48), {}, -2, "page_size"),
    (dict(page_size=2048), {}, -2, "page_size"), (dict(num_pages=-1), {}, -1, "negative"), (dict(max_pages=-1), {}, -1, "negative"), ({}, dict(total_new=-1), -1, "negative"),
    (dict(num_kv_heads=3), {}, -1, "multiple"), ({}, dict(num_q_heads=0), -1, "multiple"), (dict(max_pages=1 << 26), {}, -2, "32 bits"), ({}, dict(cu_new=None), -1, "cu_new"),
    ({}, dict(cached=None), -1, "cached"), (dict(k=None), {}, -1, "pages"), (dict(page_table=None), {}, -1, "pages")])
def test_cache_refusals(cache, chunk, code, text):
    c, n = serving(cache, chunk)
    L = sb.lib()
    refused(L.sb_cache_attn(c, n, 8, 2, BUF, BUF, BUF, BUF, None), code, text)
    refused(L.sb_cache_append(c, n, None, None, C.c_int64(0), BUF, C.c_int64(0), BUF, C.c_int64(0), None, None), code, text)


def test_cache_argument_refusals():
    c, n = serving()
    L, z, out = sb.lib(), C.c_int64(0), C.c_int64()
    refused(L.sb_cache_attn(None, n, 8, 2, BUF, BUF, BUF, BUF, None), -1, "null cache")
    refused(L.sb_cache_attn(c, n, 0, 2, BUF, BUF, BUF, BUF, None), -1, "window")
    refused(L.sb_cache_attn(c, n, 8, -2, BUF, BUF, BUF, BUF, None), -1, "sinks")
    refused(L.sb_cache_attn(c, n, 8, 2, None, BUF, BUF, BUF, None), -1, "null argument")
    refused(L.sb_cache_attn(c, n, 8, 2, C.c_void_p(4096 + 4), BUF, BUF, BUF, None), -1, "16 bytes")
    refused(L.sb_cache_attn(*serving(dict(k=4096 + 8)), 8, 2, BUF, BUF, BUF, BUF, None), -1, "16 bytes")
    refused(L.sb_cache_attn_ws_bytes(c, n, 8, 2, None), -1, "null output")
    # runs of keys need a workspace: 64 sequences of 30000 tokens
    many = serving(dict(max_pages=500), dict(num_seqs=64, total_new=64, max_new=1, max_length=30000))
    assert L.sb_cache_attn_ws_bytes(*many, 8000, 2, C.byref(out)) == 0 and out.value >= 64 * 4 * 128 * 4
    refused(L.sb_cache_attn(*many, 8000, 2, BUF, BUF, BUF, None, None), -1, "null argument")
    refused(L.sb_cache_attn_ws_bytes(c, n, 0, 2, C.byref(out)), -1, "window")
    refused(L.sb_cache_append(c, n, sb.Rope(64).ref(), BUF, z, BUF, z, BUF, z, None, None), -1, "q without q_out")
    refused(L.sb_cache_append(c, n, None, None, z, None, z, BUF, z, None, None), -1, "null argument")
    refused(L.sb_cache_append(c, n, None, None, z, BUF, C.c_int64(100), BUF, z, None, None), -1, "k_pitch")
    refused(L.sb_cache_append(c, n, None, None, z, BUF, z, BUF, C.c_int64(255), None, None), -1, "v_pitch")
    small = serving(dict(head_dim=64))
    refused(L.sb_cache_append(*small, sb.Rope(128).ref(), None, z, BUF, z, BUF, z, None, None), -1, "rot_dim")
    for chunk in (dict(total_new=0), dict(num_seqs=0)):
        c, n = serving({}, chunk)
        assert L.sb_cache_attn(c, n, 8, 2, None, None, None, None, None) == 0
        assert L.sb_cache_append(c, n, None, None, z, None, z, None, z, None, None) == 0


def test_binding_refuses_tensors_on_the_cpu():
    import torch
    pb = problem()
    x = torch.zeros(100, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(sb.SparseBalError, match="GPU tensor"):
        sb.sb_rope_apply(pb, sb.Rope(64), x, None)
    with pytest.raises(sb.SparseBalError, match="GPU tensor"):
        sb.sb_window_attn_fwd(pb, 8, 2, x, x[:, :2], x[:, :2])
    with pytest.raises(sb.SparseBalError, match="needed"):
        sb.Cache(torch.zeros(3, 2, 16, 64, dtype=torch.float16), None, None)
