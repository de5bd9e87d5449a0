"""Several axes, page tables and the four-bit cache on the CPU: which pair is which axis', joined ropes, and every refusal (a refused call enqueues nothing and reads none of its
buffers, so their addresses do not matter)."""
import ctypes as C

import pytest
import torch

import four_bits as plain
from paper_2604_13847_amd import binding as sb
from test_operators_host import BUF, problem, refused

Z = C.c_int64(0)


# ---------------------------------------------------------------- axes
def axes_of(pairs, order=0):
    a = sb.RopeAxes(pairs, order=order)
    return [x for x in a.c.axis if x < a.c.num_axes]


def test_which_pair_is_which_axis():
    assert axes_of((2, 3, 1)) == [0, 0, 1, 1, 1, 2]
    assert axes_of((2, 3, 1), 1) == [0, 1, 2, 0, 1, 1]
    assert axes_of((24, 20, 20), 1) == [0, 1, 2] * 20 + [0] * 4
    assert axes_of((0, 2), 0) == axes_of((0, 2), 1) == [1, 1]
    assert axes_of((64,)) == [0] * 64 and axes_of((8,) * 8, 1) == list(range(8)) * 8


@pytest.mark.parametrize("pairs,order", [((), 0), ((0, 0), 0), ((-1, 5), 0), ((65,), 0), ((40, 25), 1), ((1,) * 9, 0), ((2 ** 31 - 1, 2), 0), ((4, 4), 2), ((4, 4), -1)])
def test_bad_axes_are_refused(pairs, order):
    with pytest.raises(sb.SparseBalError, match="error -1:"):
        sb.RopeAxes(pairs, order=order)


def test_joined_ropes():
    a, b = sb.Rope(24, base=500.0), sb.Rope(40, scaling=sb.SB_ROPE_LINEAR, factor=4.0)
    j = sb.Rope.joined([a, b])
    assert j.c.rot_dim == 64 and list(j.c.turns[:32]) == list(a.c.turns[:12]) + list(b.c.turns[:20]) and not any(j.c.turns[32:])
    ropes = (sb.sb_rope * 2)(a.c, b.c)
    sb._check(sb.lib().sb_rope_join(C.byref(ropes[0]), ropes, 2))  # in the first one's place
    assert bytes(ropes[0]) == bytes(j.c)
    with pytest.raises(sb.SparseBalError, match="at least one"):
        sb.Rope.joined([])
    with pytest.raises(sb.SparseBalError, match="one layout"):
        sb.Rope.joined([a, sb.Rope(8, layout=1)])
    with pytest.raises(sb.SparseBalError, match="one amplitude"):
        sb.Rope.joined([a, sb.Rope(8, scaling=sb.SB_ROPE_YARN, factor=4.0, original_length=100.0)])
    with pytest.raises(sb.SparseBalError, match="more than 64 pairs"):
        sb.Rope.joined([sb.Rope(128), a])
    bad = sb.Rope(8)
    bad.c.rot_dim = 7
    with pytest.raises(sb.SparseBalError, match="rot_dim"):
        sb.Rope.joined([bad])
    refused(sb.lib().sb_rope_join(None, ropes, 1), -1, "null rope")
    refused(sb.lib().sb_rope_axes_init(None, 1, BUF, 0), -1, "null argument")


def turn(pb, r, a, pos=BUF, q=BUF, qp=0, k=BUF, kp=0, qo=C.c_void_p(8192), ko=C.c_void_p(8192), direction=0):
    return sb.lib().sb_rope_axes_apply(pb.ref(), r, a, pos, q, C.c_int64(qp), k, C.c_int64(kp), qo, ko, direction, None)


def test_turn_refusals():
    r, a = sb.Rope(64).ref(), sb.RopeAxes((16, 16)).ref()
    refused(turn(problem(), None, a), -1, "null rope")
    refused(turn(problem(), r, None), -1, "axes and their positions")
    refused(turn(problem(), r, a, pos=None), -1, "axes and their positions")
    refused(turn(problem(), sb.Rope(128).ref(), a), -1, "rot_dim")
    refused(turn(problem(), r, sb.RopeAxes((16, 15)).ref()), -1, "pair 31")   # a rope of more pairs than the axes have
    bad = sb.RopeAxes((16, 16))
    for n in (0, 9, -1):
        bad.c.num_axes = n
        refused(turn(problem(), r, bad.ref()), -1, "num_axes")
    refused(turn(problem(), r, a, direction=2), -1, "direction")
    refused(turn(problem(), r, a, qp=255), -1, "q_pitch")
    refused(turn(problem(), r, a, ko=None), -1, "without its output")
    refused(turn(problem(), r, a, kp=136, ko=BUF), -1, "in place")
    refused(turn(problem(dtype=3), r, a), -1, "dtype")
    assert turn(problem(), r, a, q=None, qo=None, k=None, ko=None) == 0
    assert turn(sb.Problem([0, 0], [1], 4, 2, 64), r, a) == 0


# ---------------------------------------------------------------- page tables
def tables(pool=(), cached=BUF, added=BUF, total=10, cu=BUF, positions=BUF, slots=BUF, missing=BUF):
    p = sb.sb_page_pool(3, 4, 10, 64, 4096, 4096, 4096, 4096)
    for k, v in dict(pool).items():
        setattr(p, k, v)
    return sb.lib().sb_cache_tables(C.byref(p), cached, added, total, cu, positions, slots, missing, None)


def test_page_table_refusals():
    refused(sb.lib().sb_cache_tables(None, BUF, BUF, 1, BUF, BUF, BUF, BUF, None), -1, "null pool")
    for field in ("num_seqs", "max_pages", "num_pages"):
        refused(tables({field: -1}), -1, "negative")
    refused(tables(total=-1), -1, "negative")
    for size in (0, 8, 48, 2048):
        refused(tables(dict(page_size=size)), -2, "page_size")
    refused(tables(dict(max_pages=1 << 26)), -2, "32 bits")
    for field in ("page_table", "held", "free_pages", "free_count"):
        refused(tables({field: None}), -1, "null argument")
    for missing in ("cached", "added", "cu"):
        refused(tables(**{missing: None}), -1, "null argument")


def test_page_tables_without_arrays_of_tokens_do_not_read_their_size():
    for positions, slots in ((BUF, BUF), (BUF, None), (None, BUF)):
        refused(tables(total=-1, positions=positions, slots=slots), -1, "negative")
    refused(tables(pool=dict(page_size=48), total=-1, positions=None, slots=None), -2, "page_size")  # (the next refusal, so that nothing is launched)


def test_plain_tables_undo():
    """(the lists that the GPU's tables are held to)"""
    x = plain.Pool(3, 10, 20, 16, [7, 3, 9, 1] + list(range(10, 26)))
    x.step([0, 0, 0], [40, 0, 17], 57)
    before = [list(r) for r in x.rows], list(x.free)
    x.step([40, 0, 17], [30, 90, -1], 120)
    x.step([40, 0, 17], [0, 0, 0], 0)
    assert ([list(r) for r in x.rows], x.free) == before


# ---------------------------------------------------------------- four bits
def serving(cache=(), chunk=()):
    c = sb.sb_cache4(10, 64, 2, 128, sb.SB_BF16, 4, 4096, 4096, 4096, 4096, 4096)
    n = sb.sb_chunk(3, 4, 20, 9, 200, 0.0, 4096, 4096)
    for k, v in dict(cache).items():
        setattr(c, k, v)
    for k, v in dict(chunk).items():
        setattr(n, k, v)
    return C.byref(c), C.byref(n)


def append(c, n, r=None, axes=None, pos=None, q=None, qp=0, k=BUF, kp=0, v=BUF, vp=0, qo=None, kh=None, vh=None):
    return sb.lib().sb_cache4_append(c, n, r, axes, pos, q, C.c_int64(qp), k, C.c_int64(kp), v, C.c_int64(vp), qo, kh, vh, None)


def append_axes(c, n, r, axes, pos, q=None, k=BUF, v=BUF, qo=None):
    return sb.lib().sb_cache_append_axes(c, n, r, axes, pos, q, Z, k, Z, v, Z, qo, None)


@pytest.mark.parametrize("cache,chunk,code,text", [
    (dict(dtype=2), {}, -1, "dtype"), (dict(head_dim=80), {}, -2, "head_dim"), (dict(page_size=8), {}, -2, "page_size"), (dict(page_size=48), {}, -2, "page_size"),
    (dict(num_pages=-1), {}, -1, "negative"), (dict(max_pages=-1), {}, -1, "negative"), ({}, dict(total_new=-1), -1, "negative"), (dict(num_kv_heads=3), {}, -1, "multiple"),
    ({}, dict(num_q_heads=0), -1, "multiple"), (dict(max_pages=1 << 26), {}, -2, "32 bits"), ({}, dict(cu_new=None), -1, "cu_new"), ({}, dict(cached=None), -1, "cached"),
    (dict(k=None), {}, -1, "pages"), (dict(v_step=None), {}, -1, "pages"), (dict(page_table=None), {}, -1, "pages"), (dict(k=4104), {}, -1, "16 bytes"),
    (dict(v_step=4098), {}, -1, "16 bytes")])
def test_cache_refusals(cache, chunk, code, text):
    c, n = serving(cache, chunk)
    refused(sb.lib().sb_cache4_attn(c, n, 8, 2, BUF, BUF, BUF, BUF, None), code, text)
    refused(append(c, n), code, text)


def test_append_overlaps():
    """5 new tokens of 4 query and 2 KV heads of 128 in bfloat16: 5120 and 2560 bytes."""
    c, n = serving({}, dict(total_new=5, num_q_heads=4))
    for out, size in (("qo", 5120), ("kh", 2560), ("vh", 2560)):
        at = dict(k=C.c_void_p(1 << 20), v=C.c_void_p(2 << 20), q=C.c_void_p(3 << 20), qo=C.c_void_p(4 << 20), kh=C.c_void_p(5 << 20), vh=C.c_void_p(6 << 20))
        for other, there in (("k", 2560), ("v", 2560), ("q", 5120), ("qo", 5120), ("kh", 2560), ("vh", 2560)):
            if other == out:
                continue
            for place in (at[other].value - size + 16, at[other].value, at[other].value + there - 16):
                refused(append(c, n, **{**at, out: C.c_void_p(place)}), -1, "in the place of inputs or of each other")
    # a slice of a fused projection: what lies between its tokens counts
    refused(append(c, n, k=C.c_void_p(1 << 20), kp=4096, v=C.c_void_p(2 << 20), kh=C.c_void_p((1 << 20) + 4 * 8192)), -1, "in the place of inputs")


def test_append_overlaps_of_what_is_not_a_tensor():
    """Outputs in the place of the pages, of their steps, of the page table or of what else a call reads: 81920 bytes of codes, 10240 of steps."""
    M = 1 << 20
    there = dict(k=(10, 81920), v=(11, 81920), k_step=(12, 10240), v_step=(13, 10240), page_table=(14, 48), cu_new=(15, 16), cached=(16, 12), positions=(17, 2 * 20 * 4))
    base = dict(k=C.c_void_p(1 * M), v=C.c_void_p(2 * M), q=C.c_void_p(3 * M), qo=C.c_void_p(4 * M), kh=C.c_void_p(5 * M), vh=C.c_void_p(6 * M))
    c, n = serving({name: there[name][0] * M for name in ("k", "v", "k_step", "v_step", "page_table")}, dict(cu_new=15 * M, cached=16 * M))
    r, a, pos = sb.Rope(128).ref(), sb.RopeAxes((32, 32)).ref(), C.c_void_p(17 * M)
    for out, size in (("qo", 20 * 4 * 128 * 2), ("kh", 20 * 2 * 128 * 2), ("vh", 20 * 2 * 128 * 2)):
        for name, (at, bytes_) in there.items():
            for place in (at * M - size + 16, at * M, at * M + (bytes_ - 1) // 16 * 16):
                refused(append(c, n, r, a, pos, **{**base, out: C.c_void_p(place)}), -1, "in the place of the pages")


def test_append_refusals():
    c, n = serving()
    r, a = sb.Rope(128).ref(), sb.RopeAxes((32, 32)).ref()
    refused(append(None, n), -1, "null cache")
    refused(append(c, None), -1, "null cache")
    refused(append(c, n, q=BUF), -1, "q without q_out")
    refused(append(c, n, k=None), -1, "null argument")
    refused(append(c, n, kp=100), -1, "k_pitch")
    refused(append(c, n, vp=255), -1, "v_pitch")
    refused(append(c, n, qp=-1), -1, "q_pitch")
    for args in ((None, a, BUF), (r, a, None), (r, None, BUF)):
        refused(append(c, n, *args), -1, "axes and their positions")
    refused(append(c, n, r, sb.RopeAxes((32, 31)).ref(), BUF), -1, "pair 63")
    refused(append(*serving(dict(head_dim=64)), r), -1, "rot_dim")
    refused(append(c, n, q=BUF, qo=BUF), -1, "in the place of inputs")
    refused(append(c, n, kh=BUF), -1, "in the place of inputs")
    refused(append(c, n, vh=BUF), -1, "in the place of inputs")
    refused(append(c, n, vh=C.c_void_p(8200)), -1, "16 bytes")
    for chunk in (dict(total_new=0), dict(num_seqs=0)):
        assert append(*serving({}, chunk), k=None, v=None) == 0
    # the cache in the tensors' own type
    own = sb.sb_cache(10, 64, 2, 128, sb.SB_BF16, 4, 4096, 4096, 4096)
    for args in ((None, a, BUF), (r, None, BUF), (r, a, None), (None, None, None)):
        refused(append_axes(C.byref(own), n, *args), -1, "axes and their positions")
    refused(append_axes(C.byref(own), n, r, a, BUF, k=None), -1, "null argument")
    refused(append_axes(None, n, r, a, BUF), -1, "null cache")


def test_attention_refusals():
    c, n = serving()
    L, out = sb.lib(), C.c_int64()
    refused(L.sb_cache4_attn(None, n, 8, 2, BUF, BUF, BUF, BUF, None), -1, "null cache")
    refused(L.sb_cache4_attn(c, n, 0, 2, BUF, BUF, BUF, BUF, None), -1, "window")
    refused(L.sb_cache4_attn(c, n, 8, -2, BUF, BUF, BUF, BUF, None), -1, "sinks")
    for missing in range(3):
        a = [BUF] * 3
        a[missing] = None
        refused(L.sb_cache4_attn(c, n, 8, 2, *a, BUF, None), -1, "null argument")
    for odd in (0, 1, 3):
        a = [BUF] * 4
        a[odd] = C.c_void_p(4100)
        refused(L.sb_cache4_attn(c, n, 8, 2, *a, None), -1, "16 bytes")
    refused(L.sb_cache4_attn_ws_bytes(c, n, 8, 2, None), -1, "null output")
    refused(L.sb_cache4_attn_ws_bytes(c, n, 0, 2, C.byref(out)), -1, "window")
    many = serving(dict(max_pages=500), dict(num_seqs=64, total_new=64, max_new=1, max_length=30000))
    assert L.sb_cache4_attn_ws_bytes(*many, 8000, 2, C.byref(out)) == 0 and out.value >= 64 * 4 * 128 * 4
    refused(L.sb_cache4_attn(*many, 8000, 2, BUF, BUF, BUF, None, None), -1, "null argument")
    # flattened rows pass 32 bits
    refused(L.sb_cache4_attn(*serving(dict(num_kv_heads=1), dict(num_q_heads=64, total_new=1 << 26)), 8, 2, BUF, BUF, BUF, BUF, None), -2, "32 bits")
    for chunk in (dict(total_new=0), dict(num_seqs=0), dict(max_new=0)):
        assert L.sb_cache4_attn(*serving({}, chunk), 8, 2, None, None, None, None, None) == 0


def test_binding_refuses_what_lies_elsewhere(monkeypatch):
    x, ints = torch.zeros(100, 2, 64, dtype=torch.bfloat16), lambda *s: torch.zeros(s, dtype=torch.int32)
    pages, steps = torch.zeros(3, 2, 16, 32, dtype=torch.uint8), torch.zeros(3, 2, 16, 2, dtype=torch.bfloat16)
    axes = sb.RopeAxes((16, 16))
    with pytest.raises(sb.SparseBalError, match="GPU tensor"):
        sb.sb_rope_axes_apply(problem(), sb.Rope(64), axes, ints(2, 100), torch.zeros(100, 4, 64, dtype=torch.bfloat16), None)
    with pytest.raises(sb.SparseBalError, match="GPU tensor"):
        sb.Cache4(pages, pages, steps, steps, ints(2, 4))
    for bad in (dict(k=pages.float()), dict(dtype=torch.float16), dict(page_table=ints(8)), dict(k=pages[0])):
        with pytest.raises(sb.SparseBalError, match="needed"):
            sb.Cache4(**{**dict(k=pages, v=pages, k_step=steps, v_step=steps, page_table=ints(2, 4)), **bad})
    with pytest.raises(sb.SparseBalError, match="GPU tensor"):
        sb.PagePool(ints(2, 4), ints(2), ints(8), ints(1), 16)
    # tensors of the CPU say that they lie on device -1, which stands for the first device here
    monkeypatch.setattr(sb, "_here", lambda: (-1, 0))
    cache, chunk, pool = sb.Cache4(pages, pages, steps, steps, ints(2, 4)), sb.Chunk(ints(3), ints(2), 4, 100, 50, 60), sb.PagePool(ints(2, 4), ints(2), ints(8), ints(1), 16)
    for total in (-1, 2 ** 31, 2 ** 32 + 1):
        monkeypatch.setattr(sb, "_tensor", lambda *a, **kw: None)
        with pytest.raises(sb.SparseBalError, match="31 bits"):
            sb.sb_cache_tables(pool, ints(2), ints(2), total)
    monkeypatch.setattr(sb, "_here", lambda: (0, 0))
    elsewhere = "the current device is cuda:0"
    q = torch.zeros(100, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(sb.SparseBalError, match="cache: .*" + elsewhere):
        sb.sb_cache4_attn(cache, chunk, q)
    with pytest.raises(sb.SparseBalError, match="cache: .*" + elsewhere):
        sb.sb_cache4_append(cache, chunk, x, x)
    with pytest.raises(sb.SparseBalError, match="pool: .*" + elsewhere):
        sb.sb_cache_tables(pool, ints(2), ints(2), 3)
    cache.device = 0
    with pytest.raises(sb.SparseBalError, match="chunk: .*" + elsewhere):
        sb.sb_cache4_attn(cache, chunk, q)
