"""Window attention and the paged cache where their inputs end or hold what is no number: against the same plain 64-bit forms as test_gpu_operators.py."""
import pytest
import torch

import operator_reference as ref
from paper_2604_13847_amd import binding as sb
from test_gpu_operators import DEV, NONE, Served, batch, nan, normal

pytestmark = pytest.mark.gpu
INF = float("inf")


# ---------------------------------------------------------------- tokens behind the page table
# (have, new, page, columns of the table, window, sinks): prompts' chunks and single tokens, rows in front of the table's end and behind it, windows and sinks that pass it
SHORT = [([0, 300], [200, 150], 16, 5, NONE, 0), ([70, 0], [130, 90], 16, 5, 40, 10), ([0, 130], [200, 100], 32, 3, 50, 500), ([64], [300], 16, 1, NONE, 7),
         ([100, 79, 80, 81, 40], [1, 1, 1, 1, 1], 16, 5, NONE, 0), ([200, 90], [1, 3], 16, 5, 20, 300), ([900, 30], [150, 1], 64, 2, 30, 400),
         ([0, 500], [180, 1], 16, 0, NONE, 3), ([600], [200], 64, 0, 100, 700)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,page,columns,window,sinks", SHORT)
def test_tokens_behind_the_page_table_are_seen_by_no_row(have, new, page, columns, window, sinks, dtype):
    x = Served(have, new, 8, 2, 128, page, dtype, spare_rows=1)
    x.table = x.table[:, :columns].contiguous()
    x.cache = sb.Cache(x.k_pages, x.v_pages, x.table)
    o, lse = x.check(window, sinks, there=lambda s, u: u < columns * page)
    for s, a in enumerate(have):
        if columns == 0 or (a - window + 1 >= columns * page and sinks == 0):
            rows = slice(x.cu[s], x.cu[s + 1])
            assert float(o[rows].abs().max()) == 0 and bool((lse[:, rows] == -INF).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,window,sinks", [([200, 1], 16, NONE), ([200, 1], NONE, 0), ([1, 2], 16, 70), ([1, 2], 100, 0), ([150, 3], 300, 64)])
def test_positions_far_behind_the_page_table(new, window, sinks, dtype):
    """Rows at the last positions that there are, over a table of 80 tokens: they see its sinks, or all of it in a window of everything, and no call walks what does not exist."""
    x = Served([60, 79], [20, 1], 8, 2, 64, 16, dtype)
    first = [2 ** 31 - 1 - n for n in new]
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=DEV)
    chunk = sb.Chunk(cu, torch.tensor(first, dtype=torch.int32, device=DEV), 8, sum(new), max(new), NONE)
    assert x.table.shape[1] == 5
    q = normal(3, sum(new), 8, 64, dtype=x.dtype)
    o, lse = sb.sb_cache_attn(x.cache, chunk, q, window, sinks)
    u = torch.arange(80, device=DEV)
    for s in (0, 1):
        rows = slice(int(cu[s]), int(cu[s + 1]))
        seen = ref.visible(torch.arange(first[s], first[s] + new[s], device=DEV), u, window, sinks)
        r = ref.Attention(q[rows].double(), x.k[s].double(), x.v[s].double(), seen, 64 ** -0.5, ref.HALF[x.dtype])
        ref.check("o", o[rows], r.o, r.o_tol)
        ref.check("lse", lse[:, rows], r.lse, r.lse_tol)


# ---------------------------------------------------------------- what is no number
# have, new, window, sinks, the key: one run of keys and several, single tokens and chunks; rows that see the key and rows that do not
PLANTED = [([50, 20], [1, 1], NONE, 0, 33), ([4000, 300], [1, 1], NONE, 0, 1003), ([4000, 300], [1, 1], 100, 0, 1003), ([0, 40], [300, 5], 100, 0, 130), ([0], [300], 100, 7, 5),
           ([3000], [100], 500, 0, 2550), ([3000], [100], NONE, 0, 3050), ([3000, 64], [12, 1], 300, 2, 2707)]


def check_planted(k, v, q, seen, o, lse, u, clean):
    """Rows [n] of one sequence, all heads: NaN where a score is NaN or +infinity, else what they are without the key: it is not seen or its weight is zero."""
    G, D = q.shape[1] // k.shape[1], q.shape[2]
    scores = torch.einsum("nhd,hd->nh", q.double(), k[u].double().repeat_interleave(G, 0))
    lost = seen[:, u, None] & (torch.isnan(scores) | (scores == INF))
    assert bool(torch.isnan(o[lost]).all()) and bool(torch.isnan(lse.T[lost]).all())
    without, kk = seen.clone(), k.double().clone()
    without[:, u], kk[u] = False, 0
    r = ref.Attention(q.double(), kk, v.double(), without, D ** -0.5, ref.HALF[o.dtype])
    hidden = ~lost & (~seen[:, u, None] | (scores == -INF))
    for name, got, want, tol in (("o", o, r.o, r.o_tol), ("lse", lse.T, r.lse.T, r.lse_tol.T)):
        ref.check(name, got[hidden], want[hidden], tol[hidden])
    rest = ~lost & ~hidden                                     # other KV heads' rows: the key is a number there
    assert torch.equal(o[rest], clean[0][rest]) and torch.equal(lse.T[rest], clean[1].T[rest])
    return int(lost.sum())


@pytest.mark.parametrize("value", [float("nan"), INF])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,window,sinks,u", PLANTED)
def test_keys_that_are_no_number_reach_the_rows_that_see_them(have, new, window, sinks, u, dtype, value):
    x = Served(have, new, 4, 2, 128, 16, dtype)
    clean = x.check(window, sinks)
    x.k[0][u, 1, 5] = value
    x.k_pages[x.table[0, u // 16].long(), 1, u % 16, 5] = value
    o, lse = x.attend(window, sinks)
    n, length = new[0], have[0] + new[0]
    seen = ref.visible(torch.arange(have[0], length, device=DEV), torch.arange(length, device=DEV), window, sinks)
    lost = check_planted(x.k[0], x.v[0], x.q[:n], seen, o[:n], lse[:, :n], u, (clean[0][:n], clean[1][:, :n]))
    assert lost > 0 or not bool(seen[:, u].any()) or (value == INF and n == 1)
    assert torch.equal(o[n:], clean[0][n:]) and torch.equal(lse[:, n:], clean[1][:, n:])   # the other sequences


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new", [([50], [1]), ([4000], [1]), ([0], [300]), ([3000], [100])])
def test_queries_that_are_no_number(have, new, dtype):
    x = Served(have, new, 4, 2, 64, 64, dtype)
    clean = x.check()
    i = new[0] // 2
    x.q[i, 1, 3], x.q[0, 2, 0] = float("nan"), float("nan")
    o, lse = x.attend()
    lost = torch.zeros(new[0], 4, dtype=torch.bool, device=DEV)
    lost[i, 1], lost[0, 2] = True, True
    assert bool(torch.isnan(o[lost]).all()) and bool(torch.isnan(lse.T[lost]).all())
    assert torch.equal(o[~lost], clean[0][~lost]) and torch.equal(lse.T[~lost], clean[1].T[~lost])


@pytest.mark.parametrize("value", [float("nan"), INF])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_keys_that_are_no_number_in_a_packed_batch(dtype, D, value):
    window, sinks, u, lens = 90, 3, 70, (250, 40)
    pb = batch(lens, 4, 2, D, dtype)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v = (normal(i, pb.T, h, D, dtype=t) for i, h in enumerate((4, 2, 2)))
    clean = sb.sb_window_attn_fwd(pb, window, sinks, q, k, v)
    k[u, 1, 5] = value
    o, lse = sb.sb_window_attn_fwd(pb, window, sinks, q, k, v)
    at = torch.arange(lens[0], device=DEV)
    n = lens[0]
    assert check_planted(k[:n], v[:n], q[:n], ref.visible(at, at, window, sinks), o[:n], lse[:, :n], u, (clean[0][:n], clean[1][:, :n])) > 0
    assert torch.equal(o[n:], clean[0][n:]) and torch.equal(lse[:, n:], clean[1][:, n:])


# ---------------------------------------------------------------- workspaces
@pytest.mark.parametrize("have,new,Hq,Hkv", [([2000, 900, 30, 0], [1, 200, 1, 90], 8, 2), ([2000, 1500], [1, 1], 8, 2), ([1500] * 5 + [4000], [1, 2, 16, 7, 1, 400], 4, 1),
                                             ([3000, 100], [3, 64], 1, 1), ([5000, 0, 2500], [1, 300, 1], 64, 1), ([3000], [100], 4, 1)])
def test_a_workspace_of_the_size_that_was_asked_for(have, new, Hq, Hkv):
    x = Served(have, new, Hq, Hkv, 128, 16)
    o, lse = x.check()
    need = sb.sb_cache_attn_ws_bytes(x.cache, x.chunk, NONE, 0)
    assert need > 0 and need % 4 == 0
    around = torch.full((need + 2048,), 0x5A, dtype=torch.uint8, device=DEV)
    again = sb.sb_cache_attn(x.cache, x.chunk, x.q, ws=around[1024: 1024 + need])
    assert torch.equal(again[0], o) and torch.equal(again[1], lse)
    assert bool((around[:1024] == 0x5A).all()) and bool((around[1024 + need:] == 0x5A).all())


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_rows_whose_scores_are_all_minus_infinity(dtype, D):
    """Such a row has no softmax: NaN in a packed batch, as in the block-sparse forward; over a cache it is a row that sees nothing."""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    pb = batch((100, 30), 2, 1, D, dtype)
    q, k, v = (normal(i, pb.T, h, D, dtype=t) for i, h in enumerate((2, 1, 1)))
    q[:, 0, 0], q[:, 1, 0] = 1.0, -1.0
    k[50:53, 0, 0] = -INF                                       # head 0: scores of -infinity, head 1: of +infinity
    o, lse = sb.sb_window_attn_fwd(pb, 2, 0, q, k, v)
    empty = torch.zeros(pb.T, dtype=torch.bool, device=DEV)
    empty[51:53] = True                                         # both keys of the window
    assert bool(torch.isnan(o[empty, 0]).all()) and bool(torch.isnan(lse[0, empty]).all())
    assert bool(torch.isfinite(o[~empty, 0]).all()) and bool(torch.isfinite(lse[0, ~empty]).all())
    assert torch.equal(o[50, 0], v[49, 0]) and torch.equal(o[53, 0], v[53, 0])
    for have, new in (([99], [1]), ([40], [60])):
        x = Served(have, new, 2, 1, D, 16, dtype)
        x.q[:, 0, 0], x.q[:, 1, 0] = 1.0, 1.0
        x.k_pages[:, :, :, 0] = -INF
        o, lse = x.attend()
        assert float(o.abs().max()) == 0 and bool((lse == -INF).all())


def near(rows, n):
    """Rows within 31 tokens of these."""
    out = rows.clone()
    for i in range(1, 32):
        out[i:] |= rows[:n - i]
        out[: n - i] |= rows[i:]
    return out


# head counts and lengths: dK/dV whole, in parts, with far rows and without, and in float32
@pytest.mark.parametrize("what", ["q", "d_o", "k", "v"])
@pytest.mark.parametrize("lens,Hq,Hkv,D,window,sinks,dtype", [((4200, 300), 16, 8, 128, 150, 0, "bf16"), ((4200, 300), 16, 8, 128, 150, 3, "bf16"), ((1300, 200), 4, 1, 64, 90, 70, "bf16"),
                                                              ((900, 200), 7, 1, 128, 400, 4, "bf16"), ((2500,), 2, 1, 64, 100, 600, "bf16"), ((900, 100), 4, 2, 64, 90, 4, "f32"),
                                                              ((600,), 2, 2, 128, 50, 0, "f32")])
def test_how_far_what_is_no_number_reaches_in_the_backward(lens, Hq, Hkv, D, window, sinks, dtype, what):
    """One NaN in the longest sequence.  Rows and keys that it must not reach are what they are without it, bit for bit."""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    pb = batch(lens, Hq, Hkv, D, dtype)
    x = {n: normal(i, pb.T, h, D, dtype=t) for i, (n, h) in enumerate((("q", Hq), ("k", Hkv), ("v", Hkv), ("d_o", Hq)))}

    def run():
        o, lse = sb.sb_window_attn_fwd(pb, window, sinks, x["q"], x["k"], x["v"])
        return (o, lse.T, *sb.sb_window_attn_bwd(pb, window, sinks, x["q"], x["k"], x["v"], o, lse, x["d_o"]))
    clean = run()
    n, at, g = lens[0], 407, Hkv - 1
    head = g if what in ("k", "v") else Hq - 1
    x[what][at, head, 3] = float("nan")
    got = run()
    u = torch.arange(n, device=DEV)
    seen = ref.visible(u, u, window, sinks)
    tiles = lambda rows, size: torch.stack([seen[:, i: i + size][rows].any() for i in range(0, n, size)]).repeat_interleave(size)[:n]
    rows = torch.zeros(n, dtype=torch.bool, device=DEV)
    if what in ("q", "d_o"):
        rows[at] = True                                   # that row alone, and the keys of the 128-token blocks that it sees any key of
        must = rows
    else:
        tile = slice(at // 64 * 64, at // 64 * 64 + 64)
        rows = near(seen[:, tile].any(1), n)              # rows that see a key of its 64-token tile, and those near them
        must = seen[:, at]
    keys = tiles(rows, 128)
    keys[at] |= what in ("k", "v")
    assert not bool(rows.all()) and (not bool(keys.all()) or sinks == 600)
    group = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
    heads = slice(Hq - 1, Hq) if what in ("q", "d_o") else group
    o, lse, dq, dk, dv = got
    for name, a, b in zip(("o", "lse", "dq", "dk", "dv"), got, clean):
        kv = name in ("dk", "dv")
        same = torch.ones(pb.T, dtype=torch.bool, device=DEV)
        same[:n] = ~(keys if kv else rows)
        assert torch.equal(a[same], b[same]), name         # rows and keys that are too far, and other sequences
        others = [h for h in range(a.shape[1]) if not (h == g if kv else heads.start <= h < heads.stop)]
        assert torch.equal(a[:, others], b[:, others]), name
        assert bool(torch.isfinite(b).all())
    # and what it has to reach
    nan_rows = lambda y: bool(torch.isnan(y).all())
    mine = [Hq - 1] if what in ("q", "d_o") else list(range(group.start, group.stop))
    for h in mine:
        assert nan_rows(dq[:n, h][must])
        if what in ("q", "k"):
            assert nan_rows(o[:n, h][must]) and nan_rows(lse[:n, h][must])
    assert nan_rows(dk[:n, g][seen[must].any(0)])
