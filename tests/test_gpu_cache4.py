"""The cache in four bits on the GPU: what an append writes, bit for bit, and attention over it against the plain 64-bit form (operator_reference.py, where the bounds are derived:
held values are operands without any rounding, probabilities times steps are rounded where the bfloat16 cache rounds probabilities)."""
import numpy as np
import pytest
import torch

import four_bits as plain
import operator_reference as ref
from paper_2604_13847_amd import binding as sb
from test_gpu_operators import DEV, NONE, SERVED, TYPE, batch, nan, normal
from test_gpu_rope_axes import positions, turned

pytestmark = pytest.mark.gpu
INF = float("inf")


class Served4:
    """Sequences with `have` cached and `new` new tokens, in scattered pages of the four-bit cache; rows that no token owns have all bits set (steps that are no numbers)."""

    def __init__(self, have, new, Hq, Hkv, D, page, dtype="bf16", spare_rows=0, seed=0, fill=True, spare_pages=0):
        self.have, self.new, self.D, self.Hq, self.Hkv, self.page, self.dtype = have, new, D, Hq, Hkv, page, TYPE[dtype][0]
        S = len(have)
        need = [(a + n + page - 1) // page for a, n in zip(have, new)]
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).int()
        self.table = torch.full((S, max(need + [1]) + spare_pages), -1, dtype=torch.int32, device=DEV)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at: at + n]
            at += n
        self.codes = [torch.full((pages, Hkv, page, D // 2), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.steps = [nan(pages, Hkv, page, D // 32) for _ in range(2)]
        self.x = [[None] * S, [None] * S]  # keys and values as held
        gen = torch.Generator(device=DEV).manual_seed(seed + 1)
        for s in range(S if fill else 0):
            u = torch.arange(have[s] + new[s], device=DEV)
            p = self.table[s, u // page].long()
            for w in (0, 1):
                code = torch.randint(0, 16, (len(u), Hkv, D), generator=gen, device=DEV)
                step = (torch.randint(32, 64, (len(u), Hkv, D // 32), generator=gen, device=DEV) / 128.0).bfloat16()
                self.codes[w][p, :, u % page], self.steps[w][p, :, u % page] = plain.pack(code, w == 1), step
                self.x[w][s] = plain.value(code, step)
        self.rows = sum(new)
        self.q = normal(seed + 7, self.rows + spare_rows, Hq, D, dtype=self.dtype)
        self.cu_dev = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
        self.cu = [int(c) for c in self.cu_dev]
        self.cached = torch.tensor(have, dtype=torch.int32, device=DEV)
        self.cache = sb.Cache4(self.codes[0], self.codes[1], self.steps[0], self.steps[1], self.table, dtype=self.dtype)
        self.chunk = sb.Chunk(self.cu_dev, self.cached, Hq, self.rows + spare_rows, max(new + [0]), max([a + n for a, n in zip(have, new)] + [0]))

    def attend(self, window=NONE, sinks=0):
        o, lse = nan(*self.q.shape, dtype=self.dtype), nan(self.Hq, len(self.q), dtype=torch.float32)
        sb.sb_cache4_attn(self.cache, self.chunk, self.q, window, sinks, o=o, lse=lse)
        return o, lse

    def check(self, window=NONE, sinks=0, there=None, scale=None):
        o, lse = self.attend(window, sinks)
        for s, (a, n) in enumerate(zip(self.have, self.new)):
            rows = slice(self.cu[s], self.cu[s + 1])
            if n == 0:
                continue
            u = torch.arange(a + n, device=DEV)
            seen = ref.visible(torch.arange(a, a + n, device=DEV), u, window, sinks)
            if there is not None:
                seen = seen & there(s, u)
            r = ref.Attention(self.q[rows].double(), self.x[0][s], self.x[1][s], seen, scale or self.D ** -0.5, ref.HALF[self.dtype])
            ref.check("o", o[rows], r.o, r.o_tol)
            ref.check("lse", lse[:, rows], r.lse, r.lse_tol)
        assert bool(torch.isnan(o[self.rows:]).all()) and bool(torch.isnan(lse[:, self.rows:]).all())
        return o, lse


# ---------------------------------------------------------------- append
@pytest.mark.parametrize("rot,layout,axes,dtype,D,page", [
    (128, 0, None, "bf16", 128, 16), (128, 1, (16, 24, 24), "bf16", 128, 64), (64, 0, (16, 16), "f32", 64, 32), (48, 1, None, "f32", 64, 16), (22, 0, (5, 6), "bf16", 64, 16),
    (62, 0, None, "bf16", 128, 32), (40, 0, None, "f32", 128, 16), (None, 0, None, "bf16", 128, 16), (None, 0, None, "f32", 64, 128)])
def test_append(rot, layout, axes, dtype, D, page):
    """Codes, steps and held values are those of the formulas, bit for bit; rows behind the last sequence and rows of pages that no new token owns are left as they were."""
    x = Served4([40, 0, 3, 500, 15], [1, 70, 0, 33, 2], 6, 2, D, page, dtype, spare_rows=3, fill=False)
    t, n = x.dtype, len(x.q)
    rope = sb.Rope(rot, layout=layout) if rot else None
    ax, pos = (sb.RopeAxes(axes), positions(7, len(axes), n, 1 << 16)) if axes else (None, None)
    k, v = normal(20, n, 2, D, dtype=t) * 3, normal(21, n, 2, D, dtype=t)
    qn, kh, vh = nan(n, 6, D, dtype=t), nan(n, 2, D, dtype=t), nan(n, 2, D, dtype=t)
    sb.sb_cache4_append(x.cache, x.chunk, k, v, rope=rope, axes=ax, positions=pos, q=x.q, q_out=qn, held=True, k_held=kh, v_held=vh)
    where = pos
    if not axes:
        where = torch.zeros(1, n, dtype=torch.int32, device=DEV)
        for s, a in enumerate(x.have):
            where[0, x.cu[s]: x.cu[s + 1]] = a + torch.arange(x.new[s], device=DEV)
    if rope:
        one = ax or sb.RopeAxes((rot // 2,))
        want_q, tol = turned(x.q.double(), where, rope, one, layout == 0)
        ref.check("q", qn[: x.rows], want_q[: x.rows], (tol + ref.HALF[t] * want_q.abs())[: x.rows])
        want_k = turned(k.double(), where, rope, one, layout == 0)[0].float()
    else:
        assert torch.equal(qn[: x.rows], x.q[: x.rows])
        want_k = k.float()
    assert bool(torch.isnan(qn[x.rows:]).all()) and bool(torch.isnan(kh[x.rows:]).all()) and bool(torch.isnan(vh[x.rows:]).all())
    seen = torch.zeros(x.codes[0].shape[0], page, dtype=torch.bool, device=DEV)
    for w, (y, held) in enumerate(((want_k, kh), (v.float(), vh))):
        step = plain.step_of(y)
        code = plain.code_of(y, step)
        assert torch.equal(held[: x.rows].double(), plain.value(code, step)[: x.rows])
        for s, (a, m) in enumerate(zip(x.have, x.new)):
            u, rows = torch.arange(a, a + m, device=DEV), slice(x.cu[s], x.cu[s + 1])
            p = x.table[s, u // page].long()
            assert torch.equal(x.codes[w][p, :, u % page], plain.pack(code[rows], w == 1)) and torch.equal(x.steps[w][p, :, u % page].double(), step[rows])
            seen[p, u % page] = True
        assert bool((x.codes[w].transpose(1, 2)[~seen] == 255).all()) and bool(torch.isnan(x.steps[w].transpose(1, 2)[~seen]).all())


def test_append_of_what_is_hard_to_round():
    """Ties and their neighbours, groups of zeros, of tiny and of huge numbers, and numbers that are none."""
    D = 64
    x = Served4([0], [40], 2, 2, D, 16, "f32", fill=False)
    v = torch.zeros(40, 2, D, device=DEV)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device=DEV)
    for i in range(20):  # steps 2^(i - 10) and 63/32 of that
        s = 2.0 ** (i - 10) * (63 / 32 if i % 2 else 1)
        v[i, 0, :8], v[i, 0, 8:16] = ties * s, -ties * s
        v[i, 0, 16:24], v[i, 0, 24:31] = torch.nextafter(ties * s, ties * 0), torch.nextafter(ties * s, ties * 99)[:7]
        v[i, 0, 32:40] = ties * s
    v[21, 0, 3], v[22, 0, 3], v[23, 0, 3] = 1e-38, -1e-44, 3.4e38
    v[24, 0, 5], v[25, 0, 5], v[26, 0, 40] = INF, float("nan"), -INF
    v[27, 0] = -0.0
    v[:, 1] = normal(1, 40, D, dtype=torch.float32)
    _, _, held = sb.sb_cache4_append(x.cache, x.chunk, torch.zeros_like(v), v, held=True)
    step = plain.step_of(v)
    code = plain.code_of(v, step)
    want = plain.value(code, step)
    fine = torch.isfinite(step).repeat_interleave(32, -1)
    assert torch.equal(held.double()[fine], want[fine]) and bool(torch.isnan(held[~fine]).all()) and int((~fine).sum()) == 96
    u = torch.arange(40, device=DEV)
    p = x.table[0, u // 16].long()
    packed, got = plain.unpack(x.codes[1][p, :, u % 16], True), x.steps[1][p, :, u % 16].double()
    assert torch.equal(packed, code) and torch.equal(got[torch.isfinite(step)], step[torch.isfinite(step)]) and bool(torch.isnan(got[~torch.isfinite(step)]).all())
    # no value is off by more than a quarter of its group's largest step between levels, and most by less
    assert float(((held - v).abs() / step.repeat_interleave(32, -1))[:, 1].max()) <= 1.0 + 2.0 ** -5 * 6


def test_what_is_not_turned_is_not_touched():
    """Infinities and negative zeros beside elements that are: in the same pair of a lane, and in the same eight."""
    x = Served4([5], [3], 1, 1, 64, 16, "f32", fill=False)
    for rot, layout in ((22, 1), (30, 1), (22, 0), (48, 0)):
        q = normal(1, 3, 1, 64, dtype=torch.float32)
        q[0, 0, rot:], q[1, 0, rot:], q[2, 0, rot:] = INF, -0.0, float("nan")
        qn = sb.sb_cache4_append(x.cache, x.chunk, q, q, rope=sb.Rope(rot, layout=layout), q=q)
        assert torch.equal(qn[..., rot:].view(torch.int32), q[..., rot:].view(torch.int32)) and bool(torch.isfinite(qn[..., :rot]).all())


def test_append_from_slices_and_without_queries():
    D = 128
    x, y = (Served4([10, 0], [5, 30], 4, 2, D, 16, fill=False) for _ in range(2))
    fused = normal(1, 35, 8, D)
    k, v, q = fused[:, 4:6], fused[:, 6:8], fused[:, :4]
    rope = sb.Rope(D)
    a = sb.sb_cache4_append(x.cache, x.chunk, k, v, rope=rope, q=q)
    odd = torch.empty(35 * 2 * D + 1, dtype=torch.bfloat16, device=DEV)[1:].view(35, 2, D)
    odd.copy_(k)
    assert sb.sb_cache4_append(y.cache, y.chunk, odd, v.contiguous(), rope=rope) is None
    for w in (0, 1):
        assert torch.equal(x.codes[w], y.codes[w]) and torch.equal(x.steps[w].view(torch.int16), y.steps[w].view(torch.int16))
    pb = batch((35,), 4, 2, D)
    where = torch.cat([torch.arange(10, 15), torch.arange(30)]).int().to(DEV)
    want = sb.sb_rope_apply(pb, rope, q, k, positions=where)[0]
    assert float((a.double() - want.double()).abs().max()) <= 2.0 ** -7 * float(want.abs().max())


def test_append_without_pages():
    """Tokens whose page is missing, or behind the table, are written nowhere; their queries are turned and their held values given all the same."""
    x = Served4([0, 20], [40, 30], 2, 1, 64, 16, fill=False)
    x.table[0, 1], x.table[1, 2] = -1, 10 ** 6
    short = x.table[:, :3].contiguous()
    cache = sb.Cache4(x.codes[0], x.codes[1], x.steps[0], x.steps[1], short)
    k, v = normal(1, 70, 1, 64), normal(2, 70, 1, 64)
    q, kh, vh = sb.sb_cache4_append(cache, x.chunk, k, v, rope=sb.Rope(64), q=x.q, held=True)
    assert not bool(torch.isnan(q).any() | torch.isnan(kh).any() | torch.isnan(vh).any())
    written = (~torch.isnan(x.steps[1].float()).any(-1)).sum()
    assert int(written) == 16 + 8 + 12  # tokens 0 .. 15 and 32 .. 39 of the first, 20 .. 31 of the second


# ---------------------------------------------------------------- attention
MORE = [([0], [1], 1, 1, 64, 16, NONE, 0), ([31, 32, 33, 127, 128, 129], [1] * 6, 16, 1, 128, 16, NONE, 0), ([5000], [1], 17, 1, 128, 16, 4000, 3),
        ([2047, 9], [16, 16], 1, 1, 64, 1024, NONE, 0), ([300, 301], [6, 7], 20, 4, 128, 16, 33, 17), ([0, 0, 7], [500, 1, 65], 4, 2, 64, 16, 70, 1), ([17000], [1], 2, 1, 128, 64, NONE, 0),
        ([8200, 8300], [1, 2], 2, 1, 64, 16, 8192, 40)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,Hq,Hkv,D,page,window,sinks", SERVED + MORE)
def test_attention(have, new, Hq, Hkv, D, page, window, sinks, dtype):
    Served4(have, new, Hq, Hkv, D, page, dtype, spare_rows=3, spare_pages=2).check(window, sinks)


# equal shares of tiles; whole items with windows and sinks, chunks of unequal lengths and single tokens beside them; keys in runs, without and with a window; whole items  (equal shares with windows: cache4_forms.py)
CHUNKS = [([2600, 2000, 3001], [400, 399, 130], 16, 8, 128, 64, NONE, 0), ([2600, 2000, 3001], [400, 399, 401], 16, 8, 64, 16, 900, 70), ([3000, 2500, 100, 2900], [300, 300, 1, 77], 24, 8, 128, 32, 500, 5),
          ([9000], [150], 4, 2, 128, 16, NONE, 0), ([0, 0], [700, 650], 16, 8, 128, 16, NONE, 0), ([1], [1300], 8, 1, 64, 64, 200, 300)]


@pytest.mark.parametrize("have,new,Hq,Hkv,D,page,window,sinks", CHUNKS)
def test_chunks(have, new, Hq, Hkv, D, page, window, sinks):
    x = Served4(have, new, Hq, Hkv, D, page, spare_rows=2, spare_pages=1)
    a = x.check(window, sinks)
    b = x.attend(window, sinks)
    assert torch.equal(a[0][: x.rows], b[0][: x.rows]) and torch.equal(a[1][:, : x.rows], b[1][:, : x.rows])


def test_chunks_without_pages():
    x = Served4([2600, 2000, 3001], [400, 399, 130], 16, 8, 128, 64)
    x.table[0, 7], x.table[0, 46], x.table[2, 0] = -1, 10 ** 8, -7
    x.table[1] = -1
    gone = {0: (7, 46), 1: range(999), 2: (0,)}
    o, lse = x.check(there=lambda s, u: torch.tensor([int(i) // 64 not in gone[s] for i in u], device=DEV))
    rows = slice(x.cu[1], x.cu[2])
    assert float(o[rows].abs().max()) == 0 and bool((lse[:, rows] == -INF).all())


@pytest.mark.parametrize("dtype,spare_pages", [("bf16", 0), ("f32", 0), ("bf16", 1 << 19)])
def test_many_sequences(dtype, spare_pages):
    """More sequences than a wavefront has lanes, most of them short, one long; and with so wide a table that strips are counted by fours."""
    have = [(37 * i) % 150 for i in range(300)]
    have[211] = 3000
    Served4(have, [i % 3 for i in range(300)], 16, 8, 64, 64, dtype, spare_rows=2, spare_pages=spare_pages).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_without_pages(dtype):
    """Entries that are no page (-1, too large), inside a sequence and for a whole one: their keys are seen by no row."""
    for new in ([1, 1, 1], [70, 3, 20]):
        x = Served4([500, 90, 300], new, 8, 2, 128, 32, dtype, spare_rows=1)
        x.table[0, 3], x.table[0, 15], x.table[2, 0] = -1, 10 ** 8, -7
        x.table[1] = -1
        gone = {0: (3, 15), 1: range(99), 2: (0,)}
        o, lse = x.check(there=lambda s, u: torch.tensor([int(i) // 32 not in gone[s] for i in u], device=DEV))
        rows = slice(x.cu[1], x.cu[2])
        assert float(o[rows].abs().max()) == 0 and bool((lse[:, rows] == -INF).all())


SHORT = [([0, 300], [200, 150], 16, 5, NONE, 0), ([0, 130], [200, 100], 32, 3, 50, 500), ([100, 79, 80, 81, 40], [1, 1, 1, 1, 1], 16, 5, NONE, 0), ([200, 90], [1, 3], 16, 5, 20, 300),
         ([0, 500], [180, 1], 16, 0, NONE, 3), ([600], [200], 64, 0, 100, 700)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,page,columns,window,sinks", SHORT)
def test_tokens_behind_the_page_table_are_seen_by_no_row(have, new, page, columns, window, sinks, dtype):
    x = Served4(have, new, 8, 2, 128, page, dtype, spare_rows=1)
    x.table = x.table[:, :columns].contiguous()
    x.cache = sb.Cache4(x.codes[0], x.codes[1], x.steps[0], x.steps[1], x.table, dtype=x.dtype)
    x.check(window, sinks, there=lambda s, u: u < columns * page)


@pytest.mark.parametrize("new", [1, 5, 150])
def test_what_is_no_number(new):
    """A key's step that is no number makes all rows NaN that see it, in its KV head alone; one of a key behind the sequence, or hidden from a whole tile, reaches nobody."""
    x = Served4([400, 300], [new, new], 4, 2, 64, 16)
    before = x.attend(window=100)
    p = lambda s, u: (int(x.table[s, u // 16]), u % 16)
    a, b = p(0, 10)
    x.steps[0][a, :, b] = float("nan")  # 90 tokens and more behind every window
    x.steps[1][a, :, b] = float("nan")
    again = x.attend(window=100)
    assert torch.equal(before[0], again[0]) and torch.equal(before[1], again[1])
    a, b = p(1, 299)
    x.steps[0][a, 1, b, 0] = float("nan")
    o, lse = x.attend(window=100)
    rows = slice(x.cu[1], min(x.cu[2], x.cu[1] + 100 - 1))
    assert bool(torch.isnan(o[rows, 2:]).all()) and bool(torch.isnan(lse[2:, rows]).all())
    assert torch.equal(o[:, :2], before[0][:, :2]) and torch.equal(o[: x.cu[1]], before[0][: x.cu[1]]) and torch.equal(lse[:2], before[1][:2])
    x.q[0, 3] = float("nan")
    o, _ = x.attend(window=100)
    assert bool(torch.isnan(o[0, 3]).all()) and torch.equal(o[0, :2], before[0][0, :2])


def between():
    """Products p0 = y0 k0 and p1 = y1 k1 of whole numbers times 2^-24 and steps of six bits, whose sum in float32 is 8 if p1 alone is rounded before it, and the next number if p0 alone is."""
    rng = np.random.default_rng(5)
    exact = lambda y, k: float(y) * 2.0 ** -24 * float(k)  # 24 and 6 bits: exact in float64, as the sums below are
    while True:
        k0, k1 = rng.integers(48, 64) / 64.0, rng.integers(33, 63) / 64.0
        y0 = int(rng.integers(int(5.0 / k0 * 2 ** 24), int(5.9 / k0 * 2 ** 24))) & ~7
        y1 = int((8.0 + 2.0 ** -21 - exact(y0, k0)) / k1 * 2 ** 24) & ~3
        for z1 in range(y1 - 8, y1 + 12, 4):
            p0, p1 = exact(y0, k0), exact(z1, k1)
            if np.float32(p0 + float(np.float32(p1))) <= 8 < np.float32(p1 + float(np.float32(p0))) and z1 < 2 ** 26:
                return y0, k0, z1, k1


@pytest.mark.parametrize("D,Hq", [(128, 4), (128, 8), (64, 8)])
def test_columns_of_a_row_agree(D, Hq):
    """Where a row is several columns of a product, each with groups of its own, all of them have to follow the row's maximum alike, also where the order of their sums decides whether it
    is followed."""
    y0, k0, y1, k1 = between()
    x = Served4([255], [1], Hq, 1, D, 16, seed=3)
    x.codes[0].zero_()
    x.x[0][0].zero_()
    half = 32 if Hq == 4 or D == 64 else 64  # a column's elements
    p, u = int(x.table[0, 130 // 16]), 130 % 16  # (the second strip of its wavefront)
    code = torch.zeros(1, 1, D, dtype=torch.long, device=DEV)
    code[..., :32], code[..., half: half + 32] = 2, 2  # levels of 1
    x.codes[0][p, :, u] = plain.pack(code, False)[0]
    x.steps[0][p, :, u] = 1.0
    x.steps[0][p, :, u, 0], x.steps[0][p, :, u, half // 32] = k0, k1
    x.x[0][0][130] = plain.value(code, x.steps[0][p, :, u][None])[0]
    x.q.zero_()
    for y, at in ((y0, 0), (y1, half)):  # eight bits an element
        for e in range(4):
            x.q[0, :, at + e] = float(y >> 8 * e & 255) * 2.0 ** (8 * e - 24)
    scale = next(s for s in (np.float32(0.6931472) + np.float32(i * 2.0 ** -24) for i in range(-8, 9)) if np.float32(s * np.float32(1.4426950408889634)) == 1)
    x.chunk = sb.Chunk(x.cu_dev, x.cached, Hq, 1, 1, 256, softmax_scale=float(scale))
    x.check(scale=float(scale))


def test_scores_of_minus_infinity_and_far_apart():
    """Steps so large that scores overflow, rows all of whose scores are -infinity, and scores thousands apart."""
    x = Served4([40], [3], 2, 1, 64, 16, "f32")
    x.q.fill_(1.0)
    x.codes[0].fill_(0xff)  # -6 everywhere
    x.steps[0].fill_(2.0 ** 124)
    o, lse = x.attend()
    assert float(o.abs().max()) == 0 and bool((lse == -INF).all())
    x = Served4([700], [2], 4, 1, 128, 16)
    x.q.mul_(200.0)
    x.check()


def test_scale_and_repeats():
    x = Served4([900, 33], [3, 40], 8, 2, 128, 16)
    x.chunk = sb.Chunk(x.cu_dev, x.cached, 8, x.rows, 40, 933, softmax_scale=0.3)
    a = x.check(scale=float(np.float32(0.3)))
    for _ in range(3):
        b = x.attend()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("length", [1, 100, 100000])
def test_the_length_is_a_hint(length):
    x = Served4([900, 2000], [1, 1], 8, 2, 64, 16)
    x.chunk = sb.Chunk(x.cu_dev, x.cached, 8, x.rows, 1, length)
    x.check()


def test_rows_beyond_max_new_are_left():
    x = Served4([50, 60], [10, 3], 4, 2, 64, 16)
    x.chunk = sb.Chunk(x.cu_dev, x.cached, 4, 13, 4, 100)
    o, lse = x.attend()
    assert bool(torch.isnan(o[4:10]).all()) and not bool(torch.isnan(o[:4]).any() | torch.isnan(o[10:]).any()) and bool(torch.isnan(lse[:, 4:10]).all())


def test_pages_behind_four_gigabytes():
    """Codes and steps whose offsets pass 32 bits: the last pages of a cache of 9 GB."""
    Hkv, D, page = 8, 128, 1024
    pages = (9 << 30) // (Hkv * page * D // 2) + 3
    x = Served4([1500], [1], 16, Hkv, D, page)
    big = [torch.empty(pages, Hkv, page, D // 2, dtype=torch.uint8, device=DEV) for _ in range(2)]
    steps = [torch.empty(pages, Hkv, page, D // 32, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32, device=DEV)
    for w in (0, 1):
        for j in (0, 1):
            old = int(x.table[0, j])
            big[w][pages - 1 - j], steps[w][pages - 1 - j] = x.codes[w][old], x.steps[w][old]
    x.cache = sb.Cache4(big[0], big[1], steps[0], steps[1], table)
    x.check()
    k, v = normal(1, 1, Hkv, D), normal(2, 1, Hkv, D)
    kh = sb.sb_cache4_append(x.cache, x.chunk, k, v, held=True)[1]
    assert torch.equal(kh[0].double(), plain.held(big[0][pages - 2, :, 1500 - 1024], steps[0][pages - 2, :, 1500 - 1024], False))


# ---------------------------------------------------------------- together, as a serving loop has them
def test_a_serving_loop_in_a_captured_graph():
    """Tables, append with positions of three axes, attention: captured once, replayed as requests grow, on a stream of its own; every replay against the plain form."""
    S, Hq, Hkv, D, page, T, most = 5, 8, 2, 128, 16, 60, 20
    pool = sb.PagePool.empty(S, 12, 40, page)
    codes = [torch.full((40, Hkv, page, D // 2), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    steps = [nan(40, Hkv, page, D // 32) for _ in range(2)]
    cached, added = (torch.zeros(S, dtype=torch.int32, device=DEV) for _ in range(2))
    q, k, v, pos = normal(1, T, Hq, D), normal(2, T, Hkv, D), normal(3, T, Hkv, D), positions(4, 3, T, 5000)
    rope, axes = sb.Rope(D), sb.RopeAxes((16, 24, 24))
    cache = sb.Cache4(codes[0], codes[1], steps[0], steps[1], pool.page_table)
    out = sb.sb_cache_tables(pool, cached, added, T)
    chunk = sb.Chunk(out[0], cached, Hq, T, most, 12 * page)
    ws = torch.empty(max(256, sb.sb_cache4_attn_ws_bytes(cache, chunk, 90, 4)), dtype=torch.uint8, device=DEV)
    qn, o, lse = nan(T, Hq, D), nan(T, Hq, D), nan(Hq, T, dtype=torch.float32)

    def step():
        sb.sb_cache_tables(pool, cached, added, T, *out)
        sb.sb_cache4_append(cache, chunk, k, v, rope=rope, axes=axes, positions=pos, q=q, q_out=qn)
        sb.sb_cache4_attn(cache, chunk, qn, 90, 4, o=o, lse=lse, ws=ws)
    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    have, held = [0] * S, [[[], []] for _ in range(S)]
    for i, n in enumerate(([20, 0, 3, 17, 1], [1, 20, 4, 1, 1], [20, 1, 1, 20, 1], [1, 1, 20, 1, 4], [1, 1, -1, 20, 1], [20, 20, 5, 1, 1])):
        new = [max(m, 0) for m in n]
        for x, seed in ((q, 10), (k, 20), (v, 30)):
            x.copy_(normal(seed + i, *x.shape))
        cached.copy_(torch.tensor(have, dtype=torch.int32))
        added.copy_(torch.tensor(n, dtype=torch.int32))
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        cu = out[0].tolist()
        assert cu[-1] == sum(new) and int(out[3][0]) == 0
        turned_k = turned(k.double(), pos, rope, axes, True)[0].float()
        for s in range(S):
            if n[s] < 0:
                held[s], have[s] = [[], []], 0
                continue
            rows = slice(cu[s], cu[s + 1])
            for w, y in ((0, turned_k[rows]), (1, v[rows].float())):
                st = plain.step_of(y)
                held[s][w].append(plain.value(plain.code_of(y, st), st))
            if new[s]:
                a, u = have[s], torch.arange(have[s] + new[s], device=DEV)
                r = ref.Attention(qn[rows].double(), torch.cat(held[s][0]), torch.cat(held[s][1]), ref.visible(u[a:], u, 90, 4), D ** -0.5, ref.HALF[torch.bfloat16])
                ref.check("o", o[rows], r.o, r.o_tol)
                ref.check("lse", lse[:, rows], r.lse, r.lse_tol)
            have[s] += new[s]
        assert bool(torch.isnan(o[cu[-1]:]).all())


def test_a_prompt_beside_its_held_values():
    """A first prompt's attention over the cache, and window attention over the packed values as the append says they are held: the same but for their roundings."""
    lens, Hq, Hkv, D = (300, 45), 8, 2, 128
    x = Served4([0, 0], list(lens), Hq, Hkv, D, 16, fill=False)
    q, kh, vh = sb.sb_cache4_append(x.cache, x.chunk, normal(1, 345, Hkv, D), normal(2, 345, Hkv, D), rope=sb.Rope(D), q=x.q, held=True)
    pb = batch(lens, Hq, Hkv, D)
    want = sb.sb_window_attn_fwd(pb, 64, 3, q, kh, vh)
    got = sb.sb_cache4_attn(x.cache, x.chunk, q, 64, 3)
    for s, (a, n) in enumerate(((0, 300), (300, 45))):
        u = torch.arange(n, device=DEV)
        r = ref.Attention(q[a: a + n].double(), kh[a: a + n].double(), vh[a: a + n].double(), ref.visible(u, u, 64, 3), D ** -0.5, ref.HALF[torch.bfloat16])
        for name, y in (("packed", want), ("paged", got)):
            ref.check(name, y[0][a: a + n], r.o, r.o_tol)
            ref.check(name, y[1][:, a: a + n], r.lse, r.lse_tol)


def test_two_calls_at_once():
    """Two batches over one cache on two streams, each with a workspace of its own."""
    x, streams = Served4([3000, 2500], [1, 1], 8, 2, 128, 64), [torch.cuda.Stream() for _ in range(2)]
    want = x.attend(), x.attend(500, 4)
    got = [None, None]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = sb.sb_cache4_attn(x.cache, x.chunk, x.q, *((NONE, 0), (500, 4))[i])
        torch.cuda.synchronize()
        for i in (0, 1):
            assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1])


def test_binding_refusals():
    x = Served4([10], [1], 4, 2, 64, 16)
    with pytest.raises(sb.SparseBalError, match="^q: "):
        sb.sb_cache4_attn(x.cache, x.chunk, x.q.float())
    with pytest.raises(sb.SparseBalError, match="^ws: "):
        y = Served4([5000], [1], 4, 2, 64, 16)
        sb.sb_cache4_attn(y.cache, y.chunk, y.q, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(sb.SparseBalError, match="axes without positions"):
        sb.sb_cache4_append(x.cache, x.chunk, normal(1, 1, 2, 64), normal(1, 1, 2, 64), rope=sb.Rope(64), axes=sb.RopeAxes((32,)))
    with pytest.raises(sb.SparseBalError, match="^positions: shape"):
        sb.sb_cache4_append(x.cache, x.chunk, normal(1, 1, 2, 64), normal(1, 1, 2, 64), rope=sb.Rope(64), axes=sb.RopeAxes((16, 16)), positions=positions(1, 1, 1))
    with pytest.raises(sb.SparseBalError, match="^k_step: shape"):
        sb.Cache4(x.codes[0], x.codes[1], x.steps[0][..., :1], x.steps[1], x.table)
    with pytest.raises(sb.SparseBalError, match="in the place of inputs"):
        q = x.q.clone()
        sb.sb_cache4_append(x.cache, x.chunk, normal(1, 1, 2, 64), normal(1, 1, 2, 64), q=q, q_out=q)
