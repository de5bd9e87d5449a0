"""Rotary positions, window attention and attention over a paged cache on the GPU, against their plain 64-bit forms (operator_reference.py, where the
bounds are derived)."""
import numpy as np
import pytest
import torch

import operator_reference as ref
from paper_2604_13847_amd import binding as sb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPE = {"bf16": (torch.bfloat16, sb.SB_BF16), "f32": (torch.float32, sb.SB_F32)}
NONE = 2 ** 31 - 1


def normal(seed, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), dtype=torch.float32, device=DEV).to(dtype)


def nan(*shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), dtype=dtype, device=DEV)


def batch(lens, Hq, Hkv, D, dtype="bf16", **kw):
    return sb.Problem(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), [1] * len(lens), Hq, Hkv, D, dtype=TYPE[dtype][1], device=DEV, **kw)


# ---------------------------------------------------------------- rotary positions
@pytest.mark.parametrize("rot,layout", [(64, 0), (64, 1), (32, 0), (48, 1), (2, 0), (2, 1), (10, 0), (22, 1), (62, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_rope(D, dtype, rot, layout):
    rot = rot * D // 64 if rot > 22 else rot
    t, half = TYPE[dtype][0], ref.HALF[TYPE[dtype][0]]
    lens, Hq, Hkv = (1, 0, 130, 64, 7), 6, 2
    pb = batch(lens, Hq, Hkv, D, dtype)
    rope = sb.Rope(rot, layout=layout, scaling=sb.SB_ROPE_YARN if rot > 4 else 0, factor=3.0, original_length=2048.0)
    turns = torch.tensor(rope.c.turns[: rot // 2], dtype=torch.float64, device=DEV)
    far = torch.randint(0, 2 ** 31 - 1, (pb.T,), generator=torch.Generator(device=DEV).manual_seed(3), dtype=torch.int32, device=DEV)
    near = torch.cat([torch.arange(n, dtype=torch.int32, device=DEV) for n in lens])
    fused = normal(1, pb.T, (Hq + 2 * Hkv) * D, dtype=t)          # a projection's output: q, k, v of a token in a row
    q, k = fused[:, : Hq * D].view(pb.T, Hq, D), fused[:, Hq * D: (Hq + Hkv) * D].view(pb.T, Hkv, D)
    for pos, positions in ((near, None), (far, far)):
        for backward in (False, True):
            out = sb.sb_rope_apply(pb, rope, q, k, positions=positions, backward=backward, q_out=nan(*q.shape, dtype=t), k_out=nan(*k.shape, dtype=t))
            for x, got in zip((q, k), out):
                want, tol = ref.turn(x.double(), pos, turns, rope.c.amplitude, layout == 0, backward)
                # positions up to 2^31: the float64 product is off by half a step of up to 2^31 / 2 pi revolutions, 2 pi 2^-25 radians at the first pair
                if positions is not None:
                    tol = tol * 2
                ref.check("rope", got, want, tol + half * want.abs() * (tol > 0))
    # in place, one tensor alone, tokens in one piece
    qc = q.contiguous()
    want = sb.sb_rope_apply(pb, rope, qc, None)[0]
    assert sb.sb_rope_apply(pb, rope, qc, None, q_out=qc) == (qc, None) and torch.equal(qc, want)


def test_rope_backward_is_the_gradient():
    """<rope(x), w> and <x, rope_backward(w)> are the same number: the transpose of a linear map."""
    pb = batch((50, 33), 4, 1, 64, "f32")
    for layout in (0, 1):
        rope = sb.Rope(48, layout=layout, scaling=sb.SB_ROPE_YARN, factor=4.0, original_length=64.0)
        x, w = normal(1, pb.T, 4, 64, dtype=torch.float32), normal(2, pb.T, 4, 64, dtype=torch.float32)
        y, z = sb.sb_rope_apply(pb, rope, x, None)[0], sb.sb_rope_apply(pb, rope, w, None, backward=True)[0]
        a, b = (y.double() * w.double()).sum(), (x.double() * z.double()).sum()
        tol = 2 * 10 * ref.EPS * rope.c.amplitude * 2 * float((x.abs().double() * w.abs().double()).sum())  # every term off by 10 steps of |x| + |y|, both ways
        assert abs(float(a - b)) <= tol, (float(a), float(b), tol)


@pytest.mark.parametrize("offset", [0, 1])
def test_rope_many_sequences_and_unaligned(offset):
    """More sequences than lanes, empty ones among them; an input that starts off a 16-byte boundary."""
    lens = [0, 3, 1, 0, 5] * 40
    pb = batch(lens, 3, 1, 64)
    buf = normal(5, pb.T * 3 * 64 + 8)
    q = buf[offset: offset + pb.T * 3 * 64].view(pb.T, 3, 64)
    rope = sb.Rope(64)
    turns = torch.tensor(rope.c.turns[:32], dtype=torch.float64, device=DEV)
    pos = torch.cat([torch.arange(n, device=DEV) for n in lens])
    want, tol = ref.turn(q.double(), pos, turns, 1.0, True)
    ref.check("q", sb.sb_rope_apply(pb, rope, q, None)[0], want, tol + ref.HALF[torch.bfloat16] * want.abs())


# ---------------------------------------------------------------- window attention
def run_window(lens, Hq, Hkv, D, window, sinks, dtype, seed=0, scale=0.0, size=1.0):
    t = TYPE[dtype][0]
    pb = batch(lens, Hq, Hkv, D, dtype, softmax_scale=scale)
    q, k, v, do = (normal(10 * seed + i, pb.T, h, D, dtype=t) * (size if i < 2 else 1) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    out = dict(o=nan(*q.shape, dtype=t), lse=nan(Hq, pb.T, dtype=torch.float32))
    sb.sb_window_attn_fwd(pb, window, sinks, q, k, v, **out)
    grads = dict(dq=nan(*q.shape, dtype=t), dk=nan(*k.shape, dtype=t), dv=nan(*k.shape, dtype=t))
    sb.sb_window_attn_bwd(pb, window, sinks, q, k, v, out["o"], out["lse"], do, **grads)
    return pb, (q, k, v, do), {**out, **grads}


def check_window(pb, x, got, window, sinks, half, scale=None, values=("o", "dq", "dk", "dv")):
    q, k, v, do = (a.double() for a in x)
    scale = scale or pb.D ** -0.5
    for a, b in zip(pb.cu_host[:-1], pb.cu_host[1:]):
        a, b = int(a), int(b)
        if a == b:
            continue
        u = torch.arange(b - a, device=DEV)
        r = ref.Attention(q[a:b], k[a:b], v[a:b], ref.visible(u, u, window, sinks), scale, half, do[a:b])
        ref.check("lse", got["lse"][:, a:b], r.lse, r.lse_tol)
        for n in values:
            ref.check(n, got[n][a:b], getattr(r, n), getattr(r, n + "_tol"))


SHAPES = [((1,), 4, 2, 128, 1, 0), ((1, 2, 0, 3), 8, 1, 64, 2, 1), ((64, 65, 63, 128, 129), 4, 4, 128, 64, 0), ((64, 65, 63, 128, 129), 4, 2, 64, 65, 5),
          ((200, 31, 33), 7, 1, 128, 17, 3), ((300,), 14, 2, 64, 1, 0), ((300,), 6, 2, 128, 1, 70), ((257, 90), 8, 2, 128, 100, 64), ((500, 12), 4, 1, 128, 128, 65),
          ((500,), 2, 2, 64, 63, 129), ((700, 1, 300), 4, 2, 128, 250, 4), ((700,), 10, 2, 64, NONE, 0), ((333, 500), 32, 8, 128, 400, NONE),
          ((520,), 16, 2, 128, NONE, 7), ((1950, 60), 2, 1, 128, 40, 70), ((150, 9), 40, 1, 128, 33, 5), ((70,), 100, 1, 64, 20, 3), ((1, 60), 33, 1, 128, 64, 2), ((1800,), 3, 1, 64, 300, 600), ((450,), 1, 1, 64, 449, 1), ((900,), 3, 1, 128, 129, 200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,Hq,Hkv,D,window,sinks", SHAPES)
def test_window_attention(lens, Hq, Hkv, D, window, sinks, dtype):
    pb, x, got = run_window(lens, Hq, Hkv, D, window, sinks, dtype)
    check_window(pb, x, got, window, sinks, ref.HALF[TYPE[dtype][0]])


def test_window_attention_scores_that_grow():
    """Keys whose scores grow along the sequence, so that every tile moves the softmax's reference, and scores of hundreds."""
    for D, dtype in ((128, "bf16"), (64, "bf16"), (128, "f32")):
        t = TYPE[dtype][0]
        pb = batch((600, 40), 4, 2, D, dtype)
        q, k, v, do = (normal(i, pb.T, h, D, dtype=t) for i, h in enumerate((4, 2, 2, 4)))
        k = (k * torch.linspace(0.1, 12, pb.T, device=DEV)[:, None, None]).to(t)
        o, lse = sb.sb_window_attn_fwd(pb, 350, 3, q, k, v)
        dq, dk, dv = sb.sb_window_attn_bwd(pb, 350, 3, q, k, v, o, lse, do)
        check_window(pb, (q, k, v, do), dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv), 350, 3, ref.HALF[t])


def test_window_attention_scale_and_many_sequences():
    lens = [3, 0, 70, 1, 20] * 27
    pb, x, got = run_window(lens, 4, 2, 64, 15, 2, "bf16", scale=0.3)
    check_window(pb, x, got, 15, 2, ref.HALF[torch.bfloat16], scale=float(np.float32(0.3)))


def test_window_gradients_against_differences():
    """<gradient, direction> against central differences of the loss <O, dO>, computed in float64 from the float32 forward's definition."""
    lens, Hq, Hkv, D, window, sinks = (90, 41), 4, 2, 64, 23, 5
    pb, x, got = run_window(lens, Hq, Hkv, D, window, sinks, "f32", size=0.5)
    q, k, v, do = (a.double() for a in x)

    def loss(q, k, v):
        total = 0.0
        for a, b in zip(pb.cu_host[:-1], pb.cu_host[1:]):
            u = torch.arange(int(b - a), device=DEV)
            total += float((ref.Attention(q[a:b], k[a:b], v[a:b], ref.visible(u, u, window, sinks), D ** -0.5, 0.0).o * do[a:b]).sum())
        return total

    for i, name in enumerate(("dq", "dk", "dv")):
        w = normal(77 + i, *x[i].shape, dtype=torch.float32).double()
        eps = 1e-4
        args = [q, k, v]
        plus, minus = list(args), list(args)
        plus[i], minus[i] = args[i] + eps * w, args[i] - eps * w
        slope = (loss(*plus) - loss(*minus)) / (2 * eps)
        mine = float((got[name].double() * w).sum())
        assert abs(mine - slope) <= 1e-5 * float((got[name].double().abs() * w.abs()).sum()), (name, mine, slope)


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (64, 4, 2)])
def test_window_attention_is_repeatable(D, Hq, Hkv):
    runs = [run_window((2000, 300), Hq, Hkv, D, 300, 70, "bf16")[2] for _ in range(3)]
    for n in runs[0]:
        assert bool(torch.isfinite(runs[0][n]).all()), n
        assert all(torch.equal(runs[0][n], r[n]) for r in runs[1:]), n


def test_window_attention_with_a_whole_window_is_dense_block_sparse_attention():
    """All blocks kept and a window of everything: the same operator by two paths of the library."""
    lens, Hq, Hkv, D = (300, 130), 8, 2, 128
    pb = sb.Problem(np.cumsum([0, *lens]).astype(np.int32), [100] * 2, Hq, Hkv, D, device=DEV)
    q, k, v, do = (normal(i, pb.T, h, D) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    _, rowptr, idx = sb.sb_score_select(pb, q, k)
    plan = sb.sb_plan_worklist(pb, rowptr, idx)
    a = sb.sb_sparse_attn_fwd(pb, q, k, v, rowptr, idx, plan)
    b = sb.sb_window_attn_fwd(pb, NONE, 0, q, k, v)
    ga = sb.sb_sparse_attn_bwd(pb, q, k, v, *a, do, rowptr, idx, plan)
    gb = sb.sb_window_attn_bwd(pb, NONE, 0, q, k, v, *b, do)
    got = lambda f, g: dict(o=f[0], lse=f[1], dq=g[0], dk=g[1], dv=g[2])
    check_window(pb, (q, k, v, do), got(b, gb), NONE, 0, ref.HALF[torch.bfloat16])
    for x, y in zip((a[0], *ga), (b[0], *gb)):
        assert float((x.double() - y.double()).norm() / y.double().norm()) < 2 ** -7


# ---------------------------------------------------------------- the paged cache
class Served:
    """Sequences with `have` cached and `new` new tokens, in scattered pages; what no token owns is NaN."""

    def __init__(self, have, new, Hq, Hkv, D, page, dtype="bf16", spare_rows=0, seed=0, fill=True, spare_pages=0):
        t = TYPE[dtype][0]
        self.have, self.new, self.D, self.Hq, self.Hkv, self.page, self.dtype = have, new, D, Hq, Hkv, page, t
        S = len(have)
        need = [(a + n + page - 1) // page for a, n in zip(have, new)]
        pages = sum(need) + 2
        order = torch.randperm(pages, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).int()
        self.table = torch.full((S, max(need + [1]) + spare_pages), -1, dtype=torch.int32, device=DEV)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at: at + n]
            at += n
        self.k_pages, self.v_pages = nan(pages, Hkv, page, D, dtype=t), nan(pages, Hkv, page, D, dtype=t)
        self.k, self.v = ([normal(seed + 100 * i + j, a + n, Hkv, D, dtype=t) for i, (a, n) in enumerate(zip(have, new))] for j in (1, 2))
        if fill:
            for s in range(S):
                for x, p in ((self.k, self.k_pages), (self.v, self.v_pages)):
                    u = torch.arange(have[s] + new[s], device=DEV)
                    p[self.table[s, u // page].long(), :, u % page] = x[s]
        self.rows = sum(new)
        self.q = normal(seed + 7, self.rows + spare_rows, Hq, D, dtype=t)
        cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
        self.cu = [int(c) for c in cu]
        self.cache = sb.Cache(self.k_pages, self.v_pages, self.table)
        self.chunk = sb.Chunk(cu, torch.tensor(have, dtype=torch.int32, device=DEV), Hq, self.rows + spare_rows, max(new + [0]), max([a + n for a, n in zip(have, new)] + [0]))

    def attend(self, window=NONE, sinks=0):
        o, lse = nan(*self.q.shape, dtype=self.dtype), nan(self.Hq, len(self.q), dtype=torch.float32)
        sb.sb_cache_attn(self.cache, self.chunk, self.q, window, sinks, o=o, lse=lse)
        return o, lse

    def check(self, window=NONE, sinks=0, there=None):
        o, lse = self.attend(window, sinks)
        for s, (a, n) in enumerate(zip(self.have, self.new)):
            rows = slice(self.cu[s], self.cu[s + 1])
            if n == 0:
                continue
            u = torch.arange(a + n, device=DEV)
            seen = ref.visible(torch.arange(a, a + n, device=DEV), u, window, sinks)
            if there is not None:
                seen = seen & there(s, u)
            r = ref.Attention(self.q[rows].double(), self.k[s].double(), self.v[s].double(), seen, self.D ** -0.5, ref.HALF[self.dtype])
            ref.check("o", o[rows], r.o, r.o_tol)
            ref.check("lse", lse[:, rows], r.lse, r.lse_tol)
        assert bool(torch.isnan(o[self.rows:]).all()) and bool(torch.isnan(lse[:, self.rows:]).all())
        return o, lse


SERVED = [  # have, new, Hq, Hkv, D, page, window, sinks
    ([0], [1], 4, 2, 128, 16, NONE, 0), ([1, 63, 64, 65, 0], [1, 1, 1, 1, 1], 4, 4, 64, 16, NONE, 0), ([700, 5, 1300], [1, 1, 1], 32, 8, 128, 64, NONE, 0),
    ([4000], [1], 14, 2, 64, 32, NONE, 0), ([900, 2500], [1, 1], 7, 1, 128, 256, 300, 5), ([2000, 10, 555], [1, 1, 1], 16, 1, 128, 128, 64, 0),
    ([100, 0, 900], [3, 1, 5], 8, 2, 128, 16, NONE, 0), ([300, 0, 17], [40, 0, 1], 6, 2, 64, 64, 50, 20), ([0, 1000], [130, 257], 4, 1, 128, 64, NONE, 0),
    ([0], [600], 28, 4, 128, 32, 128, 4), ([513, 100], [64, 65], 3, 3, 64, 16, NONE, 0), ([3000], [33], 32, 8, 128, 16, 1000, 64), ([1500] * 70, [1] * 70, 2, 1, 64, 64, NONE, 0),
    # prompts and single tokens in one batch; a long cache and rows that fill one tile, two, and a few
    ([2000, 900, 30, 0], [1, 200, 1, 90], 8, 2, 128, 16, NONE, 0), ([5000, 4900, 3], [1, 2, 150], 4, 1, 64, 64, 2000, 10), ([9000], [12], 4, 1, 128, 64, NONE, 0),
    ([6000, 100], [8, 8], 8, 1, 64, 16, NONE, 0), ([700, 3], [1, 1], 40, 1, 128, 16, NONE, 0), ([700, 64], [1, 2], 100, 1, 64, 64, 200, 9), ([9500], [20], 8, 2, 128, 32, NONE, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,Hq,Hkv,D,page,window,sinks", SERVED)
def test_cache_attention(have, new, Hq, Hkv, D, page, window, sinks, dtype):
    Served(have, new, Hq, Hkv, D, page, dtype, spare_rows=3, spare_pages=2).check(window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_attention_without_pages(dtype):
    """Entries that are no page (-1, too large), inside a sequence and for a whole one: their keys are seen by no row."""
    for new in ([1, 1, 1], [70, 3, 20]):
        x = Served([500, 90, 300], new, 8, 2, 128, 32, dtype, spare_rows=1)
        x.table[0, 3], x.table[0, 7], x.table[1, :], x.table[2, -1] = -1, 10 ** 6, -5, 2 ** 31 - 1
        bad = x.table.clone()
        pages = len(x.k_pages)
        there = lambda s, u: (bad[s, u // 32] >= 0) & (bad[s, u // 32] < pages)
        o, lse = x.check(there=there)
        rows = slice(x.cu[1], x.cu[2])
        assert float(o[rows].abs().max()) == 0 and bool((lse[:, rows] == -float("inf")).all())


def test_cache_append_and_attend_in_pieces():
    """A prompt through rope and window attention at once, and the same prompt appended and attended in chunks of any size, down to single tokens."""
    Hq, Hkv, D, page, window, sinks = 8, 2, 128, 16, 100, 6
    lens = (330, 150)
    for layout, rot in ((0, 128), (1, 48)):
        rope = sb.Rope(rot, layout=layout, scaling=sb.SB_ROPE_BANDS, factor=4.0, original_length=128.0)
        pb = batch(lens, Hq, Hkv, D)
        q, k, v = (normal(i, pb.T, h, D) for i, h in enumerate((Hq, Hkv, Hkv)))
        qr, kr = sb.sb_rope_apply(pb, rope, q, k)
        whole = sb.sb_window_attn_fwd(pb, window, sinks, qr, kr, v)
        start = [0, lens[0]]
        x = Served([0, 0], [0, 0], Hq, Hkv, D, page, fill=False)
        pages = [sum((n + page - 1) // page for n in lens) + 2, Hkv, page, D]
        kp, vp = nan(*pages), nan(*pages)
        table = torch.full((2, 24), -1, dtype=torch.int32, device=DEV)
        table[0, :21], table[1, :10] = torch.arange(21, 0, -1), torch.arange(22, 32)
        cache = sb.Cache(kp, vp, table)
        have = [0, 0]
        for step in ((7, 64), (128, 1), (1, 0), (60, 30), (133, 54), (1, 1)):
            rows = torch.cat([torch.arange(start[s] + have[s], start[s] + have[s] + step[s], device=DEV) for s in (0, 1)])
            cu = torch.tensor([0, step[0], sum(step)], dtype=torch.int32, device=DEV)
            chunk = sb.Chunk(cu, torch.tensor(have, dtype=torch.int32, device=DEV), Hq, sum(step), max(step), max(h + n for h, n in zip(have, step)))
            qn = sb.sb_cache_append(cache, chunk, k[rows], v[rows], rope=rope, q=q[rows])
            assert torch.equal(qn, qr[rows])
            o, lse = sb.sb_cache_attn(cache, chunk, qn, window, sinks)
            for s in (0, 1):
                new = slice(int(cu[s]), int(cu[s + 1]))
                if step[s] == 0:
                    continue
                a, b = start[s], start[s] + have[s] + step[s]
                u = torch.arange(b - a, device=DEV)
                r = ref.Attention(qn[new].double(), kr[a:b].double(), v[a:b].double(), ref.visible(u[have[s]:], u, window, sinks), D ** -0.5, ref.HALF[torch.bfloat16])
                ref.check("o", o[new], r.o, r.o_tol)
                ref.check("lse", lse[:, new], r.lse, r.lse_tol)
                ref.check("whole", whole[0][start[s] + have[s]: b], r.o, r.o_tol)
            have = [h + n for h, n in zip(have, step)]
        assert have == list(lens)
        # what the pages hold, bit for bit
        for s in (0, 1):
            u = torch.arange(lens[s], device=DEV)
            p = table[s, u // page].long()
            assert torch.equal(kp[p, :, u % page], kr[start[s]: start[s] + lens[s]]) and torch.equal(vp[p, :, u % page], v[start[s]: start[s] + lens[s]])
        assert int(torch.isnan(kp).any(-1).sum()) == Hkv * (len(kp) * page - sum(lens))  # and nothing else was written


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_cache_append_leaves_alone_what_it_should(dtype, D):
    """Missing pages, rows behind the last sequence, rows beyond max_new; without rope, from strided inputs."""
    t = TYPE[dtype][0]
    x = Served([30, 0, 14], [5, 4, 9], 4, 2, D, 16, dtype, spare_rows=2, fill=False)
    x.table[1, 0] = -1
    x.table[2, 1] = len(x.k_pages)
    fused = normal(3, 20, 8 * D, dtype=t)
    k, v, q = fused[:, : 2 * D].view(20, 2, D), fused[:, 2 * D: 4 * D].view(20, 2, D), fused[:, 4 * D:].view(20, 4, D)
    x.chunk.c.max_new = 8
    q_out = nan(20, 4, D, dtype=t)
    sb.sb_cache_append(x.cache, x.chunk, k, v, q=q, q_out=q_out)
    assert torch.equal(q_out[:17], q[:17]) and bool(torch.isnan(q_out[17:]).all())   # rows 0 .. 16: five, four and eight of the nine
    written = torch.zeros(len(x.k_pages), 16, dtype=torch.bool, device=DEV)
    for s, rows in ((0, range(5)), (2, range(2))):                                   # sequence 2: tokens 14 and 15 have a page, 16 .. have none
        for i in rows:
            pos = x.have[s] + i
            p, at = int(x.table[s, pos // 16]), pos % 16
            written[p, at] = True
            assert torch.equal(x.k_pages[p, :, at], k[x.cu[s] + i]) and torch.equal(x.v_pages[p, :, at], v[x.cu[s] + i])
    for p in (x.k_pages, x.v_pages):
        assert torch.equal(~torch.isnan(p).any(-1).any(1), written)


def test_decoding_in_a_captured_graph():
    """One step of decoding as a graph, replayed as the lengths grow, with eager work in between: lengths and pages are read on the device."""
    Hq, Hkv, D, page, S, most = 8, 2, 128, 16, 3, 400
    kp, vp = torch.zeros(80, Hkv, page, D, dtype=torch.bfloat16, device=DEV), torch.zeros(80, Hkv, page, D, dtype=torch.bfloat16, device=DEV)
    table = torch.randperm(78, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).int().view(S, 26).contiguous()
    cache = sb.Cache(kp, vp, table)
    cached = torch.zeros(S, dtype=torch.int32, device=DEV)
    chunk = sb.Chunk(torch.arange(S + 1, dtype=torch.int32, device=DEV), cached, Hq, S, 1, most)
    rope = sb.Rope(D)
    q, k, v = normal(1, S, Hq, D), normal(2, S, Hkv, D), normal(3, S, Hkv, D)
    o, lse = nan(S, Hq, D), nan(Hq, S, dtype=torch.float32)
    ws = torch.empty(max(256, sb.sb_cache_attn_ws_bytes(cache, chunk, 150, 4)), dtype=torch.uint8, device=DEV)
    qn = nan(S, Hq, D)

    def step():
        sb.sb_cache_append(cache, chunk, k, v, rope=rope, q=q, q_out=qn)
        sb.sb_cache_attn(cache, chunk, qn, 150, 4, o=o, lse=lse, ws=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, lens in enumerate(([0, 5, 17], [1, 6, 18], [200, 399, 64], [399, 150, 151])):
        cached.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(normal(50 + i, S, Hq, D))
        k.copy_(normal(60 + i, S, Hkv, D))
        kp.copy_(normal(70 + i, *kp.shape))
        vp.copy_(normal(80 + i, *vp.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone(), kp.clone()
        o.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], lse) and torch.equal(got[2], kp)
        for s, a in enumerate(lens):
            u = torch.arange(a + 1, device=DEV)
            p = table[s, u // page].long()
            r = ref.Attention(qn[s: s + 1].double(), kp[p, :, u % page].double(), vp[p, :, u % page].double(), ref.visible(torch.tensor([a], device=DEV), u, 150, 4), D ** -0.5,
                              ref.HALF[torch.bfloat16])
            ref.check("o", o[s: s + 1], r.o, r.o_tol)


def test_training_pass_in_a_captured_graph():
    """Rotary positions, window attention and the gradients of both, captured and replayed, against the eager calls."""
    lens, Hq, Hkv, D = (500, 77), 8, 2, 128
    pb = batch(lens, Hq, Hkv, D)
    rope = sb.Rope(64, layout=sb.SB_ROPE_INTERLEAVED)
    q, k, v, do = (normal(i, pb.T, h, D) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    buf = [torch.empty_like(x) for x in (q, k, q, q, k, v)]
    lse = torch.empty(Hq, pb.T, dtype=torch.float32, device=DEV)
    need = sb.sb_window_ws_bytes(pb, 90, 70)
    ws = torch.empty(max(need) + 256, dtype=torch.uint8, device=DEV)

    def step():
        qr, kr, o, dq, dk, dv = buf
        sb.sb_rope_apply(pb, rope, q, k, q_out=qr, k_out=kr)
        sb.sb_window_attn_fwd(pb, 90, 70, qr, kr, v, o=o, lse=lse, ws=ws)
        sb.sb_window_attn_bwd(pb, 90, 70, qr, kr, v, o, lse, do, dq=dq, dk=dk, dv=dv, ws=ws)
        sb.sb_rope_apply(pb, rope, dq, dk, backward=True, q_out=dq, k_out=dk)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        q.copy_(normal(20 + i, *q.shape))
        do.copy_(normal(30 + i, *do.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*buf, lse)]
        for x in buf:
            x.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*buf, lse)))


def test_pages_behind_four_gigabytes():
    """A cache of 6 GB of keys and as much of values, its last pages in use; two sequences share their first page."""
    Hq, Hkv, D, page = 16, 8, 128, 64
    pages = 46000
    kp, vp = (torch.empty(pages, Hkv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert kp.numel() * 2 > 5 << 30
    table = torch.stack([pages - 1 - torch.arange(12, dtype=torch.int32, device=DEV), pages - 101 - torch.arange(12, dtype=torch.int32, device=DEV)])
    table[1, 0] = table[0, 0]
    rope = sb.Rope(D)
    for new in ([1, 1], [300, 1]):
        have = [400, 330]
        k, v = ([normal(20 * j + i, have[i] + new[i], Hkv, D) for i in (0, 1)] for j in (1, 2))
        k[1][:page], v[1][:page] = k[0][:page], v[0][:page]
        for x, p in ((k, kp), (v, vp)):
            for s in (0, 1):
                u = torch.arange(have[s], device=DEV)
                p[table[s, u // page].long(), :, u % page] = x[s][: have[s]]
        cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device=DEV)
        cache = sb.Cache(kp, vp, table)
        chunk = sb.Chunk(cu, torch.tensor(have, dtype=torch.int32, device=DEV), Hq, sum(new), max(new), 1000)
        q = normal(9, sum(new), Hq, D)
        kn, vn = (torch.cat([x[s][have[s]:] for s in (0, 1)]) for x in (k, v))
        qn = sb.sb_cache_append(cache, chunk, kn, vn, rope=rope, q=q)
        turns = torch.tensor(rope.c.turns[: D // 2], dtype=torch.float64, device=DEV)
        o, lse = sb.sb_cache_attn(cache, chunk, qn)
        for s in (0, 1):
            u = torch.arange(have[s] + new[s], device=DEV)
            held = kp[table[s, u // page].long(), :, u % page]
            turned, tol = ref.turn(k[s][have[s]:].double(), u[have[s]:], turns, 1.0, True)
            ref.check("k", held[have[s]:], turned, tol + ref.HALF[torch.bfloat16] * turned.abs())
            assert torch.equal(held[: have[s]], k[s][: have[s]])
            rows = slice(int(cu[s]), int(cu[s + 1]))
            r = ref.Attention(qn[rows].double(), held.double(), v[s].double(), ref.visible(u[have[s]:], u, NONE, 0), D ** -0.5, ref.HALF[torch.bfloat16])
            ref.check("o", o[rows], r.o, r.o_tol)
            ref.check("lse", lse[:, rows], r.lse, r.lse_tol)


def test_rows_behind_four_gigabytes():
    """540001 tokens of 32 query heads: queries, outputs and their gradients pass 4 GB each.  The last rows against the reference."""
    T, Hq, Hkv, D, window, tail = 540001, 32, 1, 128, 70, 300
    pb = batch((T,), Hq, Hkv, D)
    q, k, v, do = (normal(i, T, h, D) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    assert q.numel() * 2 > 4 << 30
    rope = sb.Rope(D)
    turned = sb.sb_rope_apply(pb, rope, q, k)
    turns = torch.tensor(rope.c.turns[: D // 2], dtype=torch.float64, device=DEV)
    for x, y in zip((q, k), turned):
        want, tol = ref.turn(x[-tail:].double(), torch.arange(T - tail, T, device=DEV), turns, 1.0, True)
        ref.check("rope", y[-tail:], want, tol + ref.HALF[torch.bfloat16] * want.abs())
    del turned, x, y
    o, lse = sb.sb_window_attn_fwd(pb, window, 0, q, k, v)
    dq, dk, dv = sb.sb_window_attn_bwd(pb, window, 0, q, k, v, o, lse, do)
    assert all(bool(torch.isfinite(x).all()) for x in (lse, dk, dv))
    a = T - tail
    u = torch.arange(a, T, device=DEV)
    r = ref.Attention(q[a:].double(), k[a:].double(), v[a:].double(), ref.visible(u, u, window, 0), D ** -0.5, ref.HALF[torch.bfloat16], do[a:].double())
    near = slice(window, None)   # rows that see none of the keys in front of the tail, and keys that all their rows are there for
    for n, x in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        ref.check(n, x[a:][near], getattr(r, n)[near], getattr(r, n + "_tol")[near])
    ref.check("lse", lse[:, a:][:, near], r.lse[:, near], r.lse_tol[:, near])


def test_on_another_stream():
    pb, x, got = run_window((700,), 4, 2, 128, 130, 9, "bf16")
    q, k, v, do = x
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o, lse = sb.sb_window_attn_fwd(pb, 130, 9, q, k, v)
        grads = sb.sb_window_attn_bwd(pb, 130, 9, q, k, v, o, lse, do)
    side.synchronize()
    for a, n in zip((o, lse, *grads), ("o", "lse", "dq", "dk", "dv")):
        assert torch.equal(a, got[n]), n


def test_binding_refusals():
    pb = batch((100,), 4, 2, 64)
    q, k = normal(1, 100, 4, 64), normal(2, 100, 2, 64)
    for args in ((q[:99], k, k), (q.float(), k, k), (q, k[:, :1], k), (q.transpose(0, 1).contiguous().transpose(0, 1), k, k), (q, k.cpu(), k)):
        with pytest.raises(sb.SparseBalError):
            sb.sb_window_attn_fwd(pb, 8, 0, *args)
    with pytest.raises(sb.SparseBalError, match="lse"):
        sb.sb_window_attn_fwd(pb, 8, 0, q, k, k, lse=torch.empty(4, 99, device=DEV))
    with pytest.raises(sb.SparseBalError, match="bytes"):
        sb.sb_window_attn_bwd(pb, 8, 0, q, k, k, q, torch.empty(4, 100, device=DEV), q, ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(sb.SparseBalError, match="positions"):
        sb.sb_rope_apply(pb, sb.Rope(64), q, k, positions=torch.zeros(100, device=DEV))
    x = Served([3, 4], [1, 1], 4, 2, 64, 16)
    with pytest.raises(sb.SparseBalError, match="rows"):
        sb.sb_cache_attn(sb.Cache(x.k_pages, x.v_pages, x.table[:1]), x.chunk, x.q)
    with pytest.raises(sb.SparseBalError, match="q_out"):
        sb.sb_cache_append(x.cache, x.chunk, k[:2], k[:2], q_out=q[:2])
