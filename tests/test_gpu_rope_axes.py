"""Rotary positions with several axes on the GPU, forward, backward and in front of a cache, against the plain 64-bit form (operator_reference.py, where the bound is derived)."""
import math

import pytest
import torch

import operator_reference as ref
from paper_2604_13847_amd import binding as sb
from test_gpu_operators import DEV, TYPE, Served, batch, nan, normal

pytestmark = pytest.mark.gpu


def positions(seed, axes, n, most=1 << 20):
    return torch.randint(0, most, (axes, n), generator=torch.Generator(device=DEV).manual_seed(seed), dtype=torch.int32, device=DEV)


def turned(x, pos, rope, axes, half_layout, backward=False):
    """One pair's axis at a time: operator_reference.turn of the axis' own positions, of which the pairs of that axis are taken."""
    n = rope.c.rot_dim // 2
    turns = torch.tensor(list(rope.c.turns[:n]), dtype=torch.float64, device=DEV)
    y, tol = x.clone(), torch.zeros_like(x)
    for a in range(axes.c.num_axes):
        pairs = torch.tensor([i for i in range(n) if axes.c.axis[i] == a], dtype=torch.long, device=DEV)
        z, t = ref.turn(x, pos[a], turns, rope.c.amplitude, half_layout, backward)
        for at in ((pairs, pairs + n) if half_layout else (2 * pairs, 2 * pairs + 1)):
            y[..., at], tol[..., at] = z[..., at], t[..., at]
    return y, tol


CASES = [(128, (16, 24, 24), 0), (128, (24, 20, 20), 1), (64, (11, 21), 0), (64, (8, 8, 8, 8), 1), (48, (0, 20, 4), 1), (2, (1,), 0), (22, (5, 0, 6), 0), (62, (30, 1), 1),
         (32, (2, 2, 2, 2, 2, 2, 2, 2), 1)]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,pairs,order", CASES)
def test_turn(rot, pairs, order, dtype, layout):
    t = TYPE[dtype][0]
    for D, Hq, Hkv, lens in ((128, 5, 1, (1, 130, 0, 7)), (64, 14, 2, (300, 33))):
        if rot > D:
            continue
        pb = batch(lens, Hq, Hkv, D, dtype)
        rope, axes = sb.Rope(rot, layout=layout), sb.RopeAxes(pairs, order=order)
        pos = positions(rot, len(pairs), pb.T)
        q, k = normal(1, pb.T, Hq, D, dtype=t), normal(2, pb.T, Hkv, D, dtype=t)
        for backward in (False, True):
            got = sb.sb_rope_axes_apply(pb, rope, axes, pos, q, k, backward=backward)
            for g, x in zip(got, (q, k)):
                r, tol = turned(x.double(), pos, rope, axes, layout == 0, backward)
                ref.check("turned", g, r, tol + ref.HALF[t] * r.abs())
                assert torch.equal(g[..., rot:], x[..., rot:])


def test_equal_positions_are_one_axis():
    """Text: the same position on every axis turns as sb_rope_apply does, bit for bit, whatever the axes' shares."""
    pb = batch((70, 200, 1), 8, 2, 128)
    q, k = normal(1, pb.T, 8, 128), normal(2, pb.T, 2, 128)
    pos = positions(3, 1, pb.T)
    rope = sb.Rope(128, scaling=sb.SB_ROPE_YARN, factor=4.0, original_length=4096.0)
    want = sb.sb_rope_apply(pb, rope, q, k, positions=pos[0].contiguous())
    for pairs, order in (((64,), 0), ((16, 24, 24), 0), ((30, 30, 4), 1)):
        got = sb.sb_rope_axes_apply(pb, rope, sb.RopeAxes(pairs, order=order), pos.expand(len(pairs), -1).contiguous(), q, k)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_frequencies_that_start_anew():
    """Two axes of an image, each turned as if its part of the head were a head of its own."""
    pb = batch((100,), 2, 2, 128)
    q, pos = normal(1, 100, 2, 128, dtype=torch.bfloat16), positions(4, 2, 100, 1000)
    one = sb.Rope(64, layout=1)
    joint = sb.Rope.joined([one, one])
    assert joint.c.rot_dim == 128
    got = sb.sb_rope_axes_apply(pb, joint, sb.RopeAxes((32, 32)), pos, q, None)[0]
    part = batch((100,), 2, 2, 64)
    for a in (0, 1):
        want = sb.sb_rope_apply(part, one, q[..., 64 * a: 64 * a + 64].contiguous(), None, positions=pos[a].contiguous())[0]
        assert torch.equal(got[..., 64 * a: 64 * a + 64], want)


def test_slices_offsets_and_places():
    """Queries and keys as slices of a fused projection, off 16-byte boundaries, one without the other, in place."""
    pb = batch((33, 90), 6, 2, 64)
    rope, axes, pos = sb.Rope(64), sb.RopeAxes((10, 11, 11), order=1), positions(5, 3, 123)
    fused = normal(1, 123, 10, 64)
    q, k = fused[:, :6], fused[:, 6:8]
    want = sb.sb_rope_axes_apply(pb, rope, axes, pos, q.contiguous(), k.contiguous())
    got = sb.sb_rope_axes_apply(pb, rope, axes, pos, q, k)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    odd = torch.empty(123 * 6 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(123, 6, 64)
    odd.copy_(q)
    assert torch.equal(sb.sb_rope_axes_apply(pb, rope, axes, pos, odd, None)[0], want[0])
    assert torch.equal(sb.sb_rope_axes_apply(pb, rope, axes, pos, None, k)[1], want[1])
    a, b = q.contiguous(), k.contiguous()
    sb.sb_rope_axes_apply(pb, rope, axes, pos, a, b, q_out=a, k_out=b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_backward_is_the_gradient():
    """Against differences of the forward (a turn is linear, so they are exact but for the rounding to float32), and back again."""
    pb = batch((40,), 2, 1, 64, "f32")
    rope, axes, pos = sb.Rope(48, layout=1), sb.RopeAxes((7, 9, 8)), positions(6, 3, 40, 5000)
    q, d = normal(1, 40, 2, 64, dtype=torch.float32), normal(2, 40, 2, 64, dtype=torch.float32)
    grad = sb.sb_rope_axes_apply(pb, rope, axes, pos, d, None, backward=True)[0]
    for seed in range(5):
        e = normal(10 + seed, 40, 2, 64, dtype=torch.float32)
        up, down = (sb.sb_rope_axes_apply(pb, rope, axes, pos, q + s * e, None)[0].double() for s in (1, -1))
        # 2 * 5120 products of about one, each off by at most 2^-24 |value| 8 (the turn) and 2 (sums and rounding): far below a thousandth
        assert abs(float(((up - down) / 2 * d.double()).sum() - (grad.double() * e.double()).sum())) < 5120 * 2.0 ** -24 * 10 * 4
    back = sb.sb_rope_axes_apply(pb, rope, axes, pos, sb.sb_rope_axes_apply(pb, rope, axes, pos, q, None)[0], None, backward=True)[0]
    assert float((back - q).abs().max()) <= 2 * 8 * 2 * 2.0 ** -24 * math.sqrt(2) * float(q.abs().max())


@pytest.mark.parametrize("dtype,D,page", [("bf16", 128, 16), ("f32", 64, 64), ("bf16", 64, 32)])
def test_append(dtype, D, page):
    """Keys turned by their axes go where the tokens' order says, and what no token owns is left alone."""
    x = Served([40, 0, 3, 500], [1, 70, 0, 33], 6, 2, D, page, dtype, spare_rows=3, fill=False)
    t, n = TYPE[dtype][0], len(x.q)
    rope, axes, pos = sb.Rope(D, layout=1), sb.RopeAxes((D // 4, D // 8, D // 8), order=1), positions(7, 3, n)
    k, v, qn = normal(20, n, 2, D, dtype=t), normal(21, n, 2, D, dtype=t), nan(n, 6, D, dtype=t)
    sb.sb_cache_append_axes(x.cache, x.chunk, k, v, rope, axes, pos, q=x.q, q_out=qn)
    pb = batch((n,), 6, 2, D, dtype)
    want = sb.sb_rope_axes_apply(pb, rope, axes, pos, x.q, k)
    assert torch.equal(qn[: x.rows], want[0][: x.rows]) and bool(torch.isnan(qn[x.rows:]).all())
    seen = torch.zeros(x.k_pages.shape[0], page, dtype=torch.bool, device=DEV)
    for s, (a, m) in enumerate(zip(x.have, x.new)):
        u = torch.arange(a, a + m, device=DEV)
        p = x.table[s, u // page].long()
        rows = slice(x.cu[s], x.cu[s + 1])
        assert torch.equal(x.k_pages[p, :, u % page], want[1][rows]) and torch.equal(x.v_pages[p, :, u % page], v[rows])
        seen[p, u % page] = True
    assert bool(torch.isnan(x.k_pages.transpose(1, 2)[~seen]).all()) and bool(torch.isnan(x.v_pages.transpose(1, 2)[~seen]).all())
