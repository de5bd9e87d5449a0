"""The four-bit cache on the GPU in the forms that small calls do not take: an append of thousands of tokens, bit for bit; attention in equal shares with windows and sinks, whose kernels
test_more_operator_forms.py names; and how far steps that are no numbers reach."""
import random

import pytest
import torch

import cache4_forms as forms
import four_bits as plain
import operator_reference as ref
from paper_2604_13847_amd import binding as sb
from test_gpu_cache4 import Served4
from test_gpu_operators import DEV, TYPE, nan, normal
from test_gpu_rope_axes import positions, turned

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- append of many tokens
MOST, SPARE = 48, 3  # tokens of a sequence that are taken; rows behind the last one


def lengths(total, seed):
    """Short sequences of all lengths, empty ones and some with more than MOST tokens among them: a wavefront's run of tokens crosses their borders everywhere."""
    rng, out = random.Random(seed), []
    while sum(out) < total - SPARE:
        out.append(min(rng.choice([0, 0, 1, 1, 2, 3, 5, 17, 33, 64]), total - SPARE - sum(out)))
    return out


@pytest.mark.parametrize("total", [2047, 2048, 4097, 8197, 12301])
@pytest.mark.parametrize("rot,layout,axes,dtype,Hq,Hkv,D,page,odd", [
    (128, 0, (16, 24, 24), "bf16", 10, 5, 128, 16, False), (64, 1, None, "bf16", 9, 9, 64, 32, False), (40, 0, None, "f32", 4, 2, 128, 16, False), (48, 1, (8, 8, 8), "f32", 3, 1, 64, 64, True),
    (None, 0, None, "bf16", 6, 2, 128, 16, True), (64, 0, (20, 12), "bf16", 2, 1, 64, 16, True)])
def test_append_of_many_tokens(rot, layout, axes, dtype, Hq, Hkv, D, page, odd, total):
    """Codes, steps, held values and queries of every token; what belongs to no sequence, is beyond max_new or has no page is left as it was, in the outputs or in the pages."""
    t, new = TYPE[dtype][0], lengths(total, total + D)
    S, rows = len(new), sum(new)
    have = torch.randint(-2, 90, (S,), generator=torch.Generator(device=DEV).manual_seed(1), dtype=torch.int32, device=DEV)
    count = torch.tensor(new, device=DEV)
    cu = torch.cat([count.new_zeros(1), count.cumsum(0)]).int()
    columns = (90 + MOST) // page + 1
    table = torch.randperm(S * columns, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).int().view(S, columns)
    table[3::7, 1], table[5::11, 0] = -1, S * columns
    codes = [torch.full((S * columns, Hkv, page, D // 2), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    steps = [nan(S * columns, Hkv, page, D // 32) for _ in range(2)]

    def tensor(seed, H):
        x = normal(seed, total, H, D, dtype=t)
        if odd:  # off a 16-byte boundary
            y = torch.empty(x.numel() + 1, dtype=t, device=DEV)[1:].view(x.shape)
            x = y.copy_(x)
        return x
    q, k, v = tensor(3, Hq), tensor(4, Hkv), tensor(5, Hkv)
    rope = sb.Rope(rot, layout=layout) if rot else None
    ax, pos = (sb.RopeAxes(axes), positions(6, len(axes), total, 1 << 16)) if axes else (None, None)
    qn, held = nan(total, Hq, D, dtype=t), [nan(total, Hkv, D, dtype=t) for _ in range(2)]
    cache, chunk = sb.Cache4(codes[0], codes[1], steps[0], steps[1], table, dtype=t), sb.Chunk(cu, have, Hq, total, MOST, 90 + MOST)
    sb.sb_cache4_append(cache, chunk, k, v, rope=rope, axes=ax, positions=pos, q=q, q_out=qn, held=True, k_held=held[0], v_held=held[1])

    of = torch.repeat_interleave(torch.arange(S, device=DEV), count)
    i = torch.arange(rows, device=DEV) - cu[:-1][of]
    taken, at = i < MOST, have.clamp_min(0)[of] + i
    assert int((~taken).sum()) > 16
    where = torch.zeros(1, total, dtype=torch.int32, device=DEV)
    where[0, :rows] = at
    if rope:
        one, at_axes = ax or sb.RopeAxes((rot // 2,)), pos if axes else where
        want_q, tol = turned(q.double(), at_axes, rope, one, layout == 0)
        ref.check("q", qn[:rows][taken], want_q[:rows][taken], (tol + ref.HALF[t] * want_q.abs())[:rows][taken])
        want_k = turned(k.double(), at_axes, rope, one, layout == 0)[0].float()
    else:
        assert torch.equal(qn[:rows][taken], q[:rows][taken])
        want_k = k.float()
    for x in (qn, *held):
        assert bool(torch.isnan(x[rows:]).all()) and bool(torch.isnan(x[:rows][~taken]).all())
    page_of = table[of, (at // page).clamp_max(columns - 1).long()].long()
    kept = taken & (page_of >= 0) & (page_of < S * columns)
    assert int((taken & ~kept).sum()) > 16
    p, u = page_of[kept], (at % page).long()[kept]
    seen = torch.zeros(S * columns, page, dtype=torch.bool, device=DEV)
    seen[p, u] = True
    for w, y in enumerate((want_k, v.float())):
        step = plain.step_of(y)
        code = plain.code_of(y, step)
        assert torch.equal(held[w][:rows][taken].double(), plain.value(code, step)[:rows][taken])
        assert torch.equal(codes[w][p, :, u], plain.pack(code[:rows][kept], w == 1)) and torch.equal(steps[w][p, :, u].double(), step[:rows][kept])
        assert bool((codes[w].transpose(1, 2)[~seen] == 255).all()) and bool(torch.isnan(steps[w].transpose(1, 2)[~seen]).all())


# ---------------------------------------------------------------- attention in equal shares
def same(a, b, x):
    return torch.equal(a[0][: x.rows], b[0][: x.rows]) and torch.equal(a[1][:, : x.rows], b[1][:, : x.rows])


@pytest.mark.parametrize("case", forms.SHARED_CHUNKS, ids=lambda c: "-".join(map(str, c)))
def test_chunks_in_equal_shares(case):
    have, new, Hq, Hkv, D, page, window, sinks = case
    x = Served4(have, new, Hq, Hkv, D, page, spare_rows=2)
    a = x.check(window, sinks)
    for _ in range(3):
        assert same(a, x.attend(window, sinks), x)


@pytest.mark.parametrize("case", forms.WHOLE_FLOATS + forms.SHARED_FLOATS, ids=lambda c: "-".join(map(str, c)))
def test_float32_chunks(case):
    have, new, Hq, Hkv, D, page, window, sinks = case
    x = Served4(have, new, Hq, Hkv, D, page, "f32", spare_rows=2)
    a = x.check(window, sinks)
    assert same(a, x.attend(window, sinks), x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,case", forms.SHARED_ROWS, ids=lambda c: "-".join(map(str, c)) if isinstance(c, tuple) else str(c))
def test_few_rows_in_equal_shares(rows, case, dtype):
    have, new, Hq, Hkv, D, page, window, sinks = case
    x = Served4(have, new, Hq, Hkv, D, page, dtype, spare_rows=2)
    a = x.check(window, sinks)
    for _ in range(3):
        assert same(a, x.attend(window, sinks), x)


# ---------------------------------------------------------------- steps that are no numbers
def spoil(x, s, u, g, c):
    """Step of group c of the value of token u of sequence s, KV head g."""
    x.steps[1][int(x.table[s, u // x.page]), g, u % x.page, c] = float("nan")


def spoiled(x, s, u, g, c, window, sinks):
    """[rows, Hq, D]: what has to become NaN by that."""
    out = torch.zeros(x.rows, x.Hq, x.D, dtype=torch.bool, device=DEV)
    t = torch.arange(x.have[s], x.have[s] + x.new[s], device=DEV)
    sees = ref.visible(t, torch.tensor([u], device=DEV), window, sinks)[:, 0]
    G = x.Hq // (x.codes[0].shape[1])
    out[x.cu[s]: x.cu[s + 1], g * G: (g + 1) * G, 32 * c: 32 * c + 32] = sees[:, None, None]
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("have,new,Hq,Hkv,D,page,window,sinks", [
    ([100, 333], [3, 1], 4, 2, 64, 16, forms.NONE, 0), ([100, 333], [4, 4], 2, 2, 128, 16, 40, 3), ([100, 70], [5, 2], 4, 4, 128, 32, 50, 0), ([100, 61], [6, 6], 10, 5, 64, 16, 33, 7),
    ([500, 9], [16, 16], 4, 2, 64, 64, 90, 40), ([500, 9], [16, 16], 4, 2, 128, 16, 90, 40), ([500, 9], [30, 20], 4, 2, 128, 16, 64, 35), ([4000, 3000], [16, 16], 8, 2, 128, 64, 3000, 70)])
def test_hidden_values_that_are_no_numbers_reach_no_row(have, new, Hq, Hkv, D, page, window, sinks, dtype):
    """Of few rows (all in float32): a drafted token behind the row's own, the token that has just left its window and the one behind the sinks may be no numbers, in whatever strip they
    lie; the rows that see them have NaN in the 32 elements that share the step, and nothing else."""
    x = Served4(have, new, Hq, Hkv, D, page, dtype)
    o, lse = x.attend(window, sinks)
    assert not bool(torch.isnan(o).any() | torch.isnan(lse).any())
    clean = [y.clone() for y in x.steps]
    for s in range(len(have)):
        first, last = have[s], have[s] + new[s] - 1
        places = {first, last, (first + last) // 2, first - window, last - window, (first + last) // 2 - window, first - window + 1, sinks - 1, sinks, 0}
        for n, u in enumerate(sorted(p for p in places if 0 <= p <= last)):
            g, c = n % Hkv, n % (D // 32)
            spoil(x, s, u, g, c)
            got, got_lse = x.attend(window, sinks)
            bad = spoiled(x, s, u, g, c, window, sinks)
            assert bool(torch.isnan(got[bad]).all()), (s, u)
            assert torch.equal(got[~bad], o[~bad]) and torch.equal(got_lse, lse), (s, u, torch.isnan(got).any(-1).any(-1).nonzero().flatten().tolist())
            x.steps[1].copy_(clean[1])
    # several at once, in all groups and heads, hidden from some rows and seen by others
    bad = torch.zeros_like(o, dtype=torch.bool)
    for s in range(len(have)):
        for u in (have[s] + new[s] - 1, have[s] + new[s] // 2, max(have[s] - window, 0)):
            for g in range(Hkv):
                for c in range(D // 32):
                    if (u + g + c) % 3:
                        spoil(x, s, u, g, c)
                        bad |= spoiled(x, s, u, g, c, window, sinks)
    got, got_lse = x.attend(window, sinks)
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], o[~bad]) and torch.equal(got_lse, lse)


@pytest.mark.parametrize("have,new,Hq,Hkv,D,window,sinks", [([130, 40], [300, 200], 4, 2, 64, forms.NONE, 0), ([130, 40], [300, 200], 8, 2, 128, 70, 3), ([3000, 2500, 3100], [300, 300, 299], 16, 8, 128, 2500, 70)])
def test_values_of_chunks_that_are_no_numbers_stay_in_their_tile(have, new, Hq, Hkv, D, window, sinks):
    """Of many rows: rows that see any key of the value's 64, and rows up to 31 tokens from such, may be NaN where the mask hides the value; no others, no other KV head and no other sequence."""
    x = Served4(have, new, Hq, Hkv, D, 16)
    o, lse = x.attend(window, sinks)
    clean = x.steps[1].clone()
    for s in range(2):
        t = torch.arange(have[s], have[s] + new[s], device=DEV)
        for n, u in enumerate((have[s] + new[s] - 1, have[s] + 64, have[s] + 100, max(have[s] - window, 1), 2)):
            g, c = n % Hkv, n % (D // 32)
            spoil(x, s, u, g, c)
            got, got_lse = x.attend(window, sinks)
            bad = spoiled(x, s, u, g, c, window, sinks)
            assert bool(torch.isnan(got[bad]).all()), (s, u)
            keys = torch.arange(u // 64 * 64, u // 64 * 64 + 64, device=DEV)
            near = ref.visible(t, keys, window, sinks).any(-1)
            near = ((t[:, None] - t).abs() <= 31)[:, near].any(-1)
            may = torch.zeros_like(bad)
            may[x.cu[s]: x.cu[s + 1], g * (Hq // Hkv): (g + 1) * (Hq // Hkv)] = near[:, None, None]
            assert not bool((bad & ~may).any())
            assert torch.equal(got[~may], o[~may]) and torch.equal(got_lse, lse), (s, u)
            x.steps[1].copy_(clean)
