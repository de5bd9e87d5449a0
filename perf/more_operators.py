"""What a serving loop needs beside attention over a paged cache, as cases that can be timed and compared: rotary positions with several axes (time,
height, width), the page tables of a step, and a cache whose keys and values are held in four bits.

Five kinds of pass:

  turn     queries and keys of a packed batch turned by positions of several axes, forwards or (gradients) backwards
  append   the same in front of a cache in the tensors' own type: new keys and values into their pages, queries turned
  tables   a step's bookkeeping: pages for the new tokens of every request, their slots and positions, the pages of finished requests back; and the
           step's end, which gives back what was rejected, so that the next pass finds what this one found
  append4  new keys (turned) and values into the pages of the four-bit cache, queries turned, and the values as they are held from now on
  attn4    attention of new tokens over the four-bit cache: single tokens, a few drafted ones, whole chunks of prompts

How four bits hold a row of D elements: every 32 neighbours share a step, a bfloat16 number of at most six significant bits near their largest magnitude / 6;
an element is that step times one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign (code 0 .. 7, and 8 for the sign), the nearest one, ties to the even code.  Every value
so held is a bfloat16 number.  A row's D/2 bytes, lower half first: of keys, byte D/8 b + 4 c + e holds elements 32 c + 8 b + 2 e and the one
behind it; of values, byte D/32 i + e elements 32 e + i and 32 e + 16 + i.  Keys are turned in 64 bits and rounded to 32 before that.

New values are i.i.d. N(0, 1), as everywhere in this repository; what the cache holds is that, in four bits.  Pages are scattered over the cache.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _turn_case(tokens, hq, hkv, d, *, sections, order="sections", rot=0, layout="half", dtype="bf16", backward=False, longest=16384, seed=0):
    """sections: pairs of every axis, rot/2 in all."""
    return {"kind": "turn", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot or d, "sections": sections, "order": order, "layout": layout, "dtype": dtype,
            "backward": backward, "longest": longest, "batch_seed": seed}


def _tables_case(seqs, new, *, longest, page, prompts=0, finished=0, seed=0):
    """`new` tokens for every request (drafted ones among them), `prompts` of them with up to `longest` new ones; every `finished`-th request leaves (0: none)."""
    return {"kind": "tables", "seqs": seqs, "new": new, "longest": longest, "page": page, "prompts": prompts, "finished": finished, "batch_seed": seed}


def _serve(kind, seqs, new, hq, hkv, d, *, longest, shortest=1, page=64, window=0, sinks=0, sections="", order="sections", rot=0, layout="half", dtype="bf16", seed=0):
    """`new` tokens behind `shortest` .. `longest` cached ones of every sequence; window 0: every key is seen; sections "": positions of one axis."""
    return {"kind": kind, "seqs": seqs, "new": new, "hq": hq, "hkv": hkv, "d": d, "longest": longest, "shortest": shortest, "page": page, "window": window,
            "sinks": sinks, "sections": sections, "order": order, "rot": rot or d, "layout": layout, "dtype": dtype, "batch_seed": seed}


def listed():
    cases = {
        # the ragged end of an epoch in float32, three axes: a unit of debugging
        "turn_2k_f32": _turn_case(2039, 16, 2, 128, sections="16,24,24", dtype="f32", longest=700),
        # gradients of a long pack of images and text, pairs dealt to the axes in turn
        "turn_back_64k": _turn_case(65536, 32, 8, 128, sections="24,20,20", order="in_turn", layout="interleaved", backward=True, longest=65536),
        # a prompt of images and text, half of the head turned, into a bfloat16 cache
        "append_prompt_8k": _serve("append", 2, 4096, 32, 8, 128, longest=4000, page=16, sections="8,12,12", rot=64),
        # one step of decoding with many users, four tokens drafted for each: the smallest pass of all
        "tables_64": _tables_case(64, 4, longest=32768, page=64, finished=16),
        # prompts come in among many requests: small pages, many slots
        "tables_prompts": _tables_case(1000, 1, longest=16384, page=16, prompts=8, finished=50),
        # one step of decoding with many users
        "append4_64": _serve("append4", 64, 1, 32, 8, 128, longest=2000),
        # a prompt's chunk of images and text
        "append4_prompt_8k": _serve("append4", 2, 4096, 32, 8, 128, longest=4000, page=16, sections="16,24,24"),
        # decoding for one user: latency counts
        "attn4_one": _serve("attn4", 1, 1, 32, 8, 128, longest=4097, shortest=4097),
        # decoding for many users with caches of very different lengths
        "attn4_64": _serve("attn4", 64, 1, 32, 8, 128, longest=32768, shortest=500),
        # five drafted tokens a sequence on the smaller head shape, in float32
        "attn4_draft_f32": _serve("attn4", 16, 5, 14, 2, 64, longest=8000, shortest=100, page=32, dtype="f32"),
        # a prompt's chunk behind a long cached part, window and sinks, seven query heads per KV head
        "attn4_chunk_2k_window": _serve("attn4", 2, 2000, 28, 4, 128, longest=30001, shortest=20000, page=32, window=8192, sinks=4),
        # a first prompt, nothing cached
        "attn4_prompt_6k": _serve("attn4", 1, 6001, 32, 8, 128, longest=0, shortest=0, page=16),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _between(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _split(rng, pairs, axes):
    cuts = sorted(rng.sample(range(1, pairs), axes - 1))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))


def draw(rng):
    """Another case of the same ranges, no dearer than the largest listed one of its kind."""
    kind = rng.choice(["turn", "turn", "append", "tables", "append4", "append4", "attn4", "attn4", "attn4", "attn4"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (16, 2), (14, 2), (4, 2), (8, 8), (1, 1)])
    d = rng.choice([128, 128, 64])
    rot, layout = rng.choice([d, d, d // 2, 32]), rng.choice(["half", "interleaved"])
    sections, order = _split(rng, rot // 2, rng.choice([2, 3, 3, 4])), rng.choice(["sections", "in_turn", "anew"])
    page, seed = rng.choice([16, 32, 64, 128, 256]), rng.randrange(1000)
    if kind == "turn":
        tokens = _between(rng, 200, 65536)
        dtype = "f32" if tokens < 16384 and rng.random() < 0.3 else "bf16"
        return _turn_case(tokens, hq, hkv, d, sections=sections, order=order, rot=rot, layout=layout, dtype=dtype, backward=rng.random() < 0.5,
                          longest=max(64, tokens // 2), seed=seed)
    if kind == "tables":
        seqs = _between(rng, 1, 2000)
        return _tables_case(seqs, rng.choice([1, 1, 4, 7]), longest=_between(rng, 200, 16384), page=page, prompts=min(seqs, rng.choice([0, 0, 1, 5])),
                            finished=rng.choice([0, 3, 20]), seed=seed)
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind in ("append", "append4"):
        seqs, new = rng.choice([(_between(rng, 1, 128), 1), (_between(rng, 1, 8), _between(rng, 2, 1000))])
        if kind == "append4" and rng.random() < 0.4:
            sections = ""
        return _serve(kind, seqs, new, hq, hkv, d, longest=4000, page=page, sections=sections, order=order, rot=rot, layout=layout, dtype=dtype, seed=seed)
    window, sinks = rng.choice([(0, 0), (0, 0), (_between(rng, 100, 8192), rng.choice([0, 4, 64]))])
    seqs, new = rng.choice([(_between(rng, 1, 64), 1), (_between(rng, 1, 16), _between(rng, 2, 16)), (_between(rng, 1, 3), _between(rng, 100, 2000))])
    if dtype == "f32":
        new = min(new, 300)
    longest = _between(rng, 100, 30000)
    c = _serve("attn4", seqs, new, hq, hkv, d, longest=longest, shortest=_between(rng, 1, longest), page=page, window=window, sinks=sinks, dtype=dtype, seed=seed)
    while work(c)["flops"] > 4.5e11:
        c["new"] //= 2
    return c


def _lens(c):
    """Lengths of a packed batch: some short ones, some long."""
    rng, left, out = random.Random(c["batch_seed"] * 7919 + c["tokens"]), c["tokens"], []
    while left:
        n = min(left, _between(rng, 1, 700) if rng.random() < 0.6 else _between(rng, 64, max(65, c["longest"])))
        out.append(n)
        left -= n
    return out


def _cached(c):
    """(tokens in the cache, new tokens) of every served sequence: the first as long as may be, chunks of a prompt of unequal lengths."""
    rng = random.Random(c["batch_seed"] * 104729 + c["seqs"])
    if c["kind"] == "tables":
        have = [_between(rng, 1, c["longest"]) for _ in range(c["seqs"])]
        new = [c["longest"] - rng.randrange(1 + c["longest"] // 4) if i < c["prompts"] else c["new"] for i in range(c["seqs"])]
        have = [0 if i < c["prompts"] else n for i, n in enumerate(have)]
        if c["finished"]:
            new = [-1 if i % c["finished"] == c["finished"] - 1 and i >= c["prompts"] else n for i, n in enumerate(new)]
        return have, new
    have = [c["longest"] if i == 0 else _between(rng, c["shortest"], c["longest"]) for i in range(c["seqs"])]
    new = [c["new"] if i == 0 else max(1, c["new"] - rng.randrange(1 + c["new"] // 8)) for i in range(c["seqs"])]
    return have, new


# ---------------------------------------------------------------- rotary positions of several axes
# Pair i of a head belongs to one axis, and turns by that axis' position times its frequency 10000^(-2 i / rot).  `sections`: the first pairs are
# axis 0's, the next ones axis 1's; `in_turn`: pairs are dealt to the axes in turn, one whose share is used up being left out; `anew`: as `sections`,
# and the frequencies of every axis start again, as if it were a head of its own.
def _pairs(c):
    return [int(x) for x in c["sections"].split(",")] if c["sections"] else [c["rot"] // 2]


def _axes(c):
    """(axis, revolutions a token) of every pair."""
    n, left, axis, turns = _pairs(c), _pairs(c), [], []
    while sum(left):
        for a in range(len(n)):
            for _ in range(min(left[a], 1 if c["order"] == "in_turn" else left[a])):
                i, width = (n[a] - left[a], n[a]) if c["order"] == "anew" else (len(axis), c["rot"] // 2)
                axis.append(a)
                turns.append(10000.0 ** (-i / width) / (2 * math.pi))
                left[a] -= 1
    return torch.tensor(axis, device=DEV), torch.tensor(turns, dtype=torch.float64, device=DEV)


def _positions(c, pos, far):
    """[axes][tokens]: stretches of 512 tokens of text, where all axes go on together, and images of 32 by 32 between them."""
    r, base = pos % 1536, pos // 1536 * 544 + far
    image = r >= 512
    y = (r - 512).clamp_min(0)
    of = [torch.where(image, 512 + step, r) + base for step in (torch.zeros_like(y), y // 32, y % 32, y % 3)]
    return torch.stack(of[: len(_pairs(c))] if c["sections"] else [pos]).int()


def _turn(x, positions, c, backward=False, wide=False):
    """Plain form, of x [tokens, heads, d]: angles in 64 bits (far positions), products in 32, or (wide) in 64 and then rounded to 32."""
    axis, turns = _axes(c)
    rot, kind = c["rot"], torch.float64 if wide else torch.float32
    angle = 2 * math.pi * torch.remainder(positions.double().mT[:, axis] * turns, 1.0)
    cos, sin = torch.cos(angle).to(kind)[:, None], torch.sin(angle).to(kind)[:, None]
    if backward:
        sin = -sin
    y = x.to(kind)
    a, b = (y[..., : rot // 2], y[..., rot // 2: rot]) if c["layout"] == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([a, b], -1) if c["layout"] == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(torch.float32 if wide else x.dtype)


def _turn_exact(x, positions, c, backward=False):
    """The same as a product of complex numbers, in 64 bits."""
    axis, turns = _axes(c)
    rot = c["rot"]
    at = torch.gather(positions.double(), 0, axis[:, None].expand(-1, positions.shape[1])).mT
    z = torch.polar(torch.ones_like(at), at * turns * (-2 * math.pi if backward else 2 * math.pi))[:, None]
    y = x.double().clone()
    if c["layout"] == "half":
        w = torch.complex(y[..., : rot // 2].contiguous(), y[..., rot // 2: rot].contiguous()) * z
        y[..., :rot] = torch.cat([w.real, w.imag], -1)
    else:
        w = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:-1], rot // 2, 2).contiguous()) * z
        y[..., :rot] = torch.view_as_real(w).flatten(-2)
    return y


def _destination(s):
    """(page, token of the page) of every new token."""
    c = s["case"]
    pos = s["have"][s["seq_of"]] + s["pos_of"]
    return s["table"].long()[s["seq_of"], pos // c["page"]], pos % c["page"]


def _append_plain(s):
    page, slot = _destination(s)
    s["cache_k"][page, :, slot] = _turn(s["k"], s["positions"], s["case"])
    s["cache_v"][page, :, slot] = s["v"]
    return _turn(s["q"], s["positions"], s["case"]), s["cache_k"], s["cache_v"]


def _append_exact(s):
    page, slot = _destination(s)
    k, v = s["cache_k"].double(), s["cache_v"].double()
    k.permute(0, 2, 1, 3)[page, slot] = _turn_exact(s["k"], s["positions"], s["case"])
    v.permute(0, 2, 1, 3)[page, slot] = s["v"].double()
    return _turn_exact(s["q"], s["positions"], s["case"]), k, v


# ---------------------------------------------------------------- four bits
SIXTH = 0.16666667163372040  # 1/6 rounded to 32 bits
MOST_STEP = 1.3125 * 2.0 ** 125  # six times that is still a bfloat16 number


def _steps(x):
    """x [..., D] in 32 bits -> [..., D/32]: six significant bits, halves away from zero."""
    t = x.unflatten(-1, (-1, 32)).abs().amax(-1) * SIXTH
    bits = torch.bitwise_and(t.view(torch.int32) + 0x20000, -0x40000)
    return bits.view(torch.float32).clamp_max(MOST_STEP)


def _four_bits(x):
    """x [..., D] in 32 bits -> (codes [..., D] uint8, steps [..., D/32], values [..., D])."""
    step = _steps(x)
    wide = step.repeat_interleave(32, -1)
    y = x.abs()
    # thresholds are exact: a step of six bits times three
    level = ((y > 0.25 * wide).to(torch.uint8) + (y >= 0.75 * wide) + (y > 1.25 * wide) + (y >= 1.75 * wide) + (y > 2.5 * wide) + (y >= 3.5 * wide) + (y > 5.0 * wide))
    code = level + torch.signbit(x).to(torch.uint8) * 8
    return code, step, _levels(code) * wide


def _levels(code):
    m = (code & 7).float()
    m = torch.where(m < 4, 0.5 * m, torch.where(m < 6, m - 2, 2 * m - 8))
    return torch.where(code >= 8, -m, m)


def _four_bits_exact(x):
    """Values and steps, in 64 bits, of x [..., D] (32 bits): the nearest number of so many bits, found by rounding."""
    step = _steps(x).double()
    wide = step[..., None].expand(*step.shape, 32).flatten(-2)
    y = torch.where(wide > 0, x.double().abs() / wide, torch.zeros_like(wide)).clamp_max(6.0)
    unit = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    return torch.round(y / unit) * unit * wide * torch.sign(x.double()), step


def _pack_keys(code):
    """[..., D] -> [..., D/2]"""
    x = code.unflatten(-1, (-1, 4, 4, 2))  # c, b, e, half
    return (x[..., 0] | x[..., 1] << 4).transpose(-3, -2).flatten(-3)


def _pack_values(code):
    x = code.unflatten(-1, (-1, 2, 16))  # e, half, i
    return (x[..., 0, :] | x[..., 1, :] << 4).transpose(-2, -1).flatten(-2)


def _unpack_keys(b, d):
    x = b.unflatten(-1, (4, d // 32, 4)).transpose(-3, -2)
    return torch.stack([x & 15, x >> 4], -1).flatten(-4)


def _unpack_values(b, d):
    x = b.unflatten(-1, (16, d // 32)).transpose(-2, -1)
    return torch.stack([x & 15, x >> 4], -2).flatten(-3)


def _held(codes, steps, d, values):
    """Values of rows of the cache, in 32 bits."""
    level = _levels((_unpack_values if values else _unpack_keys)(codes, d))
    return (level.unflatten(-1, (-1, 32)) * steps.float()[..., None]).flatten(-2)


def _held_exact(codes, steps, d, values):
    """The same element by element from a table of sixteen numbers, in 64 bits."""
    e = torch.arange(d, device=DEV)
    byte, upper = ((e % 16) * (d // 32) + e // 32, e // 16 % 2) if values else (d // 8 * (e // 8 % 4) + 4 * (e // 32) + e % 8 // 2, e % 2)
    code = codes[..., byte].long() // (1 + 15 * upper) % 16
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    return torch.cat([table, -table])[code] * steps.double()[..., e // 32]


def _append4_plain(s):
    c = s["case"]
    page, slot = _destination(s)
    out = []
    for x, codes, steps, pack in ((_turn(s["k"], s["positions"], c, wide=True), s["k4"], s["k_step"], _pack_keys), (s["v"].float(), s["v4"], s["v_step"], _pack_values)):
        code, step, value = _four_bits(x)
        codes[page, :, slot] = pack(code)
        steps[page, :, slot] = step.bfloat16()
        out.append(value.to(s["k"].dtype))
    return _turn(s["q"], s["positions"], c), *out, s["k4"], s["k_step"], s["v4"], s["v_step"]


def _append4_exact(s):
    c = s["case"]
    page, slot = _destination(s)
    k, k_step = _four_bits_exact(_turn_exact(s["k"], s["positions"], c).float())
    v, v_step = _four_bits_exact(s["v"].float())
    ks, vs = s["k_step"].double(), s["v_step"].double()
    ks.permute(0, 2, 1, 3)[page, slot] = k_step
    vs.permute(0, 2, 1, 3)[page, slot] = v_step
    return _turn_exact(s["q"], s["positions"], c), k, v, None, ks, None, vs


# ---------------------------------------------------------------- attention over the four-bit cache
# [pages][KV heads][tokens of a page][...]; table[s][j] is the page of tokens j * page .. of sequence s.
def _attn4_plain(s):
    c = s["case"]
    seqs, d, hkv, g, window, sinks = c["seqs"], c["d"], c["hkv"], c["hq"] // c["hkv"], s["window"], c["sinks"]
    most = max(s["new_host"])
    have, new = s["have"], s["new"]
    length = have + new
    # the keys that any row of the sequence's chunk can see: the first `sinks`, and the last ones
    near = min(max(s["total_host"]), window + most - 1)
    first = (length - near).clamp_min(0)
    u = first[:, None] + torch.arange(near, device=DEV)
    if sinks:
        far = torch.arange(sinks, device=DEV).expand(seqs, -1)
        u = torch.cat([torch.where(far < first[:, None], far, length[:, None]), u], 1)
    exists = u < length[:, None]
    at = torch.where(exists, u, torch.zeros_like(u))
    page, slot = torch.gather(s["table"].long(), 1, at // c["page"]), at % c["page"]
    k, v = (_held(x[page, :, slot], y[page, :, slot], d, w).transpose(1, 2).contiguous()  # [seqs, hkv, keys, d]
            for x, y, w in ((s["k4"], s["k_step"], False), (s["v4"], s["v_step"], True)))
    r = torch.arange(most, device=DEV)
    row = (s["cu"].long()[:-1, None] + r).clamp_max(len(s["q"]) - 1)
    t = (have[:, None] + r)[:, :, None]
    q = s["q"][row].float().view(seqs, most, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, g * most, d)
    x = torch.matmul(q, k.mT.contiguous()).mul_(1.0 / math.sqrt(d)).view(seqs, hkv, g, most, -1)
    un = u[:, None, :]
    seen = exists[:, None, :] & (un <= t) & ((t - un < window) | (un < sinks))
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min_(-3e38)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(seqs, hkv, g * most, -1), v).view(seqs, hkv, g, most, d) / total.clamp_min(1e-30)
    lse = (top + total.log())[..., 0]
    o = o.permute(0, 3, 1, 2, 4).reshape(seqs, most, hkv * g, d)
    lse = lse.permute(0, 3, 1, 2).reshape(seqs, most, hkv * g)
    return o[s["seq_of"], s["pos_of"]].to(s["q"].dtype), lse[s["seq_of"], s["pos_of"]].mT.contiguous()


def _attn4_exact(s):
    """Sequence by sequence, head by head and piece of rows by piece, in 64 bits."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    o = torch.empty((len(s["q"]), hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((hq, len(s["q"])), dtype=torch.float64, device=DEV)
    start = 0
    for i, n in enumerate(s["new_host"]):
        length = s["total_host"][i]
        have = length - n
        pages = s["table"][i, : (length + c["page"] - 1) // c["page"]].long()
        for h in range(hkv):
            k, v = (_held_exact(x[pages, h].flatten(0, 1)[:length], y[pages, h].flatten(0, 1)[:length], d, w)
                    for x, y, w in ((s["k4"], s["k_step"], False), (s["v4"], s["v_step"], True)))
            for a in range(0, n, 512):
                b = min(n, a + 512)
                t, u = torch.arange(have + a, have + b, device=DEV)[:, None], torch.arange(length, device=DEV)
                hidden = (u > t) | ((t - u >= s["window"]) & (u >= c["sinks"]))
                q = s["q"][start + a: start + b, h * g: (h + 1) * g].double().transpose(0, 1)
                x = (q @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                e = torch.logsumexp(x, -1)
                o[start + a: start + b, h * g: (h + 1) * g] = (torch.exp(x - e[..., None]) @ v).transpose(0, 1)
                lse[h * g: (h + 1) * g, start + a: start + b] = e
        start += n
    return o, lse


# ---------------------------------------------------------------- page tables
# Row s of the table holds pages for tokens 0 .. cached + new - 1 of request s (none where new < 0: it is finished); `held` says how many it holds.  Entries that
# are too many go back on the stack of free pages, the last entry of the last row first; entries that lack get pages from its top in order.
def _tables_plain(s, cached, new):
    c = s["case"]
    page, table, held, free, count = c["page"], s["table"], s["held"], s["free"], s["count"]
    wide = table.shape[1]
    length = torch.where(new < 0, 0, cached + new)
    want = ((length + page - 1) // page).clamp_max(wide)
    j = torch.arange(wide, device=DEV)
    back = ((j >= want[:, None]) & (j < held[:, None])).flatten()
    rank = torch.cumsum(back, 0)
    given = rank[-1]
    padded = torch.cat([free, free[:1]])
    padded[torch.where(back, count + given - rank, len(free))] = table.flatten()
    flat = torch.where(back, -1, table.flatten())
    now = count + given
    lack = ((j >= held[:, None]) & (j < want[:, None])).flatten()
    rank = torch.cumsum(lack, 0)
    there = lack & (rank <= now)
    flat = torch.where(there, padded[(now - rank).clamp(0, len(free) - 1)], flat)
    table.copy_(flat.view_as(table))
    held.copy_(torch.minimum(want, held) + there.view_as(table).sum(1))
    free.copy_(padded[:-1])
    count.copy_(now - there.sum())
    missing = (lack.sum() - there.sum()).int().view(1)
    cu = torch.cat([torch.zeros_like(new[:1]), torch.cumsum(new.clamp_min(0), 0)])
    t = torch.arange(s["total"], device=DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    pos = cached[seq] + t - cu[seq]
    at = table[seq, pos // page].long()
    return cu.int(), pos.int(), torch.where(at < 0, -1, at * page + pos % page), missing


# ---------------------------------------------------------------- a case's data and its pass
def _tables_state(c, gen):
    have, new = _cached(c)
    page, s = c["page"], {"case": c}
    held = [-(-n // page) for n in have]
    wide = max(-(-(a + max(b, 0)) // page) for a, b in zip(have, new))
    pages = sum(held) + sum(-(-(a + max(b, 0)) // page) - h for a, b, h in zip(have, new, held)) + 10
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    s["held"] = torch.tensor(held, dtype=torch.int32, device=DEV)
    own_page = torch.arange(wide, device=DEV) < s["held"][:, None]
    s["table"] = torch.full((len(have), wide), -1, dtype=torch.int32, device=DEV)
    s["table"][own_page] = order[: sum(held)]
    s["free"] = torch.cat([order[sum(held):], order[: sum(held)] * 0])
    s["count"] = torch.tensor([pages - sum(held)], dtype=torch.int32, device=DEV)
    s["cached"], s["new"] = torch.tensor(have, dtype=torch.int32, device=DEV), torch.tensor(new, dtype=torch.int32, device=DEV)
    s["none"], s["total"] = torch.zeros_like(s["new"]), sum(max(n, 0) for n in new)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    c = case
    if c["kind"] == "tables":
        s = _tables_state(c, gen)
        if own:
            from paper_2604_13847_amd import binding as sb

            s["sb"], s["pool"] = sb, sb.PagePool(s["table"], s["held"], s["free"], s["count"], c["page"])
        return s
    dtype = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, dtype=torch.float32, device=DEV).to(dtype)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    s = {"case": case}
    serving = c["kind"] != "turn"
    have, lens = _cached(c) if serving else (None, _lens(c))
    t = s["tokens"] = sum(lens)
    count = torch.tensor(lens, device=DEV)
    s["cu"] = torch.cat([count[:1] * 0, count.cumsum(0)]).int()
    s["seq_of"] = torch.repeat_interleave(torch.arange(len(lens), device=DEV), count)
    s["pos_of"] = torch.arange(t, device=DEV) - s["cu"][:-1].long()[s["seq_of"]]
    s["q"] = normal(t, hq, d)
    if c["kind"] != "attn4":
        s["k"], s["v"] = normal(t, hkv, d), normal(t, hkv, d) if serving else None
        far = torch.randint(0, 1 << 18, (len(lens),), generator=gen, device=DEV)[s["seq_of"]]
        pos = s["pos_of"] + (torch.tensor(have, device=DEV)[s["seq_of"]] if serving else 0)
        s["positions"] = _positions(c, pos, far)
    if serving:
        s["have"], s["new"], s["new_host"] = torch.tensor(have, device=DEV), count, lens
        s["total_host"] = [a + b for a, b in zip(have, lens)]
        s["window"] = c["window"] or 1 << 30
        need = [(n + c["page"] - 1) // c["page"] for n in s["total_host"]]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=gen, device=DEV).int()
        mine = torch.arange(max(need), device=DEV) < torch.tensor(need, device=DEV)[:, None]
        s["table"] = torch.full((len(need), max(need)), -1, dtype=torch.int32, device=DEV)
        s["table"][mine] = order[: sum(need)]
        if c["kind"] == "append":
            s["cache_k"], s["cache_v"] = normal(pages, hkv, c["page"], d), normal(pages, hkv, c["page"], d)
        else:
            for name, pack in (("k", _pack_keys), ("v", _pack_values)):
                codes = torch.empty((pages, hkv, c["page"], d // 2), dtype=torch.uint8, device=DEV)
                steps = torch.empty((pages, hkv, c["page"], d // 32), dtype=torch.bfloat16, device=DEV)
                some = max(1, (1 << 27) // (hkv * c["page"] * d))  # pages at a time
                for a in range(0, pages, some):
                    x = torch.randn((min(some, pages - a), hkv, c["page"], d), generator=gen, dtype=torch.float32, device=DEV)
                    code, step, _ = _four_bits(x)
                    codes[a: a + some], steps[a: a + some] = pack(code), step.bfloat16()
                s[name + "4"], s[name + "_step"] = codes, steps
    if own:
        import numpy as np

        from paper_2604_13847_amd import binding as sb

        s["sb"] = sb
        code = sb.SB_F32 if c["dtype"] == "f32" else sb.SB_BF16
        if c["kind"] != "attn4":
            layout = sb.SB_ROPE_HALF if c["layout"] == "half" else sb.SB_ROPE_INTERLEAVED
            n = _pairs(c)
            s["rope"] = sb.Rope.joined([sb.Rope(2 * x, layout=layout) for x in n]) if c["order"] == "anew" else sb.Rope(c["rot"], layout=layout)
            s["axes"] = sb.RopeAxes(n, order=sb.SB_AXES_IN_TURN if c["order"] == "in_turn" else sb.SB_AXES_SECTIONS)
        if serving:
            four = c["kind"] != "append"
            s["cache"] = sb.Cache4(s["k4"], s["v4"], s["k_step"], s["v_step"], s["table"], dtype=dtype) if four else sb.Cache(s["cache_k"], s["cache_v"], s["table"])
            s["chunk"] = sb.Chunk(s["cu"], s["have"].int(), hq, total_new=t, max_new=max(lens), max_length=max(s["total_host"]))
            if c["kind"] == "attn4":
                s["ws"] = torch.empty(max(256, sb.sb_cache4_attn_ws_bytes(s["cache"], s["chunk"], s["window"], c["sinks"])), dtype=torch.uint8, device=DEV)
        else:
            s["pb"] = sb.Problem(s["cu"].cpu().numpy(), np.ones(len(lens), dtype=np.int32), hq, hkv, d, dtype=code, device=torch.device(DEV, torch.cuda.current_device()))
    return s


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        sb = s["sb"]
        if kind == "turn":
            return sb.sb_rope_axes_apply(s["pb"], s["rope"], s["axes"], s["positions"], s["q"], s["k"], backward=c["backward"])
        if kind == "append":
            return sb.sb_cache_append_axes(s["cache"], s["chunk"], s["k"], s["v"], s["rope"], s["axes"], s["positions"], q=s["q"]), s["cache_k"], s["cache_v"]
        if kind == "append4":
            where = (s["axes"], s["positions"]) if c["sections"] else (None, None)
            out = sb.sb_cache4_append(s["cache"], s["chunk"], s["k"], s["v"], rope=s["rope"], axes=where[0], positions=where[1], q=s["q"], held=True)
            return (*out, s["k4"], s["k_step"], s["v4"], s["v_step"])
        if kind == "attn4":
            return sb.sb_cache4_attn(s["cache"], s["chunk"], s["q"], window=s["window"], sinks=c["sinks"], ws=s["ws"])
        out = sb.sb_cache_tables(s["pool"], s["cached"], s["new"], s["total"])
        sb.sb_cache_tables(s["pool"], s["cached"], s["none"], 0)
    else:
        if kind == "turn":
            return tuple(_turn(x, s["positions"], c, c["backward"]) for x in (s["q"], s["k"]))
        if kind == "append":
            return _append_plain(s)
        if kind == "append4":
            return _append4_plain(s)
        if kind == "attn4":
            return _attn4_plain(s)
        out = _tables_plain(s, s["cached"], s["new"])
        _tables_plain(dict(s, total=0), s["cached"], s["none"])
    return (*out, s["table"], s["held"], s["free"], s["count"])


def exact(case, seed):
    if case["kind"] == "tables":
        return None  # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "turn":
        return tuple(_turn_exact(x, s["positions"], case, case["backward"]) for x in (s["q"], s["k"]))
    return {"append": _append_exact, "append4": _append4_exact, "attn4": _attn4_exact}[case["kind"]](s)


def _visible(first, n, window, sinks):
    """Visible keys of rows first .. first + n - 1 of a sequence, added up."""
    t = lambda x: x * (x + 1) // 2
    near = lambda upto: t(upto) if upto <= window else t(window) + (upto - window) * window  # rows 0 .. upto - 1

    def far(upto):  # sinks behind the window: row r has min(sinks, r - window + 1) of them
        m = max(0, upto - window)
        return t(m) if m <= sinks else t(sinks) + (m - sinks) * sinks
    return near(first + n) - near(first) + far(first + n) - far(first)


def work(case):
    c = case
    if c["kind"] == "tables":
        have, new = _cached(c)
        page = c["page"]
        change = sum(abs((-(-(a + b) // page) if b >= 0 else 0) - -(-a // page)) for a, b in zip(have, new))
        # lengths and held counts twice, slots and positions, and every page that changes hands: read, written and cleared, there and back
        return {"bytes": 2 * 16 * len(have) + 12 * sum(max(b, 0) for b in new) + 2 * 12 * change, "flops": 0}
    size = 4 if c["dtype"] == "f32" else 2
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    axes = len(_pairs(c))
    if c["kind"] == "turn":
        t = c["tokens"]
        return {"bytes": 2 * t * (hq + hkv) * d * size + 4 * axes * t, "flops": 3 * t * (hq + hkv) * c["rot"]}
    have, new = _cached(c)
    t = sum(new)
    row = d // 2 + d // 32 * 2  # bytes of a row in four bits
    if c["kind"] == "append":
        return {"bytes": 2 * t * (hq + 2 * hkv) * d * size + 4 * axes * t, "flops": 3 * t * (hq + hkv) * c["rot"]}
    if c["kind"] == "append4":
        return {"bytes": t * (2 * hq + 4 * hkv) * d * size + 2 * t * hkv * row + (4 * axes * t if c["sections"] else 0), "flops": 3 * t * (hq + hkv) * c["rot"] + 10 * t * 2 * hkv * d}
    window = c["window"] or 1 << 30
    pairs = sum(_visible(a, n, window, c["sinks"]) for a, n in zip(have, new)) * hq
    keys = sum(min(a + n, window + n - 1 + min(c["sinks"], max(0, a + 1 - window))) for a, n in zip(have, new))
    return {"bytes": keys * hkv * row * 2 + 2 * t * hq * d * size + 4 * t * hq, "flops": 4 * pairs * d}
