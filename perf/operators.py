"""The operators beside the block-sparse path, as cases that can be timed and compared: rotary positions, attention with a sliding window
and sinks, and the paged cache that serves a model of such layers.

Five kinds of pass:

  rope     queries and keys of a packed batch turned by their positions, forwards or (gradients) backwards
  forward  window attention of a packed batch, output and log-sum-exp: a pass over evaluation data
  step     the same and its backward pass: an attention layer's part of a training step
  append   new tokens' keys (turned) and values into the pages of a cache, and their queries turned: what a serving step does first
  chunk    attention of the new tokens over the cache, for single tokens (decoding) and for whole chunks (prompts)

Row t of a sequence sees the keys u <= t with t - u < window or u < sinks.

Values are i.i.d. N(0, 1), as everywhere in this repository.  Lengths of a packed batch come from `mix`: one sequence; `mixed`, 60 % short and
40 % long ones; `ragged`, few short ones with one-token and tile-sized ones among them.  Lengths of cached sequences lie between
`shortest` and `longest`, spread over their logarithm; their pages are scattered over the cache.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rope(tokens, hq, hkv, d, *, rot=0, layout="half", scaling="none", dtype="bf16", backward=False, mix="mixed", longest=16384, positions=False, seed=0):
    return {"kind": "rope", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rot": rot or d, "layout": layout, "scaling": scaling, "dtype": dtype,
            "backward": backward, "mix": mix, "longest": longest, "positions": positions, "batch_seed": seed}


def _window(kind, tokens, hq, hkv, d, *, window, sinks, dtype="bf16", mix="mixed", longest=16384, seed=0):
    return {"kind": kind, "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "window": window, "sinks": sinks, "dtype": dtype, "mix": mix,
            "longest": longest, "batch_seed": seed}


def _serve(kind, seqs, new, hq, hkv, d, *, longest, shortest=1, page=64, window=0, sinks=0, rot=0, layout="half", scaling="none", dtype="bf16", seed=0):
    """`new` tokens behind `shortest` .. `longest` cached ones of every sequence; window 0: every key is seen."""
    return {"kind": kind, "seqs": seqs, "new": new, "hq": hq, "hkv": hkv, "d": d, "longest": longest, "shortest": shortest, "page": page,
            "window": window, "sinks": sinks, "rot": rot or d, "layout": layout, "scaling": scaling, "dtype": dtype, "batch_seed": seed}


def listed():
    cases = {
        # the ragged end of an epoch in float32: a unit of debugging
        "rope_2k_f32": _rope(2039, 16, 2, 128, dtype="f32", mix="ragged"),
        # gradients of a long pack, part of the head turned, neighbouring elements paired, scaled for a long context
        "rope_back_64k_part": _rope(65536, 32, 8, 128, rot=64, layout="interleaved", scaling="yarn", backward=True, longest=65536),
        # one short sequence, one head, float32 tensors: gradient checks
        "step_1k_one_head_f32": _window("step", 1024, 1, 1, 64, window=200, sinks=4, dtype="f32", mix="one"),
        # a short packed batch of ragged sequences
        "step_2k_ragged": _window("step", 2039, 16, 2, 128, window=512, sinks=4, mix="ragged"),
        # the ordinary training step: a 32768-token pack, 32/8 heads
        "step_32k": _window("step", 32768, 32, 8, 128, window=4096, sinks=4),
        # a longer pack on the smaller head shape, a short window and a tile of sinks
        "step_64k_d64": _window("step", 65536, 14, 2, 64, window=1024, sinks=64, longest=32768),
        # evaluation on one long sequence, odd token count
        "forward_100k": _window("forward", 100001, 32, 8, 128, window=2000, sinks=16, mix="one"),
        # one step of decoding with many users: the smallest pass of all
        "append_64": _serve("append", 64, 1, 32, 8, 128, longest=2000, scaling="bands"),
        # a prompt's chunk
        "append_prompt_8k": _serve("append", 2, 4096, 32, 8, 128, longest=4000, page=16, layout="interleaved", rot=64),
        # decoding for one user: latency counts
        "decode_one": _serve("chunk", 1, 1, 32, 8, 128, longest=4097, shortest=4097),
        # decoding for many users with caches of very different lengths
        "decode_64": _serve("chunk", 64, 1, 32, 8, 128, longest=32768, shortest=500),
        # a prompt's chunk behind a long cached part, window and sinks, seven query heads per KV head
        "chunk_2k_window": _serve("chunk", 2, 2000, 28, 4, 128, longest=30001, shortest=20000, page=32, window=8192, sinks=4),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _between(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """Another case of the same ranges, no dearer than the largest listed one of its kind."""
    kind = rng.choice(["rope", "step", "step", "forward", "append", "chunk", "chunk"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (16, 2), (14, 2), (4, 2), (8, 8), (1, 1)])
    d = rng.choice([128, 128, 64])
    rot, layout, scaling = rng.choice([d, d, d // 2, 32]), rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "ntk", "yarn", "bands"])
    seed = rng.randrange(1000)
    if kind == "rope":
        tokens = _between(rng, 200, 65536)
        dtype = "f32" if tokens < 16384 and rng.random() < 0.3 else "bf16"
        return _rope(tokens, hq, hkv, d, rot=rot, layout=layout, scaling=scaling, dtype=dtype, backward=rng.random() < 0.5, mix=rng.choice(["one", "mixed", "ragged"]),
                     longest=max(64, tokens // 2), positions=rng.random() < 0.3, seed=seed)
    if kind in ("step", "forward"):
        tokens = _between(rng, 200, 65536 if kind == "step" else 100001)
        dtype = "f32" if tokens < 4096 and rng.random() < 0.3 else "bf16"
        c = _window(kind, tokens, hq, hkv, d, window=_between(rng, 40, 5000), sinks=rng.choice([0, 1, 4, 16, 64, 100]), dtype=dtype,
                    mix=rng.choice(["one", "mixed", "mixed", "ragged" if tokens <= 8192 else "mixed"]), longest=max(64, min(32768, tokens // 2)), seed=seed)
        while work(c)["flops"] > 4.7e12:
            c["window"] //= 2
        return c
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        seqs, new = rng.choice([(_between(rng, 1, 128), 1), (_between(rng, 1, 8), _between(rng, 2, 1000))])
        return _serve("append", seqs, new, hq, hkv, d, longest=4000, page=page, rot=rot, layout=layout, scaling=scaling, seed=seed)
    window, sinks = rng.choice([(0, 0), (0, 0), (_between(rng, 100, 8192), rng.choice([0, 4, 64]))])
    seqs, new = rng.choice([(_between(rng, 1, 64), 1), (_between(rng, 1, 16), _between(rng, 2, 16)), (_between(rng, 1, 3), _between(rng, 100, 2000))])
    longest = _between(rng, 100, 30000)
    return _serve("chunk", seqs, new, hq, hkv, d, longest=longest, shortest=_between(rng, 1, longest), page=page, window=window, sinks=sinks, seed=seed)


def _lens(c):
    """Lengths of a packed batch."""
    rng, left, out = random.Random(c["batch_seed"] * 7919 + c["tokens"]), c["tokens"], []
    if c["mix"] == "one":
        return [left]
    first = [1, 64, 63, 65, 128] if c["mix"] == "ragged" else []
    while left:
        if first:
            n = first.pop()
        elif c["mix"] == "ragged":
            n = rng.randint(1, 700)
        else:
            n = _between(rng, 64, 2048) if rng.random() < 0.6 else _between(rng, 2048, max(2049, c["longest"]))
        n = min(n, left)
        out.append(n)
        left -= n
    rng.shuffle(out)
    return out


def _cached(c):
    """(tokens in the cache, new tokens) of every served sequence: the first as long as may be, chunks of a prompt of unequal lengths."""
    rng = random.Random(c["batch_seed"] * 104729 + c["seqs"])
    have = [c["longest"] if i == 0 else _between(rng, c["shortest"], c["longest"]) for i in range(c["seqs"])]
    new = [c["new"] if i == 0 else max(1, c["new"] - rng.randrange(1 + c["new"] // 8)) for i in range(c["seqs"])]
    return have, new


# ---------------------------------------------------------------- rotary positions
# What a pair of elements turns by at every token, in radians: base^(-2 i / rot), base 10000, changed for long contexts: `linear` divides
# it by the factor 4; `ntk` raises the base; `yarn` divides the slow pairs only, which turn less than once in 8192 tokens, leaves
# those alone that turn more than 32 times, goes over linearly in the pair's index, and scales the result by 0.1 ln 4 + 1; `bands` divides
# by the wave length, between 8192 / 4 and 8192 tokens linearly in its inverse.
FACTOR, LONG = 4.0, 8192
CODES = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}


def _frequencies(rot, scaling):
    """(radians a token of every pair, factor on the result), in 64 bits."""
    i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot
    base = 10000.0 * FACTOR ** (rot / (rot - 2)) if scaling == "ntk" else 10000.0
    f = base ** -i
    if scaling == "linear":
        return f / FACTOR, 1.0
    if scaling == "yarn":
        pair = lambda turns: rot * math.log(LONG / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
        slow = ((torch.arange(rot // 2, dtype=torch.float64, device=DEV) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / FACTOR * slow + f * (1 - slow), 0.1 * math.log(FACTOR) + 1.0
    if scaling == "bands":
        fast = ((LONG * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / FACTOR * (1 - fast) + f * fast, 1.0
    return f, 1.0


def _turn(x, pos, rot, layout, scaling, backward):
    """Plain form, of x [tokens, heads, d]: angles in 64 bits (far positions), products in 32."""
    f, amp = _frequencies(rot, scaling)
    angle = pos.double()[:, None] * f
    cos, sin = (amp * torch.cos(angle)).float()[:, None], (amp * torch.sin(angle)).float()[:, None]
    if backward:
        sin = -sin
    y = x.float()
    a, b = (y[..., : rot // 2], y[..., rot // 2: rot]) if layout == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([a, b], -1) if layout == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _turn_exact(x, pos, rot, layout, scaling, backward):
    """The same as a product of complex numbers, in 64 bits."""
    f, amp = _frequencies(rot, scaling)
    z = torch.polar(torch.full_like(f, amp).expand(len(pos), -1), pos.double()[:, None] * f * (-1.0 if backward else 1.0))[:, None]
    y = x.double().clone()
    if layout == "half":
        w = torch.complex(y[..., : rot // 2].contiguous(), y[..., rot // 2: rot].contiguous()) * z
        y[..., :rot] = torch.cat([w.real, w.imag], -1)
    else:
        w = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:-1], rot // 2, 2).contiguous()) * z
        y[..., :rot] = torch.view_as_real(w).flatten(-2)
    return y


# ---------------------------------------------------------------- window attention
# The packed batch is cut into blocks of W rows, W the window or, where that is longer, the longest sequence.  A block's rows see keys of the
# block before it, of their own, and of the first tokens of their sequences.
def _blocked(x, nb, w):
    """[T, H, D] -> [H, nb, w, D] in 32 bits, zeros behind the last row."""
    y = torch.zeros((nb * w, *x.shape[1:]), dtype=torch.float32, device=DEV)
    y[: len(x)] = x
    return y.view(nb, w, *x.shape[1:]).permute(2, 0, 1, 3).contiguous()


def _before(x):
    return torch.cat([torch.zeros_like(x[:, :1]), x[:, :-1]], 1)


def _window_plain(s, backward):
    c = s["case"]
    t, d, g = s["tokens"], c["d"], c["hq"] // c["hkv"]
    w = min(c["window"], max(s["lens"]))
    nb = (t + w - 1) // w
    sink_rows, sink_seq, sink_pos = s["sink_rows"], s["sink_seq"], s["sink_pos"]
    n_sink = len(sink_rows)
    rows = torch.full((nb * w,), -1, dtype=torch.int64, device=DEV)
    pos = rows.clone()
    rows[:t], pos[:t] = s["seq_of"], s["pos_of"]
    rows, pos = rows.view(nb, w, 1), pos.view(nb, w, 1)
    back = lambda x: torch.cat([torch.full_like(x[:1], -2), x[:-1]], 0)
    key_seq, key_pos = torch.cat([back(rows), rows], 1).mT, torch.cat([back(pos), pos], 1).mT
    seen = (key_seq == rows) & (key_pos <= pos) & ((pos - key_pos < c["window"]) | (key_pos < c["sinks"]))
    if n_sink:  # sinks in the two blocks have been counted there
        behind = (torch.arange(nb, device=DEV) * w - w).view(nb, 1, 1)
        seen = torch.cat([seen, (sink_seq == rows) & (sink_pos <= pos) & (sink_rows < behind)], 2)
    seen = seen[None]
    q, k, v = s["q"], s["k"], s["v"]
    scale = 1.0 / math.sqrt(d)
    o = torch.empty((t, c["hq"], d), dtype=torch.float32, device=DEV)
    lse = torch.empty((c["hq"], t), dtype=torch.float32, device=DEV)
    if backward:
        dq, dk, dv = torch.empty_like(o), torch.zeros((t, c["hkv"], d), dtype=torch.float32, device=DEV), torch.zeros((t, c["hkv"], d), dtype=torch.float32, device=DEV)
    unblock = lambda x: x.permute(1, 2, 0, 3).reshape(nb * w, x.shape[0], d)[:t]
    for h in range(c["hkv"]):  # (all heads' probabilities at once would not fit the card)
        heads = slice(h * g, (h + 1) * g)
        qb, kb, vb = _blocked(q[:, heads], nb, w), _blocked(k[:, h: h + 1], nb, w), _blocked(v[:, h: h + 1], nb, w)
        near = lambda x: torch.cat([_before(x), x] + ([s_of(x)] if n_sink else []), 2)
        s_of = lambda x: (k if x is kb else v)[sink_rows, h].float().expand(1, nb, n_sink, d)
        kc, vc = near(kb), near(vb)
        p = torch.matmul(qb, kc.mT.contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
        top = p.amax(-1, keepdim=True).clamp_min_(-3e38)
        p = p.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        total = torch.where(total > 0, total, torch.ones_like(total))
        p = p.div_(total)
        ob = torch.matmul(p, vc)
        o[:, heads] = unblock(ob)
        lse[heads] = (top + total.log()).reshape(g, nb * w)[:, :t]
        if backward:
            do = _blocked(s["d_o"][:, heads], nb, w)
            dvc = torch.matmul(p.mT.contiguous(), do).sum(0)
            ds = torch.matmul(do, vc.mT.contiguous()).sub_((do * ob).sum(-1, keepdim=True)).mul_(p).mul_(scale)
            dq[:, heads] = unblock(torch.matmul(ds, kc))
            dkc = torch.matmul(ds.mT.contiguous(), qb).sum(0)
            for to, x in ((dk, dkc), (dv, dvc)):
                far = torch.cat([x[1:, :w], torch.zeros_like(x[:1, :w])], 0) + x[:, w: 2 * w]
                to[:, h] = far.reshape(nb * w, d)[:t]
                if n_sink:
                    to[sink_rows, h] += x[:, 2 * w:].sum(0)
        del p
    o = o.to(q.dtype)
    return (o, lse, dq.to(q.dtype), dk.to(q.dtype), dv.to(q.dtype)) if backward else (o, lse)


def _window_exact(s, backward):
    """Sequence by sequence and piece of rows by piece, in 64 bits, gradients of shared keys added up."""
    c = s["case"]
    t, d, hq, hkv = s["tokens"], c["d"], c["hq"], c["hkv"]
    g, scale = hq // hkv, 1.0 / math.sqrt(d)
    o = torch.empty((t, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((hq, t), dtype=torch.float64, device=DEV)
    if backward:
        dq, dk, dv = torch.empty_like(o), torch.zeros((t, hkv, d), dtype=torch.float64, device=DEV), torch.zeros((t, hkv, d), dtype=torch.float64, device=DEV)
    start = 0
    for n in s["lens"]:
        for a in range(0, n, 1024):
            b = min(n, a + 1024)
            lo = max(0, a - c["window"] + 1)
            u = torch.cat([torch.arange(min(c["sinks"], lo), device=DEV), torch.arange(lo, b, device=DEV)])
            r = torch.arange(a, b, device=DEV)[:, None]
            hidden = (u > r) | ((r - u >= c["window"]) & (u >= c["sinks"]))
            at = slice(start + a, start + b)
            for h in range(hkv):
                heads = slice(h * g, (h + 1) * g)
                q = s["q"][at, heads].double().transpose(0, 1)
                k, v = s["k"][start + u, h].double(), s["v"][start + u, h].double()
                x = (q @ k.T * scale).masked_fill(hidden, -math.inf)
                e = torch.logsumexp(x, -1)
                p = torch.exp(x - e[..., None])
                y = p @ v
                o[at, heads], lse[heads, at] = y.transpose(0, 1), e
                if backward:
                    z = s["d_o"][at, heads].double().transpose(0, 1)
                    ds = p * (z @ v.T - (z * y).sum(-1, keepdim=True)) * scale
                    dq[at, heads] = (ds @ k).transpose(0, 1)
                    dk[:, h].index_add_(0, start + u, ds.flatten(0, 1).T @ q.flatten(0, 1))
                    dv[:, h].index_add_(0, start + u, p.flatten(0, 1).T @ z.flatten(0, 1))
        start += n
    return (o, lse, dq, dk, dv) if backward else (o, lse)


# ---------------------------------------------------------------- the paged cache
# [pages][KV heads][tokens of a page][d]; table[s][j] is the page of tokens j * page .. of sequence s.
def _append_plain(s):
    c = s["case"]
    cache_k, cache_v = s["cache_k"], s["cache_v"]
    pos = s["have"][s["seq_of"]] + s["pos_of"]
    page, slot = s["table"].long()[s["seq_of"], pos // c["page"]], pos % c["page"]
    cache_k[page, :, slot] = _turn(s["k"], pos, c["rot"], c["layout"], c["scaling"], False)
    cache_v[page, :, slot] = s["v"]
    return _turn(s["q"], pos, c["rot"], c["layout"], c["scaling"], False), cache_k, cache_v


def _chunk_plain(s):
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
    k, v = (x[page, :, slot].permute(0, 2, 1, 3).float() for x in (s["cache_k"], s["cache_v"]))  # [seqs, hkv, keys, d]
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


def _chunk_exact(s):
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
            k, v = (x[pages, h].reshape(-1, d)[:length].double() for x in (s["cache_k"], s["cache_v"]))
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


# ---------------------------------------------------------------- a case's data and its pass
def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, dtype=torch.float32, device=DEV).to(dtype)
    c, hq, hkv, d = case, case["hq"], case["hkv"], case["d"]
    s = {"case": case}
    serving = case["kind"] in ("append", "chunk")
    lens = _cached(c)[1] if serving else _lens(c)
    t = s["tokens"] = sum(lens)
    s["lens"] = lens
    count = torch.tensor(lens, device=DEV)
    cu = torch.zeros(len(lens) + 1, dtype=torch.int32, device=DEV)
    cu[1:] = count.cumsum(0)
    s["cu"] = cu
    s["seq_of"] = torch.repeat_interleave(torch.arange(len(lens), device=DEV), count)
    s["pos_of"] = torch.arange(t, device=DEV) - cu[:-1].long()[s["seq_of"]]
    s["q"] = normal(t, hq, d)
    if case["kind"] != "chunk":
        s["k"], s["v"] = normal(t, hkv, d), normal(t, hkv, d) if case["kind"] != "rope" else None
    if case["kind"] == "rope" and case["positions"]:
        s["positions"] = torch.randint(0, 1 << 20, (t,), generator=gen, dtype=torch.int32, device=DEV)
    if case["kind"] == "step":
        s["d_o"] = normal(t, hq, d)
    if case["kind"] in ("step", "forward"):
        head = s["pos_of"] < case["sinks"]
        s["sink_rows"] = head.nonzero()[:, 0]
        s["sink_seq"], s["sink_pos"] = s["seq_of"][s["sink_rows"]], s["pos_of"][s["sink_rows"]]
    if serving:
        have, new = _cached(c)
        s["have"], s["new"], s["new_host"] = torch.tensor(have, device=DEV), count, new
        s["total_host"] = [a + b for a, b in zip(have, new)]
        s["window"] = case["window"] or 1 << 30
        need = [(n + c["page"] - 1) // c["page"] for n in s["total_host"]]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=gen, device=DEV).int()
        s["table"] = torch.full((len(need), max(need)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(need):
            s["table"][i, :n] = order[at: at + n]
            at += n
        s["cache_k"], s["cache_v"] = normal(pages, hkv, c["page"], d), normal(pages, hkv, c["page"], d)
    if own:
        import numpy as np

        from paper_2604_13847_amd import binding as sb

        s["sb"] = sb
        code = sb.SB_F32 if case["dtype"] == "f32" else sb.SB_BF16
        if case["kind"] in ("rope", "append"):
            s["rope"] = sb.Rope(c["rot"], layout=sb.SB_ROPE_HALF if c["layout"] == "half" else sb.SB_ROPE_INTERLEAVED, base=10000.0, scaling=CODES[c["scaling"]],
                                factor=FACTOR, original_length=LONG)
        if serving:
            s["cache"] = sb.Cache(s["cache_k"], s["cache_v"], s["table"])
            s["chunk"] = sb.Chunk(s["cu"], s["have"].int(), hq, total_new=t, max_new=max(s["new_host"]), max_length=max(s["total_host"]))
            s["ws"] = torch.empty(max(256, sb.sb_cache_attn_ws_bytes(s["cache"], s["chunk"], s["window"], c["sinks"])), dtype=torch.uint8, device=DEV)
        else:
            s["pb"] = sb.Problem(cu.cpu().numpy(), np.ones(len(lens), dtype=np.int32), hq, hkv, d, dtype=code, device=torch.device(DEV, torch.cuda.current_device()))
    return s


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        sb = s["sb"]
        if kind == "rope":
            return sb.sb_rope_apply(s["pb"], s["rope"], s["q"], s["k"], positions=s.get("positions"), backward=c["backward"])
        if kind == "append":
            q = sb.sb_cache_append(s["cache"], s["chunk"], s["k"], s["v"], rope=s["rope"], q=s["q"])
            return q, s["cache_k"], s["cache_v"]
        if kind == "chunk":
            return sb.sb_cache_attn(s["cache"], s["chunk"], s["q"], window=s["window"], sinks=c["sinks"], ws=s["ws"])
        o, lse = sb.sb_window_attn_fwd(s["pb"], c["window"], c["sinks"], s["q"], s["k"], s["v"])
        if kind == "forward":
            return o, lse
        return (o, lse, *sb.sb_window_attn_bwd(s["pb"], c["window"], c["sinks"], s["q"], s["k"], s["v"], o, lse, s["d_o"]))
    if kind == "rope":
        pos = s.get("positions", s["pos_of"])
        return tuple(_turn(x, pos, c["rot"], c["layout"], c["scaling"], c["backward"]) for x in (s["q"], s["k"]))
    if kind == "append":
        return _append_plain(s)
    return _chunk_plain(s) if kind == "chunk" else _window_plain(s, kind == "step")


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["kind"] == "rope":
        pos = s.get("positions", s["pos_of"])
        return tuple(_turn_exact(x, pos, c["rot"], c["layout"], c["scaling"], c["backward"]) for x in (s["q"], s["k"]))
    if c["kind"] == "append":
        pos = s["have"][s["seq_of"]] + s["pos_of"]
        k, v = s["cache_k"].double(), s["cache_v"].double()
        flat = lambda x: x.permute(0, 2, 1, 3)  # [pages, tokens of a page, KV heads, d]
        table = s["table"].tolist()
        page = torch.tensor([table[i][p // c["page"]] for i, p in zip(s["seq_of"].tolist(), pos.tolist())], device=DEV)
        flat(k)[page, pos % c["page"]] = _turn_exact(s["k"], pos, c["rot"], c["layout"], c["scaling"], False)
        flat(v)[page, pos % c["page"]] = s["v"].double()
        return _turn_exact(s["q"], pos, c["rot"], c["layout"], c["scaling"], False), k, v
    return _chunk_exact(s) if c["kind"] == "chunk" else _window_exact(s, c["kind"] == "step")


def _visible(first, n, window, sinks):
    """Visible keys of rows first .. first + n - 1 of a sequence, added up."""
    t = lambda x: x * (x + 1) // 2
    near = lambda upto: t(upto) if upto <= window else t(window) + (upto - window) * window  # rows 0 .. upto - 1

    def far(upto):  # sinks behind the window: row r has min(sinks, r - window + 1) of them
        m = max(0, upto - window)
        return t(m) if m <= sinks else t(sinks) + (m - sinks) * sinks
    return near(first + n) - near(first) + far(first + n) - far(first)


def work(case):
    c, size = case, 4 if case["dtype"] == "f32" else 2
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "rope":
        t = c["tokens"]
        return {"bytes": 2 * t * (hq + hkv) * d * size + (4 * t if c["positions"] else 0), "flops": 3 * t * (hq + hkv) * c["rot"]}
    if c["kind"] in ("step", "forward"):
        t = c["tokens"]
        pairs = sum(_visible(0, n, c["window"], c["sinks"]) for n in _lens(c)) * hq
        forward = t * (2 * hq + 2 * hkv) * d * size + 4 * t * hq
        # backward: q, o, dO read and dQ written, k, v read and dK, dV written; the log-sum-exp read
        back = t * (4 * hq + 4 * hkv) * d * size + 4 * t * hq
        return {"bytes": forward + (back if c["kind"] == "step" else 0), "flops": pairs * d * (14 if c["kind"] == "step" else 4)}
    have, new = _cached(c)
    t = sum(new)
    if c["kind"] == "append":
        return {"bytes": 2 * t * (hq + 2 * hkv) * d * size, "flops": 3 * t * (hq + hkv) * c["rot"]}
    window = c["window"] or 1 << 30
    pairs = sum(_visible(a, n, window, c["sinks"]) for a, n in zip(have, new)) * hq
    keys = sum(min(a + n, window + n - 1 + min(c["sinks"], max(0, a + 1 - window))) for a, n in zip(have, new))
    return {"bytes": keys * hkv * d * 2 * size + 2 * t * hq * d * size + 4 * t * hq, "flops": 4 * pairs * d}
