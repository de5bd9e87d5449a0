"""Plain 64-bit forms of the rotary positions and of window attention, with elementwise bounds on what a kernel may be off by.

The bounds follow from the roundings that the kernels make, `half` being half a step of the storage type relative to the value (2^-8 or 2^-24):
  score   the product over d in float32, in any order:  c = (D + 8) 2^-24 max(scale |q|.|k|); it, and the same error in LSE, move a probability by a factor
  P, dS   rounded to the storage type before the second product: half |P|, half |dS|
  sums    over N keys in float32: N 2^-24 of the sum of magnitudes
  output  rounded to the storage type: half |result|
  Dr      = rowsum(dO * O) from the stored O, whose own bound counts
so a result X = sum_j w_j x_j is off by at most  half |X| + (half + 3 c + N 2^-24) sum_j |w_j x_j|  plus, in the backward, what Dr is off by."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
EPS = 2.0 ** -24


def visible(tq, u, window, sinks):
    """[rows, keys]"""
    t = tq[:, None]
    return (u <= t) & ((t - u < window) | (u < sinks))


class Attention:
    """Rows q [n, Hq, D] at positions tq over keys k, v [m, Hkv, D] (float64), those of seen [n, m]."""

    def __init__(self, q, k, v, seen, scale, half, d_o=None):
        n, Hq, D = q.shape
        m, Hkv, _ = k.shape
        G = Hq // Hkv
        qh, kh, vh = q.permute(1, 0, 2), k.permute(1, 0, 2).repeat_interleave(G, 0), v.permute(1, 0, 2).repeat_interleave(G, 0)
        s = (qh @ kh.mT * scale).masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True) if m else torch.full((Hq, n, 1), -math.inf, dtype=q.dtype, device=q.device)
        e = torch.exp(s - top.clamp_min(-1e300))
        total = e.sum(-1, keepdim=True)
        p = e / total.clamp_min(1e-300)
        self.lse = (top + total.log())[..., 0]
        o = p @ vh
        c = (D + 8) * EPS * float((qh.abs() @ kh.abs().mT * scale).masked_fill(~seen, 0).max()) if m and n else 0.0
        err = half + 3 * c + (m + 8) * EPS
        self.lse_tol = 2 * c + (m + 8) * EPS + 4 * EPS * self.lse.abs()
        o_tol = half * o.abs() + err * (p @ vh.abs())
        back = lambda x: x.permute(1, 0, 2)
        self.o, self.o_tol = back(o), back(o_tol)
        if d_o is None:
            return
        do = d_o.permute(1, 0, 2)
        dp = do @ vh.mT
        dr = (do * o).sum(-1, keepdim=True)
        ds = p * (dp - dr)
        # Dr from the stored O; dP and Dr are sums over D in float32
        dr_err = (do.abs() * o_tol).sum(-1, keepdim=True) + (D + 8) * EPS * ((do.abs() * o.abs()).sum(-1, keepdim=True) + do.abs() @ vh.abs().mT)
        ds_abs = err * ds.abs() + p * dr_err                    # what dS is off by
        group = lambda x: x.view(Hkv, G, m, D).sum(1).permute(1, 0, 2)
        self.dq = back(ds @ kh * scale)
        self.dq_tol = half * self.dq.abs() + scale * back((ds_abs + err * ds.abs()) @ kh.abs())
        self.dk = group(ds.mT @ qh * scale)
        self.dk_tol = half * self.dk.abs() + scale * group((ds_abs + (err + n * G * EPS) * ds.abs()).mT @ qh.abs())
        self.dv = group(p.mT @ do)
        self.dv_tol = half * self.dv.abs() + group((err + n * G * EPS) * p.mT @ do.abs())


def check(name, got, ref, tol):
    got = got.double()
    both = torch.isinf(ref) & (got == ref)
    d = torch.where(both, torch.zeros_like(ref), (got - ref).abs())
    bad = ~(d <= torch.where(both, torch.zeros_like(tol), tol) + 1e-30)
    assert not bool(bad.any()), f"{name}: {int(bad.sum())} of {bad.numel()} values off, the first at {bad.nonzero()[0].tolist()}: {got[bad][0]:.6g}, {ref[bad][0]:.6g} +- {tol[bad][0]:.2g}"


def turn(x, pos, turns, amplitude, half_layout, backward=False):
    """x [n, H, D] in float64; turns: revolutions per token of every pair.  Returns (result, bound without the storage type's rounding)."""
    r = 2 * len(turns)
    a = 2 * math.pi * torch.remainder(pos.double()[:, None] * turns, 1.0)[:, None]
    cos, sin = amplitude * torch.cos(a), amplitude * torch.sin(a) * (-1.0 if backward else 1.0)
    y, tol = x.clone(), torch.zeros_like(x)
    i, j = (slice(0, r // 2), slice(r // 2, r)) if half_layout else (slice(0, r, 2), slice(1, r, 2))
    y[..., i], y[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., j] * cos + x[..., i] * sin
    # angle 2^-23.3 (half a step below half a revolution, times 2 pi), sine and cosine 2 steps, the factor, two products and their sum: together at most 8 steps
    tol[..., i] = tol[..., j] = 8 * EPS * amplitude * (x[..., i].abs() + x[..., j].abs())
    return y, tol
