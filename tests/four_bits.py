"""Plain forms of the four-bit cache's rows (element by element, from the layout's words) and of the page tables (lists)."""
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def places(D, values, device):
    """(byte, upper half or not) of every element of a row."""
    if values:  # byte D/32 i + e holds elements 32 e + i and 32 e + 16 + i
        d = torch.arange(D, device=device)
        return (d % 16) * (D // 32) + d // 32, d // 16 % 2
    d = torch.arange(D, device=device)  # byte D/8 b + 4 c + e holds elements 32 c + 8 b + 2 e and the next
    return (d // 8 % 4) * (D // 8) + 4 * (d // 32) + d % 8 // 2, d % 2


def pack(code, values):
    """Codes [..., D] (0 .. 15) -> bytes [..., D/2]"""
    byte, upper = places(code.shape[-1], values, code.device)
    out = torch.zeros(*code.shape[:-1], code.shape[-1] // 2, dtype=torch.int64, device=code.device)
    out.index_add_(-1, byte, code.long() << 4 * upper)
    return out.to(torch.uint8)


def unpack(rows, values):
    byte, upper = places(2 * rows.shape[-1], values, rows.device)
    return rows[..., byte].long() >> 4 * upper & 15


def value(code, step):
    """Codes [..., D] and steps [..., D/32] as the numbers that they stand for, in float64."""
    table = torch.tensor(LEVELS, dtype=torch.float64, device=code.device)
    return torch.cat([table, -table])[code] * step.double().repeat_interleave(32, -1)


def held(rows, step, values):
    return value(unpack(rows, values), step)


def step_of(x):
    """Of x [..., D] (float32), in float64: 1/6 of the largest magnitude of 32, to six significant bits (and multiples of 2^-131), halves away from zero; NaN where one of them is no
    number or infinite."""
    most = x.unflatten(-1, (-1, 32)).abs().amax(-1)
    sixth = (most * torch.tensor(1.0 / 6.0, dtype=torch.float32, device=x.device)).double()
    exponent = torch.frexp(sixth)[1]
    quantum = (exponent.long() - 6 + 1023 << 52).view(torch.float64).clamp_min(2.0 ** -131)  # 2^(exponent - 6), from its bits: torch.ldexp is not exact on the GPU
    y = (torch.floor(sixth / quantum + 0.5) * quantum).clamp_max(1.3125 * 2.0 ** 125)
    return torch.where(torch.isfinite(most), y, torch.full_like(y, float("nan")))


def code_of(x, step):
    """The nearest level's code, by distance, ties to the even code; the largest one's beyond it; 0 where the step is 0 or no number."""
    wide = step.repeat_interleave(32, -1)
    y = torch.where(wide > 0, x.double().abs() / wide, torch.zeros_like(wide)).clamp_max(6.0)
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    far = (y[..., None] - levels).abs()
    far[..., 1::2] += 1e-9  # (in steps: no float32 number over a step of six bits is so near to a tie without being one)
    return torch.where(wide > 0, far.argmin(-1) + 8 * torch.signbit(x), 0)


class Pool:
    """The page tables as lists."""

    def __init__(self, num_seqs, max_pages, num_pages, page, order=None):
        self.page, self.max_pages = page, max_pages
        self.rows, self.free, self.num_pages = [[] for _ in range(num_seqs)], list(range(num_pages)) if order is None else list(order), num_pages

    def step(self, cached, added, total):
        """(cu, positions, slots, missing) and the new state."""
        want = [0 if n < 0 else min(-(-(max(c, 0) + n) // self.page), self.max_pages) for c, n in zip(cached, added)]
        for row, n in reversed(list(zip(self.rows, want))):
            while len(row) > n:
                self.free.append(row.pop())
        missing = 0
        for row, n in zip(self.rows, want):
            while len(row) < n and self.free:
                row.append(self.free.pop())
            missing += n - len(row)
        cu, pos, slots = [0], [], []
        for c, n, row in zip(cached, added, self.rows):
            cu.append(cu[-1] + max(n, 0))
            for t in range(max(c, 0), max(c, 0) + min(max(n, 0), total - len(pos))):
                pos.append(t)
                j = t // self.page
                slots.append(row[j] * self.page + t % self.page if j < len(row) else -1)
        return cu, pos + [0] * (total - len(pos)), slots + [-1] * (total - len(slots)), missing
