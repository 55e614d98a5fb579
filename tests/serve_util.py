"""Plain statements of the 4-bit cache, rotary positions and page bookkeeping (not a test module)."""
import math

import torch

import kv_util

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def quantise4(x: torch.Tensor):
    """The header's rule, in fp32 as it states it: (bytes [..., dim / 2], group bytes [..., dim / 16], scale) of rows x [..., dim]."""
    x = x.float()
    top = x.abs().amax(-1)
    finite = torch.isfinite(x).all(-1)
    use = torch.where(finite, top, torch.zeros_like(top))
    m, e = torch.frexp(use)
    k = torch.where(m <= 0.65625, e - 12, e - 11).clamp_min(-126)             # 6 * 448 = 0.65625 * 2^12
    live = finite & (use > 0)
    two = lambda n: ((n + 127) << 23).to(torch.int32).view(torch.float32)  # noqa: E731
    s = torch.where(live, two(k), torch.zeros_like(use))
    s = torch.where(finite, s, torch.full_like(s, math.nan))
    y = torch.where(live[..., None], x * two(torch.where(live, -k, torch.zeros_like(k)))[..., None], torch.zeros_like(x)).unflatten(-1, (-1, 16))
    group = (y.abs().amax(-1) * torch.tensor(1 / 6, dtype=torch.float32)).to(torch.float8_e4m3fn)
    g = group.float()[..., None]
    y = torch.where(g > 0, y / torch.where(g > 0, g, torch.ones_like(g)), torch.zeros_like(y)).flatten(-2)
    a = y.abs()
    code = sum((a > b if strict else a >= b).to(torch.uint8) for b, strict in
               ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)))
    code = code | torch.signbit(y).to(torch.uint8) * 8
    return code[..., 0::2] | code[..., 1::2] << 4, group.view(torch.uint8), s


def held4(codes, group, scale):
    """What they stand for, fp64: group bytes are read without their sign, 0x7f as 480."""
    table = torch.tensor(E2M1 + [-v for v in E2M1], dtype=torch.float64)
    v = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()]
    b = group.long() & 127
    e, m = b >> 3, b & 7
    g = torch.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7).double(), m / 8.0 * 2.0 ** -6)
    return v * g.repeat_interleave(16, -1) * scale.double()[..., None]


class Pool4(kv_util.Pool):
    """kv_util.Pool in 4 bits."""

    def __init__(self, fmt, heads, dim, page, lengths, seed, spare=2, garbage=True):
        super().__init__("int8", heads, dim, page, lengths, seed, spare, garbage)
        self.fmt = "e2m1"
        shape = (self.pages, heads, page)
        g = torch.Generator().manual_seed(seed + 1)
        # what was never written: any codes, group scales among them that would be NaN as E4M3
        fill = lambda n: torch.randint(0, 256, shape + (n,), generator=g, dtype=torch.uint8) if garbage else torch.zeros(shape + (n,), dtype=torch.uint8)  # noqa: E731
        self.k, self.v, self.kg, self.vg = fill(dim // 2), fill(dim // 2), fill(dim // 16), fill(dim // 16)

    def sides(self):
        return (self.k, self.kg, self.ks), (self.v, self.vg, self.vs)

    def write(self, b, pos, k, v):
        pg, line = self.place(b, pos)
        for x, side in zip((k, v), self.sides()):
            for t, w in zip(side, quantise4(x)):
                t[pg, :, line] = w

    def rows(self, b, n):
        pg, line = self.place(b, torch.arange(n))
        return [held4(*(t[pg, :, line] for t in side)) for side in self.sides()]

    def device(self, dev, permuted=False):
        def move(t):
            if permuted and t is not self.ks and t is not self.vs and t is not self.kg and t is not self.vg:
                return t.permute(0, 2, 1, 3).contiguous().to(dev).permute(0, 2, 1, 3)
            return t.to(dev)
        return (*(move(t) for t in (self.k, self.v, self.ks, self.vs)),
                *(move(t).view(torch.float8_e4m3fn) for t in (self.kg, self.vg)))


def weights_and_scales(q, keys, scales, ctx, sees, scale):
    """One request in fp64: softmax weights [q_heads, n, positions] and the largest weight times its value's scale [n, q_heads]; q
    [n, q_heads, dim], keys [positions, heads, dim], scales (of the values) [positions, heads]."""
    n, hq, dim = q.shape
    heads = keys.shape[1]
    z = torch.einsum("jhd,thgd->hgtj", keys, q.double().view(n, heads, hq // heads, dim)) * scale
    seen = torch.ones(n, keys.shape[0], dtype=torch.bool)
    seen[:, ctx:] = sees
    z = z.masked_fill(~seen, -math.inf)
    p = torch.nan_to_num(torch.softmax(z, -1))                           # heads, group, n, positions
    largest = (p * scales.T[:, None, None]).amax(-1)                     # heads, group, n
    return p.flatten(0, 1), largest.permute(2, 0, 1).reshape(n, hq)


def attention_bound4(out, mass, big, largest, values, scales, dim, scale):
    """How far a bf16 result over a 4-bit cache may be from fp64.

    The result's rounding, 2^-8 of it.  A weight times its value's scale enters the second product in f16: 2^-11 of it, and steps of
    2^-31 of the row's largest such product (`largest`, weights as shares of their sum): the sum over the positions of that times
    |code * group scale|.  Scores as in kv_util.attention_bound, twice.  The second product sums one product per position in fp32 with
    truncation: 2^-23 each of at most sum p |v|."""
    length, heads = values.shape[:2]
    score = dim * 2.0 ** -23 * big * abs(scale) + 2.0 ** -20
    codes = (values.abs() / torch.where(scales > 0, scales, torch.ones_like(scales))[..., None]).sum(0)         # heads, dim
    flush = 2.0 ** -31 * largest[..., None] * codes.repeat_interleave(out.shape[1] // heads, 0)
    return 2.0 ** -8 * out.abs() + (2.0 ** -11 + 2 * score + length * 2.0 ** -23)[..., None] * mass + flush + 1e-30


def cos_sin(turns, positions, amplitude=1.0):
    """fp64 [tokens, pairs] from the fixed-point frequencies: the angle is exact."""
    c, s = [], []
    for t in positions.tolist():
        a = [((t * (w & (2 ** 64 - 1))) % 2 ** 64) / 2.0 ** 64 * 2 * math.pi for w in turns.tolist()]
        c.append([math.cos(x) for x in a])
        s.append([math.sin(x) for x in a])
    return amplitude * torch.tensor(c, dtype=torch.float64), amplitude * torch.tensor(s, dtype=torch.float64)


def turned(x, turns, positions, layout, amplitude=1.0, inverse=False):
    """x [tokens, heads, dim] turned, fp64, and what its bound below needs: |x| + |y| of the pair at every element that is turned."""
    x = x.double()
    pairs = turns.numel()
    c, s = (t[:, None] for t in cos_sin(turns, positions, amplitude))
    if inverse:
        s = -s
    at = (torch.arange(pairs), torch.arange(pairs) + pairs) if layout == 0 else (2 * torch.arange(pairs), 2 * torch.arange(pairs) + 1)
    a, b = x[..., at[0]], x[..., at[1]]
    out, size = x.clone(), torch.zeros_like(x)
    out[..., at[0]], out[..., at[1]] = a * c - b * s, b * c + a * s
    size[..., at[0]] = size[..., at[1]] = a.abs() + b.abs()
    return out, size


def turned_bound(out, size, amplitude, dtype):
    """An angle rounded to fp32 within an eighth of a turn is off by 0.8 * 2^-24, its cosine and sine by that and a unit (2^-23 at
    most) in the last place, twice; times the amplitude: 2^-24 more; two products and a sum in fp32: 2 * 2^-24.  Then the rounding."""
    return size * abs(amplitude) * 8 * 2.0 ** -24 + torch.finfo(dtype).eps / 2 * (out.abs() + size * abs(amplitude) * 8 * 2.0 ** -24) + 1e-38


class Tables:
    """Page tables on the CPU, worked on entry by entry."""

    def __init__(self, requests, width, pages, page):
        self.page, self.width, self.pages = page, width, pages
        self.table = [[-1] * width for _ in range(requests)]
        self.held = [0] * requests
        self.holders = [0] * pages

    def reserve(self, start, tokens):
        """(moves, missing)"""
        need = [min(-(-t // self.page), self.width) if t >= 0 else 0 for t in tokens]
        writers = {}
        for b, (s, t) in enumerate(zip(start, tokens)):
            s = max(s, 0)
            if t > s:
                for e in range(s // self.page, min(need[b], self.held[b])):
                    if self.holders[self.table[b][e]] > 1:
                        writers.setdefault(self.table[b][e], []).append((b, e))
        leave = set()
        for p, who in writers.items():
            leave.update(who[1:] if len(who) == self.holders[p] else who)
        fresh = [(b, e) for b in range(len(need)) for e in range(need[b]) if e >= self.held[b] or (b, e) in leave]
        free = [p for p, n in enumerate(self.holders) if n == 0]
        if len(fresh) > len(free):
            return [], len(fresh) - len(free)
        moves = []
        for (b, e), p in zip(fresh, free):
            s = max(start[b], 0)
            if (b, e) in leave:
                self.holders[self.table[b][e]] -= 1
                if e == s // self.page and s % self.page:
                    moves.append((self.table[b][e], p, s % self.page))
            self.table[b][e] = p
            self.holders[p] = 1
        self.held = [max(h, n) for h, n in zip(self.held, need)]
        return moves, 0

    def release(self, tokens=None):
        for b in range(len(self.held)):
            t = 0 if tokens is None else tokens[b]
            while t >= 0 and self.held[b] > -(-t // self.page):
                self.held[b] -= 1
                self.holders[self.table[b][self.held[b]]] -= 1
                self.table[b][self.held[b]] = -1

    def fork(self, from_, to, tokens):
        """How many forks were left out."""
        held, taken, out = list(self.held), set(), 0
        for f, t, n in zip(from_, to, tokens):
            if not (0 <= f < len(held) and 0 <= t < len(held)) or held[t] or t in taken:
                out += 1
                continue
            taken.add(t)
            k = min(-(-max(n, 0) // self.page), held[f])
            self.table[t][:k] = self.table[f][:k]
            for p in self.table[f][:k]:
                self.holders[p] += 1
            self.held[t] = k
        return out

    def compact(self, most):
        in_use, moves, went = sum(n > 0 for n in self.holders), [], {}
        low, high = 0, self.pages - 1
        while len(moves) < most:
            while low < self.pages and self.holders[low]:
                low += 1
            while high >= 0 and not self.holders[high]:
                high -= 1
            if low >= high:
                break
            moves.append((high, low, self.page))
            went[high] = low
            self.holders[low], self.holders[high] = self.holders[high], 0
        for b, n in enumerate(self.held):
            self.table[b][:n] = [went.get(p, p) for p in self.table[b][:n]]
        return moves, in_use
