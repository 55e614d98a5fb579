"""Plain 64-bit statements of the key/value cache, tree attention and draft verification (not a test module)."""
import math

import numpy as np
import torch

TOP = {"e4m3": 448.0, "int8": 127.0}
DTYPE = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def quantise(x: torch.Tensor, fmt: str):
    """The header's rule, in fp32 as it states it: (codes, scale) of rows x [..., dim]; a non-finite row has scale NaN."""
    x = x.float()
    if fmt == "bf16":
        return x.to(torch.bfloat16), None
    a = x.abs().amax(-1)
    finite = torch.isfinite(x).all(-1)
    s = torch.where(finite, a * torch.tensor(1 / TOP[fmt], dtype=torch.float32), torch.full_like(a, math.nan))
    y = torch.where((finite & (s > 0))[..., None], x / s[..., None], torch.zeros_like(x))
    y = y.clamp(-TOP[fmt], TOP[fmt])
    return (y.round().to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)), s


def held(codes: torch.Tensor, scale) -> torch.Tensor:
    """What the codes stand for, fp64."""
    c = codes.float().double()
    return c if scale is None else c * scale.double()[..., None]


class Pool:
    """A cache pool on the CPU with a page table for `lengths` tokens per request; pages in a random order."""

    def __init__(self, fmt, heads, dim, page, lengths, seed, spare=2, garbage=True):
        g = torch.Generator().manual_seed(seed)
        self.fmt, self.heads, self.dim, self.page, self.g = fmt, heads, dim, page, g
        need = [max(1, -(-n // page)) for n in lengths]
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = torch.full((len(lengths), max(need)), 2 ** 31 - 1, dtype=torch.int32)    # unused entries are never read
        for b, n in enumerate(need):
            self.table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        shape = (self.pages, heads, page, dim)
        # what was never written: NaN patterns in every format that has them, and NaN scales
        fill = {"bf16": math.nan, "e4m3": math.nan, "int8": -128}[fmt] if garbage else 0
        self.k = torch.full(shape, fill, dtype=torch.float32).to(DTYPE[fmt])
        self.v = self.k.clone()
        self.ks = torch.full(shape[:3], math.nan) if fmt != "bf16" else None
        self.vs = torch.full(shape[:3], math.nan) if fmt != "bf16" else None

    def place(self, b, pos):
        return self.table[b, pos // self.page].long(), pos % self.page

    def write(self, b, pos, k, v):
        """k, v [n, heads, dim] at positions pos [n]."""
        pg, line = self.place(b, pos)
        for x, codes, scales in ((k, self.k, self.ks), (v, self.v, self.vs)):
            c, s = quantise(x, self.fmt)
            view = codes.view(torch.uint8) if self.fmt == "e4m3" else codes
            view[pg, :, line] = c.view(torch.uint8) if self.fmt == "e4m3" else c
            if s is not None:
                scales[pg, :, line] = s

    def rows(self, b, n):
        """fp64 keys and values [n, heads, dim] of request b's first n positions."""
        pg, line = self.place(b, torch.arange(n))
        out = []
        for codes, scales in ((self.k, self.ks), (self.v, self.vs)):
            c = codes.float()[pg, :, line]
            out.append(held(c, None if scales is None else scales[pg, :, line]))
        return out

    def device(self, dev, permuted=False):
        """CUDA copies (k, v, ks, vs); permuted: stored [pages, page_tokens, heads, dim], viewed as the cache wants it."""
        def move(t):
            if t is None:
                return None
            if permuted and t.dim() == 4:
                return t.permute(0, 2, 1, 3).contiguous().to(dev).permute(0, 2, 1, 3)
            return t.to(dev)
        return tuple(move(t) for t in (self.k, self.v, self.ks, self.vs))


def random_tree(n, branch, rng):
    """Parents of a random tree of n nodes with at most `branch` children each."""
    parents, used = [-1], [0]
    for i in range(1, n):
        free = [j for j in range(i) if used[j] < branch]
        p = int(free[rng.integers(0, len(free))])
        used[p] += 1
        parents.append(p)
        used.append(0)
    return parents


def tree_bits(parents, words):
    """int32 [n, words]."""
    out = np.zeros((len(parents), words), dtype=np.uint32)
    for i in range(len(parents)):
        j = i
        while j >= 0:
            if j // 32 < words:
                out[i, j // 32] |= np.uint32(1 << (j % 32))
            j = parents[j]
    return torch.from_numpy(out.view(np.int32))


def attention(q, keys, values, ctx, sees, scale):
    """One request in fp64: q [n, q_heads, dim], keys / values [ctx + n, heads, dim], sees [n, n] bool.

    Returns out, lse, and what the bound below needs: sum_j p_j |v_j| and the largest sum_d |q_d k_jd|.
    """
    n, hq, dim = q.shape
    heads = keys.shape[1]
    q = q.double()
    out = torch.zeros(n, hq, dim, dtype=torch.float64)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64)
    mass, big = torch.zeros_like(out), torch.zeros(n, hq, dtype=torch.float64)
    full = torch.ones(n, ctx + n, dtype=torch.bool)
    full[:, ctx:] = sees
    for h in range(hq):
        k, v = keys[:, h // (hq // heads)], values[:, h // (hq // heads)]
        for i in range(n):
            at = full[i]
            if not bool(at.any()):
                continue
            z = (k[at] @ q[i, h]) * scale
            lse[i, h] = torch.logsumexp(z, 0)
            p = torch.softmax(z, 0)
            out[i, h] = p @ v[at]
            mass[i, h] = p @ v[at].abs()
            big[i, h] = (k[at].abs() @ q[i, h].abs()).max()
    return out, lse, mass, big


def attention_bound(out, mass, big, values, fmt, dim, scale, length):
    """How far a bf16 result may be from fp64.

    Rounding to nearest is off by at most 2^-8 of the value in bf16 and 2^-11 in f16: once for the result; weights may
    enter the second product in bf16, or f16 for 8-bit caches (then also 2^-25 of the largest weight where they are
    subnormal).  A score of dim exact products summed in fp32 with truncation is off by dim 2^-23 sum |q k|; scaling and
    exponential add 2^-20; both count twice, in the weights and in their sum.
    """
    weight = 2.0 ** -8 if fmt == "bf16" else 2.0 ** -11
    score = dim * 2.0 ** -23 * big * abs(scale) + 2.0 ** -20
    tiny = 0.0 if fmt == "bf16" else length * 2.0 ** -24 * float(values.abs().max() if values.numel() else 0.0)
    return 2.0 ** -8 * out.abs() + (weight + 2 * score)[..., None] * mass + tiny + 1e-30


def verify(target, draft, tokens, parents, accept, sample, most):
    """One request, fp64 (numpy): (path, next token), the rule of the header."""
    n, vocab = target.shape
    clean = lambda x: np.where(x > 0, x, 0.0).astype(np.float64)  # noqa: E731  (NaN counts as zero)
    path, node = [0], 0
    while True:
        p = clean(target[node])
        r, mass, went = p.copy(), 1.0, None
        kids = [i for i in range(node + 1, n) if parents[i] == node] if len(path) < most else []
        for c in kids:
            x = tokens[c]
            inside = 0 <= x < vocab
            q = (clean(draft[node]) if draft is not None else None)
            qx = (q[x] if q is not None else 1.0) if inside else 0.0
            rx = r[x] if inside else 0.0
            if float(accept[c]) * qx * mass < rx:
                went = c
                break
            if q is not None:
                r = np.maximum(r - mass * q, 0.0)
                mass = float(r.sum())
            else:
                if inside:
                    r[x] = 0.0
                mass -= min(rx, mass)
            if not mass > 0:
                r = p
                break
        if went is None:
            break
        path.append(went)
        node = went
    if not r.sum() > 0:
        r = p
    if not r.sum() > 0:
        return path, -1
    cum = np.cumsum(r)
    hit = np.nonzero((cum > float(sample) * cum[-1]) & (r > 0))[0]
    return path, int(hit[0] if hit.size else np.nonzero(r > 0)[0][-1])
