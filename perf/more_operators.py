"""What is measured of the operators that a serving loop needs around the paged key/value cache:

  rope     rotary positions of a prompt's queries and keys, of gradients on their way back, and of a decoding step whose keys
           go straight into the cache
  attend   attention of a step's tokens over a cache held in 4 bits (E2M1 codes, an E4M3 scale per 16 of them, a power of
           two per token and head)
  cache    a prompt's chunk quantised into such a cache, and the whole context read back
  pages    whose pages are whose: forking requests, taking and returning pages, moving the pages in use together

`run` computes each with elementary torch operations, or, where `own` is true, through the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
ELEM = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------ cases

def rows_case(name, tokens, heads, dim, rot, layout, elem, inverse, scaling, first):
    return {"name": name, "op": "rope", "kind": "rows", "tokens": tokens, "heads": heads, "dim": dim, "rot": rot, "layout": layout,
            "elem": elem, "inverse": inverse, "scaling": scaling, "first": first}


def step_case(name, requests, tokens, ctx, q_heads, kv_heads, dim, rot, layout, page, scaling):
    return {"name": name, "op": "rope", "kind": "step", "requests": requests, "tokens": tokens, "ctx": ctx, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "rot": rot, "layout": layout, "page": page, "scaling": scaling}


def attend_case(name, requests, tokens, ctx, q_heads, kv_heads, dim, page, tree):
    return {"name": name, "op": "attend", "requests": requests, "tokens": tokens, "ctx": ctx, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "tree": tree}


def cache_case(name, requests, tokens, ctx, kv_heads, dim, page):
    return {"name": name, "op": "cache", "requests": requests, "tokens": tokens, "ctx": ctx, "kv_heads": kv_heads, "dim": dim,
            "page": page}


def fork_case(name, parents, children, ctx, kv_heads, dim, page, spare):
    return {"name": name, "op": "pages", "kind": "fork", "parents": parents, "children": children, "ctx": ctx, "kv_heads": kv_heads,
            "dim": dim, "page": page, "spare": spare}


def turn_case(name, requests, ctx, page, spare):
    return {"name": name, "op": "pages", "kind": "turn", "requests": requests, "ctx": ctx, "page": page, "spare": spare}


def compact_case(name, requests, ctx, kv_heads, dim, page, spare):
    return {"name": name, "op": "pages", "kind": "compact", "requests": requests, "ctx": ctx, "kv_heads": kv_heads, "dim": dim,
            "page": page, "spare": spare}


def listed():
    return [
        # queries and keys of a prompt of 8192 tokens out of one fused product (64 query and 8 key heads, whole heads turned,
        # the frequencies of a model whose context was stretched by wavelength)
        rows_case("rope prompt 8192", 8192, 72, 128, 128, "half", "bf16", False, "bands", 0),
        # the gradient's way back through the same in training: fp32, neighbouring pairs, part of an odd-sized head
        rows_case("rope back 1501x20 part", 1501, 20, 80, 48, "interleaved", "f32", True, "none", 0),
        # a decoding step of a batch, far into a stretched context: queries turned, keys turned and appended, values appended
        step_case("rope step 32x1", 32, 1, 1000, 64, 8, 128, 128, "half", 32, "ramp"),
        # one user at the start of a conversation, no drafts: the latency of a single token
        attend_case("attend 1x1 short", 1, 1, 407, 32, 4, 128, 16, False),
        # ordinary decoding of a batch, one token per request (64 query and 8 key/value heads)
        attend_case("attend 32x1", 32, 1, 4100, 64, 8, 128, 32, False),
        # odd sizes: three query heads per key head, 64-wide heads, a ragged tree of drafts
        attend_case("attend 4x13 tree d64", 4, 13, 1531, 27, 9, 64, 64, True),
        # trees of 32 drafts, contexts of a few thousand tokens
        attend_case("attend 8x32 tree", 8, 32, 8000, 64, 8, 128, 32, True),
        # one user with a very long context and a wide tree: the largest
        attend_case("attend 1x64 tree long", 1, 64, 100000, 64, 8, 128, 16, True),
        # a prompt's chunk quantised on its way in, and the whole context read back for what follows
        cache_case("cache fill 4x2048", 4, 2048, 6000, 8, 128, 32),
        # eight prompts, four continuations of each: forked, then every continuation gets its own copy of the page it writes
        fork_case("pages fork 8x4", 8, 4, 1900, 8, 128, 32, 40),
        # between two steps of a large batch: finished requests return their pages, the others take one more where they need it
        turn_case("pages turnover 512", 512, 4000, 32, 9000),
        # a pool that long traffic has scattered: the pages in use are moved to its front (bf16)
        compact_case("pages compact 150", 150, 2000, 8, 128, 32, 3500),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    scalings = ["none", "linear", "bands", "ramp"]
    while True:
        op = rng.choice(["rows", "step", "attend", "attend", "attend", "cache", "fork", "turn", "compact"])
        kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8, 16])
        dim, page = rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128])
        layout = rng.choice(["half", "interleaved"])
        if op == "rows":
            dim = rng.choice([64, 80, 96, 128, 128, 256])
            rot = dim if rng.random() < 0.5 else 2 * rng.randint(1, dim // 2)
            c = rows_case("", _spread(rng, 1, 16384), _spread(rng, 1, 80), dim, rot, layout, rng.choice(["bf16", "f32"]),
                          rng.random() < 0.5, rng.choice(scalings), rng.choice([0, 0, _spread(rng, 1, 1000000)]))
        elif op == "step":
            rot = dim if rng.random() < 0.5 else 2 * rng.randint(1, dim // 2)
            c = step_case("", _spread(rng, 1, 64), _spread(rng, 1, 64), _spread(rng, 1, 2000), kv * group, kv, dim, rot, layout, page,
                          rng.choice(scalings))
        elif op == "attend":
            c = attend_case("", _spread(rng, 1, 64), _spread(rng, 1, 64), _spread(rng, 1, 100000), kv * group, kv, dim, page,
                            rng.random() < 0.6)
        elif op == "cache":
            c = cache_case("", _spread(rng, 1, 64), _spread(rng, 1, 4096), _spread(rng, 1, 8000), kv, dim, page)
        elif op == "fork":
            c = fork_case("", _spread(rng, 1, 32), _spread(rng, 1, 8), _spread(rng, 1, 8000), kv, dim, page, 300 + _spread(rng, 1, 2000))
        elif op == "turn":
            c = turn_case("", _spread(rng, 1, 1000), _spread(rng, 1, 8000), page, _spread(rng, 1, 50000))
        else:
            c = compact_case("", _spread(rng, 1, 400), _spread(rng, 1, 8000), kv, dim, page, _spread(rng, 1, 20000))
        c.pop("name")
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and _held(c) <= 1.2e9:
            return c


def _held(c):
    """The most values a drawn case makes of its inputs at once: it bounds what the plain form holds."""
    if c["op"] == "attend":
        return c["requests"] * c["ctx"] * (c["tokens"] * c["q_heads"] + 2 * c["kv_heads"] * c["dim"])
    if c["op"] == "cache":
        return 4 * c["requests"] * (c["ctx"] + c["tokens"]) * c["kv_heads"] * c["dim"]
    if c["op"] == "pages":
        pages = c.get("requests", c.get("parents", 0)) * (1 + c.get("children", 0)) * (c["ctx"] // c["page"] + 2) + c["spare"]
        return pages * 8 if c["kind"] == "turn" else pages * 2 * c["page"] * c["kv_heads"] * c["dim"]
    if c["kind"] == "step":
        return 2 * c["requests"] * (c["ctx"] + c["tokens"]) * c["kv_heads"] * c["dim"]
    return 4 * c["tokens"] * c["heads"] * c["dim"]


def contexts(c):
    """Tokens in the cache before the step, request by request: from half of ctx to all of it, one request with all."""
    return [max(0, int(c["ctx"] * (1.0 - 0.5 * ((0.6180339887 * b) % 1.0)))) for b in range(c.get("requests", c.get("parents", 0)))]


def counts(c):
    """The step's tokens, request by request: trees are ragged, the first request has the most."""
    if not c.get("tree", False):
        return [c["tokens"]] * c["requests"]
    return [max(1, int(c["tokens"] * (1.0 - 0.4 * ((0.7548776662 * b) % 1.0)))) for b in range(c["requests"])]


def row_bytes(c):
    """A token's keys and values in the 4-bit cache: codes, a byte per 16, and the row's scale."""
    return 2 * c["kv_heads"] * (c["dim"] // 2 + c["dim"] // 16 + 4)


def work(c):
    if c["op"] == "rope":
        if c["kind"] == "rows":
            item = 2 if c["elem"] == "bf16" else 4
            return {"bytes": 2.0 * c["tokens"] * c["heads"] * c["dim"] * item + 4.0 * c["tokens"],
                    "flops": 3.0 * c["tokens"] * c["heads"] * c["rot"]}
        total = c["requests"] * c["tokens"]
        return {"bytes": 2.0 * total * (c["q_heads"] + 2 * c["kv_heads"]) * c["dim"] * 2,
                "flops": 3.0 * total * (c["q_heads"] + c["kv_heads"]) * c["rot"]}
    if c["op"] == "attend":
        n = counts(c)
        # every token sees the whole context, its own chain or branch behind that
        pairs = sum((x + (m + 1) / 2 if not c["tree"] else x + math.log2(m + 1)) * m for x, m in zip(contexts(c), n))
        return {"bytes": float(sum(x + m for x, m in zip(contexts(c), n)) * row_bytes(c) + sum(n) * 4 * c["q_heads"] * c["dim"]),
                "flops": 4.0 * pairs * c["q_heads"] * c["dim"]}
    if c["op"] == "cache":
        wide, total = 4 * c["kv_heads"] * c["dim"], c["requests"] * c["tokens"]
        back = sum(contexts(c)) + total
        return {"bytes": float((total + back) * (row_bytes(c) + wide)), "flops": 4.0 * (total + back) * c["kv_heads"] * c["dim"]}
    held = [-(-x // c["page"]) for x in contexts(c)]
    if c["kind"] == "fork":
        tails = [x % c["page"] for x in contexts(c)]
        n = c["children"]
        entries, rows = n * sum(held), sum(tails) * n
        # tables of the continuations, holders looked through once; tails copied once and read back
        return {"bytes": float(8 * entries + 4 * (sum(held) + c["spare"]) + rows * (2 * row_bytes(c) + row_bytes(c) + 4 * c["kv_heads"] * c["dim"])),
                "flops": float(rows * row_bytes(c))}
    if c["kind"] == "turn":
        pool = sum(held) + c["spare"]
        gone = sum(h for b, h in enumerate(held) if b % 8 == 3)
        return {"bytes": float(4 * pool + 12 * gone + 16 * len(held)), "flops": float(pool)}
    moved = sum(held) * (c["spare"] / (sum(held) + c["spare"]))
    return {"bytes": moved * 2 * 2 * c["page"] * c["kv_heads"] * c["dim"] * 2 + 8.0 * sum(held) + 8.0 * (sum(held) + c["spare"]),
            "flops": moved * c["page"] * c["kv_heads"] * c["dim"]}


# ----------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 6151 + 29)
    return g


BASE, FACTOR, ORIGINAL = 500000.0, 8.0, 8192.0


def _frequencies(c, dtype=torch.float64):
    """Angle per position of every pair, in 64 bits."""
    n = c["rot"] // 2
    i = torch.arange(n, dtype=dtype, device=DEV)
    f = BASE ** (-2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        return f / FACTOR
    if c["scaling"] == "bands":        # long wavelengths are stretched, short ones left, between 1 and 4 turns blended
        t = ((ORIGINAL * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return (1 - t) * f / FACTOR + t * f
    if c["scaling"] == "ramp":         # the same by the pair's number, between those that turn 32 times and once
        at = lambda turns: c["rot"] * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), c["rot"] - 1)
        t = ((i - lo) / (hi - lo if hi > lo else 0.001)).clamp(0, 1)
        return t * f / FACTOR + (1 - t) * f
    return f


def _amplitude(c):
    return 0.1 * math.log(FACTOR) + 1.0 if c["scaling"] == "ramp" else 1.0


def _own_rope(c):
    from paper_2607_04031_b200 import binding as tl
    kind = {"none": tl.ROPE_PLAIN, "linear": tl.ROPE_LINEAR, "bands": tl.ROPE_BANDS, "ramp": tl.ROPE_RAMP}[c["scaling"]]
    low, high = (1.0, 32.0) if c["scaling"] == "ramp" else (1.0, 4.0)
    turns = tl.rope_turns(c["rot"], BASE, kind, factor=FACTOR, original=ORIGINAL, low=low, high=high).to(DEV)
    return tl.rope(turns, tl.ROPE_HALF if c["layout"] == "half" else tl.ROPE_INTERLEAVED, _amplitude(c))


def _quantise(x):
    """x [..., dim] (fp32) -> codes (two of a byte, the first one low), a byte's E4M3 scale per 16, a power of two per row."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)                                               # the least s = 2^k with 6 * 448 s >= the largest
    k = torch.where(m <= 0.65625, e - 12, e - 11)
    two = lambda e: ((e + 127) << 23).view(torch.float32)  # noqa: E731      (exactly)
    s = torch.where(top > 0, two(k), torch.zeros_like(top))
    y = torch.where((top > 0).unsqueeze(-1), x * two(-k).unsqueeze(-1), torch.zeros_like(x)).unflatten(-1, (-1, 16))
    group = (y.abs().amax(-1) * torch.tensor(1 / 6, dtype=torch.float32, device=x.device)).to(torch.float8_e4m3fn)
    g = group.float().unsqueeze(-1)
    y = torch.where(g > 0, y / torch.where(g > 0, g, 1.0), torch.zeros_like(y)).flatten(-2)
    a = y.abs()                                                           # to the nearest, ties to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    code |= (torch.signbit(y) * 8).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, group, s


def _values(codes, group, scale, dtype=torch.float32):
    """What they stand for: code times group scale times the row's."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=dtype, device=codes.device)
    v = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()]
    return (v.unflatten(-1, (-1, 16)) * group.to(dtype).unsqueeze(-1)).flatten(-2) * scale.to(dtype).unsqueeze(-1)


def _offsets(n):
    return torch.tensor([0] + n, device=DEV).cumsum(0).to(torch.int32)


def _trees(n, host):
    """Trees by request: node 0 is the root, parents before children, at most four children of one node."""
    out = []
    for m in n:
        up, used = [-1], [0]
        for i in range(1, m):
            free = [j for j in range(i) if used[j] < 4]
            p = free[max(0, len(free) - 1 - int(host.expovariate(0.5)))]            # mostly recent nodes: trees grow deep
            used[p] += 1
            up.append(p)
            used.append(0)
        out.append(up)
    return out


def _mask(trees, words):
    """Bit j of row i: token i sees token j (itself and its ancestors)."""
    rows = []
    for t in trees:
        seen = []
        for i, p in enumerate(t):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows += [[(v >> (32 * w)) & 0xffffffff for w in range(words)] for v in seen]
    return torch.tensor(rows, dtype=torch.int64, device=DEV).to(torch.int32)


def _table(per, spare, g, width=0):
    """A shuffled page table [requests, width] with `per` pages of each request (-1 behind them), and how many pages there are."""
    width = max(width, max(per), 1)
    order = torch.randperm(sum(per) + spare, generator=g, device=DEV).to(torch.int32)
    at = torch.tensor([0] + per, device=DEV).cumsum(0)
    col = torch.arange(width, device=DEV)
    real = col[None] < torch.tensor(per, device=DEV)[:, None]
    return torch.where(real, order[(at[:-1, None] + col).clamp_max(order.numel() - 1)], -1).to(torch.int32).contiguous(), order.numel()


def _filled(pages, c, g):
    """A 4-bit pool with keys and values in it, some channels larger than the others as in trained models."""
    shape = (pages, c["kv_heads"], c["page"], c["dim"])
    wide = torch.ones(c["dim"], device=DEV)
    wide[:: 16] = 2.5
    out = []
    for spread in (wide, torch.ones_like(wide)):
        codes = torch.empty(shape[:3] + (c["dim"] // 2,), dtype=torch.uint8, device=DEV)
        group = torch.empty(shape[:3] + (c["dim"] // 16,), dtype=torch.float8_e4m3fn, device=DEV)
        scale = torch.empty(shape[:3], device=DEV)
        step = max(1, (1 << 26) // math.prod(shape[1:]))
        for a in range(0, pages, step):
            x = torch.randn((min(step, pages - a),) + shape[1:], generator=g, device=DEV) * spread
            codes[a:a + step], group[a:a + step], scale[a:a + step] = _quantise(x)
        out.append((codes, group, scale))
    return out


def _own_cache(pool):
    from paper_2607_04031_b200 import binding as tl
    (k, kg, ks), (v, vg, vs) = pool
    return tl.kv_cache(k, v, ks, vs, kg, vg)


def prepare(case, seed):
    import random
    return {"rope": _prepare_rope, "attend": _prepare_cached, "cache": _prepare_cached, "pages": _prepare_pages}[case["op"]](
        case, _gen(seed), random.Random(int(seed)))


def _prepare_rope(c, g, host):
    s = {"case": c, "freq": _frequencies(c)}
    if own:
        s["rope"] = _own_rope(c)
    if c["kind"] == "rows":
        s["x"] = torch.randn(c["tokens"], c["heads"], c["dim"], generator=g, device=DEV).to(ELEM[c["elem"]])
        s["out"] = torch.empty_like(s["x"])
        # three sequences packed one behind the other
        n = -(-c["tokens"] // 3)
        s["positions"] = (c["first"] + torch.arange(c["tokens"], device=DEV) % n).to(torch.int32)
        return s
    n = counts(c)
    kv, dim, heads = c["kv_heads"], c["dim"], c["q_heads"]
    s.update(offsets=_offsets(n), total=sum(n), ctx=torch.tensor(contexts(c), dtype=torch.int32, device=DEV))
    s["table"], pages = _table([-(-(x + m) // c["page"]) for x, m in zip(contexts(c), n)], 3, g)
    s["k"], s["v"] = (torch.randn(pages, kv, c["page"], dim, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    qkv = torch.randn(s["total"], (heads + 2 * kv) * dim, generator=g, device=DEV).to(torch.bfloat16)
    s["q"] = qkv[:, :heads * dim].view(-1, heads, dim)
    s["new_k"] = qkv[:, heads * dim:(heads + kv) * dim].view(-1, kv, dim)
    s["new_v"] = qkv[:, (heads + kv) * dim:].view(-1, kv, dim)
    s["out"] = torch.empty(s["total"], heads, dim, dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2607_04031_b200 import binding as tl
        s["cache"] = tl.kv_cache(s["k"], s["v"])
        s["batch"] = tl.kv_batch(s["table"], s["ctx"], s["offsets"], s["total"])
    return s


def _prepare_cached(c, g, host):
    n = counts(c)
    kv, dim = c["kv_heads"], c["dim"]
    s = {"case": c, "offsets": _offsets(n), "total": sum(n), "most": max(n),
         "ctx": torch.tensor(contexts(c), dtype=torch.int32, device=DEV), "longest": max(x + m for x, m in zip(contexts(c), n))}
    s["table"], pages = _table([-(-(x + m) // c["page"]) for x, m in zip(contexts(c), n)], 3, g)
    s["pool"] = _filled(pages, c, g)
    if c["op"] == "attend":
        s["q"] = torch.randn(s["total"], c["q_heads"], dim, generator=g, device=DEV).to(torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(dim)
        s["out"] = torch.empty_like(s["q"])
        s["mask"] = _mask(_trees(n, host), -(-s["most"] // 32)) if c["tree"] else None
    else:
        new = torch.randn(s["total"], 2 * kv * dim, generator=g, device=DEV).to(torch.bfloat16)
        s["new"] = [new[:, :kv * dim].view(-1, kv, dim), new[:, kv * dim:].view(-1, kv, dim)]
        back = [x + m for x, m in zip(contexts(c), n)]
        s["back"], s["back_total"], s["zero"] = _offsets(back), sum(back), torch.zeros_like(s["ctx"])
        s["read"] = [torch.empty(s["back_total"], kv, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    if own:
        from paper_2607_04031_b200 import binding as tl
        s["cache"] = _own_cache(s["pool"])
        s["batch"] = tl.kv_batch(s["table"], s["ctx"], s["offsets"], s["total"])
        if c["op"] == "cache":
            s["reads"] = tl.kv_batch(s["table"], s["zero"], s["back"], s["back_total"])
    return s


def _prepare_pages(c, g, host):
    x, page = contexts(c), c["page"]
    per = [-(-n // page) for n in x]
    kids = c["children"] if c["kind"] == "fork" else 0
    s = {"case": c}
    # room for a step's growth; continuations stand behind their parents
    table, pages = _table(per + [0] * (len(per) * kids), c["spare"] + len(per) * (1 + kids), g, max(per) + 2)
    holders = torch.zeros(pages + 1, dtype=torch.int32, device=DEV)
    holders.scatter_(0, torch.where(table >= 0, table, pages).long().flatten(), 1)
    s.update(table=table, holders=holders[:pages].contiguous(), held=torch.tensor(per + [0] * (len(per) * kids), dtype=torch.int32, device=DEV))
    s["work"] = {k: torch.empty_like(s[k]) for k in ("table", "holders", "held")}
    requests = table.shape[0]
    s["moves"] = torch.full((max(requests, pages if c["kind"] == "compact" else 0), 3), -1, dtype=torch.int32, device=DEV)
    s["n_moves"], s["missing"] = (torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2))
    if c["kind"] == "fork":
        s["pool"] = _filled(pages, c, g)
        s["from"] = torch.arange(len(per), device=DEV).repeat_interleave(kids).to(torch.int32)
        s["to"] = (len(per) + torch.arange(len(per) * kids, device=DEV)).to(torch.int32)
        s["tokens"] = torch.tensor(x, dtype=torch.int32, device=DEV).repeat_interleave(kids)
        # every continuation is about to write one token; their parents are done
        s["start"] = torch.cat([torch.full((len(per),), -1, dtype=torch.int32, device=DEV), s["tokens"]])
        s["wanted"] = torch.where(s["start"] < 0, -1, s["start"] + 1)
        tails = [n % page for n in x for _ in range(kids)]
        s["tail"] = _offsets([0] * len(per) + tails)
        s["tail_from"] = torch.where(s["start"] < 0, 0, s["start"] // page * page).to(torch.int32)
        s["tail_total"] = sum(tails)
        s["read"] = [torch.empty(s["tail_total"], c["kv_heads"], c["dim"], dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    elif c["kind"] == "turn":
        # every eighth request is over (keeps nothing), the others are about to write four tokens
        over = torch.arange(requests, device=DEV) % 8 == 3
        lengths = torch.tensor(x, dtype=torch.int32, device=DEV)
        s["keep"] = torch.where(over, 0, -1).to(torch.int32)
        s["start"] = torch.where(over, -1, lengths).to(torch.int32)
        s["wanted"] = torch.where(over, -1, lengths + 4).to(torch.int32)
    else:
        s["k"], s["v"] = (torch.empty(pages, c["kv_heads"], page, c["dim"], dtype=torch.bfloat16, device=DEV) for _ in range(2))
        for t in (s["k"], s["v"]):
            for a in range(0, pages, 1024):
                t[a:a + 1024] = torch.randn(t[a:a + 1024].shape, generator=g, device=DEV).to(torch.bfloat16)
    if own:
        from paper_2607_04031_b200 import binding as tl
        s["tables"] = tl.page_tables(s["work"]["table"], s["work"]["held"], s["work"]["holders"], page)
        if c["kind"] == "fork":
            s["cache"] = _own_cache(s["pool"])
            s["reads"] = tl.kv_batch(s["work"]["table"], s["tail_from"], s["tail"], s["tail_total"])
        elif c["kind"] == "compact":
            s["cache"] = tl.kv_cache(s["k"], s["v"])
    return s


# ------------------------------------------------------------------------------------------------------- runs

def run(s):
    return {"rope": _rope, "attend": _attend, "cache": _cache, "pages": _pages}[s["case"]["op"]](s)


def _rows(offsets, start, total):
    """For every row of a ragged batch: its request, and its place in the cache."""
    row = torch.arange(total, device=DEV)
    b = torch.searchsorted(offsets[1:].long(), row, right=True)
    return b, row - offsets[b] + start[b]


def _turned(x, positions, freq, c, inverse=False):
    """x [tokens, heads, dim] in fp32, each pair turned by its position's angle."""
    angle = positions.double()[:, None] * freq
    cos, sin = ((f(angle) * _amplitude(c)).float()[:, None] for f in (torch.cos, torch.sin))
    if inverse:
        sin = -sin
    x = x.float()
    half = c["rot"] // 2
    out = x.clone()
    if c["layout"] == "half":
        a, b = x[..., :half], x[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    return out


def _rope(s):
    c = s["case"]
    if own:
        from paper_2607_04031_b200 import binding as tl
        if c["kind"] == "rows":
            tl.rope_rows(s["rope"], s["x"], s["out"], s["positions"], inverse=c["inverse"])
            return s["out"]
        tl.rope_append(s["cache"], s["batch"], s["rope"], s["q"], s["out"], s["new_k"], s["new_v"])
        return [s["out"], s["k"], s["v"]]
    if c["kind"] == "rows":
        return _turned(s["x"], s["positions"], s["freq"], c, c["inverse"]).to(s["x"].dtype)
    b, pos = _rows(s["offsets"], s["ctx"], s["total"])
    at, line = s["table"][b, pos // c["page"]].long(), pos % c["page"]
    s["k"][at, :, line] = _turned(s["new_k"], pos, s["freq"], c).to(torch.bfloat16)
    s["v"][at, :, line] = s["new_v"]
    return [_turned(s["q"], pos, s["freq"], c).to(torch.bfloat16), s["k"], s["v"]]


def _attend(s):
    if own:
        from paper_2607_04031_b200 import binding as tl
        tl.tree_attention(s["cache"], s["batch"], s["q"], s["out"], mask=s["mask"], scale=s["scale"])
        return s["out"]
    c, ctx, most = s["case"], s["ctx"], s["most"]
    B, kv, dim, page = c["requests"], c["kv_heads"], c["dim"], c["page"]
    group = c["q_heads"] // kv
    n = s["offsets"][1:] - s["offsets"][:-1]
    pos = torch.arange(s["longest"], device=DEV)
    at = s["table"].long()[:, pos // page].clamp_min(0)
    live = pos < (ctx + n)[:, None]
    k, v = (_values(*(t[at, :, pos % page] for t in side)) for side in s["pool"])            # B, pos, kv, dim
    v = torch.where(live[:, :, None, None], v, 0.0)
    t = torch.arange(most, device=DEV)
    row = (s["offsets"][:-1, None] + t).clamp_max(s["total"] - 1)                            # B, most
    q = s["q"][row].float().view(B, most, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(B, kv, most * group, dim)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) * s["scale"]                                  # B, kv, most * group, pos
    j = pos - ctx[:, None]                                                                   # place among the step's tokens
    if s["mask"] is None:
        seen = j[:, None] <= t[:, None]
    else:
        word = s["mask"][row].long().gather(2, (j // 32).clamp(0, s["mask"].shape[1] - 1)[:, None].expand(-1, most, -1))
        seen = (word >> (j % 32)[:, None] & 1).bool() | (j < 0)[:, None]
    seen = (seen & live[:, None])[:, None, :, None].expand(-1, -1, -1, group, -1).reshape(B, 1, most * group, -1)
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v.transpose(1, 2)) / torch.where(total == 0, 1.0, total)
    o = o.view(B, kv, most, group, dim).permute(0, 2, 1, 3, 4).reshape(B, most, kv * group, dim)
    b, place = _rows(s["offsets"], torch.zeros_like(ctx), s["total"])
    return o[b, place].to(torch.bfloat16)


def _cache(s):
    c = s["case"]
    if own:
        from paper_2607_04031_b200 import binding as tl
        tl.kv_append(s["cache"], s["batch"], *s["new"])
        tl.kv_read(s["cache"], s["reads"], *s["read"])
        return list(s["read"])
    b, pos = _rows(s["offsets"], s["ctx"], s["total"])
    at, line = s["table"][b, pos // c["page"]].long(), pos % c["page"]
    back, where = _rows(s["back"], s["zero"], s["back_total"])
    back_at, back_line = s["table"][back, where // c["page"]].long(), where % c["page"]
    out = []
    for new, side in zip(s["new"], s["pool"]):
        for held, x in zip(side, _quantise(new.float())):
            held[at, :, line] = x
        out.append(_values(*(t[back_at, :, back_line] for t in side)).to(torch.bfloat16))
    return out


def _forked(table, held, holders, from_, to, tokens, page):
    n = torch.minimum(-(-tokens // page), held[from_])
    col = torch.arange(table.shape[1], device=DEV)
    mine = col[None] < n[:, None]
    got = table[from_]
    table[to] = torch.where(mine, got, table[to])
    held[to] = n
    holders.scatter_add_(0, torch.where(mine, got, 0).long().flatten(), mine.int().flatten())


def _released(table, held, holders, keep, page):
    kept = torch.where(keep < 0, held, torch.minimum(-(-keep.clamp_min(0) // page), held))
    col = torch.arange(table.shape[1], device=DEV)
    gone = (col[None] >= kept[:, None]) & (col[None] < held[:, None])
    holders.scatter_add_(0, torch.where(gone, table, 0).long().flatten(), -gone.int().flatten())
    table.copy_(torch.where(gone, -1, table))
    held.copy_(kept)


def _reserved(table, held, holders, start, wanted, page, most):
    """Pages for the positions start .. wanted - 1 of every request, none of them anybody else's: (moves, how many, missing)."""
    B, W = table.shape
    P = holders.numel()
    col = torch.arange(W, device=DEV)[None]
    need = torch.where(wanted < 0, 0, (-(-wanted.clamp_min(0) // page)).clamp_max(W))[:, None]
    first, have = (start.clamp_min(0) // page)[:, None], held[:, None]
    writes = (wanted > start)[:, None] & (col >= first) & (col < need) & (col < have)
    at = torch.where(writes, table, P).long()
    count = torch.cat([holders, holders.new_zeros(1)])
    shared = writes & (count[at] > 1)
    # where every holder is about to write, the first of them keeps the page
    here = torch.zeros(P + 1, dtype=torch.int32, device=DEV).scatter_add_(0, torch.where(shared, at, P).flatten(), shared.int().flatten())
    order = torch.arange(B * W, device=DEV).view(B, W)
    lowest = torch.full((P + 1,), B * W, device=DEV).scatter_reduce_(0, torch.where(shared, at, P).flatten(), order.flatten(), "amin")
    stays = shared & (here[at] == count[at]) & (lowest[at] == order)
    leaves = shared & ~stays
    fresh = leaves | (col >= have) & (col < need)
    rank = fresh.flatten().cumsum(0).view(B, W) - 1
    free = (holders == 0)
    total, there = fresh.sum(), free.sum()
    missing = (total - there).clamp_min(0).to(torch.int32).view(1)
    place = torch.full((P + B * W + 1,), -1, device=DEV)
    place.scatter_(0, torch.where(free, free.cumsum(0) - 1, P + B * W), torch.arange(P, device=DEV))
    go = missing == 0
    new = place[rank.clamp_min(0)].to(torch.int32)
    copied = leaves & (col == first) & (start % page != 0)[:, None] & go
    line = torch.where(copied.any(1), copied.any(1).cumsum(0) - 1, most)
    moves = torch.full((most + 1, 3), -1, dtype=torch.int32, device=DEV)
    pick = first.clamp_max(W - 1).long()
    moves[line] = torch.stack([table.gather(1, pick)[:, 0], new.gather(1, pick)[:, 0], (start % page).to(torch.int32)], 1)
    holders.copy_(torch.where(go, (count.scatter_add(0, torch.where(leaves, at, P).flatten(), -leaves.int().flatten()))[:P], holders))
    took = torch.where(fresh & go, new, P).long().flatten()
    holders.copy_(torch.cat([holders, holders.new_zeros(1)]).scatter(0, took, 1)[:P])
    table.copy_(torch.where(fresh & go, new, table))
    held.copy_(torch.where(go, torch.maximum(held, need[:, 0].to(torch.int32)), held))
    return moves[:most], copied.sum().to(torch.int32).view(1), missing


def _compacted(table, held, holders):
    """The highest pages in use change places with the lowest free ones: (from, to), as many as lie on the wrong side."""
    P = holders.numel()
    live = holders > 0
    n = live.sum()
    at = torch.arange(P, device=DEV)
    frees, lives = at[~live], at[live].flip(0)
    k = int((frees < n).sum())
    from_, to = lives[:k], frees[:k]
    new = torch.arange(P + 1, device=DEV)
    new[from_] = to
    col = torch.arange(table.shape[1], device=DEV)
    table.copy_(torch.where(col[None] < held[:, None], new[table.long()].to(torch.int32), table))
    holders[to] = holders[from_]
    holders[from_] = 0
    return from_, to, n.to(torch.int32).view(1)


def _pages(s):
    c, page = s["case"], s["case"]["page"]
    # each pass begins from the same tables, as a scheduler hands them over; the calls change them in place
    w = s["work"]
    for k in w:
        w[k].copy_(s[k])
    out = [w["table"], w["held"], w["holders"]]
    if own:
        from paper_2607_04031_b200 import binding as tl
        if c["kind"] == "compact":
            tl.page_compact(s["tables"], s["moves"], s["n_moves"], s["missing"])
            tl.page_copy(s["cache"], s["moves"], s["n_moves"])
            return out + [s["moves"], s["n_moves"], s["missing"], s["k"], s["v"]]
        if c["kind"] == "fork":
            tl.page_fork(s["tables"], s["from"], s["to"], s["tokens"])
        else:
            tl.page_release(s["tables"], s["keep"])
        tl.page_reserve(s["tables"], s["start"], s["wanted"], s["moves"], s["n_moves"], s["missing"])
        if c["kind"] == "turn":
            return out + [s["moves"], s["n_moves"], s["missing"]]
        tl.page_copy(s["cache"], s["moves"], s["n_moves"])
        tl.kv_read(s["cache"], s["reads"], *s["read"])
        return out + [s["moves"], s["n_moves"], s["missing"]] + s["read"]
    if c["kind"] == "compact":
        from_, to, live = _compacted(*out)
        moves = torch.full_like(s["moves"], -1)
        moves[:from_.numel()] = torch.stack([from_, to, torch.full_like(to, page)], 1).to(torch.int32)
        for t in (s["k"], s["v"]):
            t[to] = t[from_]
        return out + [moves, torch.full((1,), from_.numel(), dtype=torch.int32, device=DEV), live, s["k"], s["v"]]
    if c["kind"] == "fork":
        _forked(*out, s["from"].long(), s["to"].long(), s["tokens"], page)
    else:
        _released(*out, s["keep"], page)
    moves, n, missing = _reserved(*out, s["start"], s["wanted"], page, s["moves"].shape[0])
    if c["kind"] == "turn":
        return out + [moves, n, missing]
    m = moves[moves[:, 0] >= 0].long()
    line = torch.arange(page, device=DEV)
    b, pos = _rows(s["tail"], s["tail_from"], s["tail_total"])
    at = w["table"][b, pos // page].long()
    read = []
    for side in s["pool"]:
        for t in side:
            t = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
            keep = (line[None] < m[:, 2:]).view(len(m), 1, page, *[1] * (t.dim() - 3))
            t[m[:, 1]] = torch.where(keep, t[m[:, 0]], t[m[:, 1]])
        read.append(_values(*(t[at, :, pos % page] for t in side)).to(torch.bfloat16))
    return out + [moves, n, missing] + read


# ------------------------------------------------------------------------------------------------------ exact

def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "cache": _exact_cache, "pages": _exact_pages}[case["op"]](s)


def _exact_turned(x, positions, c, inverse=False):
    z = x.double()
    half = c["rot"] // 2
    pair = [(i, i + half) if c["layout"] == "half" else (2 * i, 2 * i + 1) for i in range(half)]
    freq = _frequencies(c)
    out = z.clone()
    for i, (p, q) in enumerate(pair):
        turn = torch.polar(torch.full((x.shape[0],), _amplitude(c), dtype=torch.float64, device=DEV),
                           positions.double() * freq[i] * (-1.0 if inverse else 1.0))[:, None]
        r = torch.complex(z[..., p], z[..., q]) * turn
        out[..., p], out[..., q] = r.real, r.imag
    return out


def _request(s, b):
    first, end = s["offsets"][b:b + 2].tolist()
    return first, end - first


def _exact_rope(s):
    c = s["case"]
    if c["kind"] == "rows":
        return _exact_turned(s["x"], s["positions"], c, c["inverse"])
    pos = torch.cat([int(s["ctx"][b]) + torch.arange(_request(s, b)[1], device=DEV) for b in range(c["requests"])])
    k, v = s["k"].double(), s["v"].double()
    new = _exact_turned(s["new_k"], pos, c)
    for b in range(c["requests"]):
        first, m = _request(s, b)
        for i in range(m):
            p = int(s["ctx"][b]) + i
            at = int(s["table"][b, p // c["page"]])
            k[at, :, p % c["page"]] = new[first + i]
            v[at, :, p % c["page"]] = s["new_v"][first + i].double()
    return [_exact_turned(s["q"], pos, c), k, v]


def _exact_attend(s):
    c = s["case"]
    if sum((x + m) * m for x, m in zip(contexts(c), counts(c))) * c["q_heads"] * c["dim"] > 4e11:
        return None
    group = c["q_heads"] // c["kv_heads"]
    out = torch.zeros(s["total"], c["q_heads"], c["dim"], dtype=torch.float64, device=DEV)
    for b in range(c["requests"]):
        first, m = _request(s, b)
        ctx = int(s["ctx"][b])
        where = torch.arange(ctx + m, device=DEV)
        pg, line = s["table"][b].long()[where // c["page"]], where % c["page"]
        seen = torch.ones(m, ctx + m, dtype=torch.bool, device=DEV)
        for i in range(m):
            if s["mask"] is None:
                seen[i, ctx + i + 1:] = False
            else:
                words = [w & 0xffffffff for w in s["mask"][first + i].tolist()]
                seen[i, ctx:] = torch.tensor([(words[j // 32] >> (j % 32)) & 1 == 1 for j in range(m)], device=DEV)
        for h in range(c["kv_heads"]):
            key, value = (_exact_values(*(t[pg, h, line] for t in side)) for side in s["pool"])
            for e in range(h * group, (h + 1) * group):
                z = s["q"][first:first + m, e].double() @ key.T * s["scale"]
                z = z.masked_fill(~seen, -math.inf)
                out[first:first + m, e] = torch.nan_to_num(torch.softmax(z, -1)) @ value
    return out


def _two(k):
    """2^k, exactly (a device's power function may be off by its last bit, and ties with it)."""
    return (k.long() + 1023 << 52).view(torch.float64)


def _exact_values(codes, group, scale):
    """From the bits: sign, two of exponent, one of mantissa."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    e, m = c >> 1 & 3, c & 1
    v = torch.where(e > 0, (1 + 0.5 * m.double()) * _two(e - 1), 0.5 * m.double())
    v = torch.where(c >= 8, -v, v)
    return v * group.double().repeat_interleave(16, -1) * scale.double()[..., None]


def _exact_held(x):
    """What a row's values become in the 4-bit cache, from the definition in 64 bits."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    s = _two(torch.ceil(torch.log2(top.clamp_min(1e-300) / 2688.0)))
    s = torch.where(s / 2 * 2688.0 >= top, s / 2, torch.where(s * 2688.0 < top, s * 2, s))  # (the logarithm's rounding)
    y = (x / s).unflatten(-1, (-1, 16))
    want = y.abs().amax(-1, keepdim=True) / 6.0
    step = _two(torch.floor(torch.log2(want.clamp_min(2.0 ** -6))) - 3)                     # E4M3: three bits behind the first
    g = torch.round(want / step) * step
    a = y.abs() / torch.where(g > 0, g, 1.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp_max(6.0)
    out = (torch.copysign(a, y) * g).flatten(-2) * s
    return torch.where(top > 0, out, torch.zeros_like(out))


def _exact_cache(s):
    c = s["case"]
    outs = []
    for new, side in zip(s["new"], s["pool"]):
        held, rows = _exact_held(new), []
        for b in range(c["requests"]):
            first, m = _request(s, b)
            where = torch.arange(int(s["ctx"][b]), device=DEV)
            pg, line = s["table"][b].long()[where // c["page"]], where % c["page"]
            rows += [_exact_values(*(t[pg, :, line] for t in side)), held[first:first + m]]
        outs.append(torch.cat(rows))
    return outs


def _exact_pages(s):
    """Page by page, with lists."""
    c, page = s["case"], s["case"]["page"]
    table, held, holders = (s[k].tolist() for k in ("table", "held", "holders"))
    moves = []
    missing = 0
    if c["kind"] == "compact":
        live = sum(h > 0 for h in holders)
        low, high = 0, len(holders) - 1
        went = {}
        while True:
            while low < len(holders) and holders[low] > 0:
                low += 1
            while high >= 0 and holders[high] == 0:
                high -= 1
            if low >= high:
                break
            moves.append((high, low, page))
            went[high] = low
            holders[low], holders[high] = holders[high], 0
        for b, row in enumerate(table):
            row[:held[b]] = [went.get(p, p) for p in row[:held[b]]]
        missing = live
    elif c["kind"] == "fork":
        for f, t, n in zip(s["from"].tolist(), s["to"].tolist(), s["tokens"].tolist()):
            held[t] = min(-(-n // page), held[f])
            for e in range(held[t]):
                table[t][e] = table[f][e]
                holders[table[f][e]] += 1
    else:
        for b, n in enumerate(s["keep"].tolist()):
            while n >= 0 and held[b] > -(-n // page):
                held[b] -= 1
                holders[table[b][held[b]]] -= 1
                table[b][held[b]] = -1
    if c["kind"] != "compact":
        start, wanted = s["start"].tolist(), s["wanted"].tolist()
        writes = {}
        for b in range(len(table)):
            if wanted[b] > start[b]:
                for e in range(start[b] // page, min(-(-wanted[b] // page), held[b])):
                    writes.setdefault(table[b][e], []).append((b, e))
        leave = set()
        for p, places in writes.items():
            if holders[p] > 1:
                leave.update(places[1:] if len(places) == holders[p] else places)
        free = [p for p, h in enumerate(holders) if h == 0]
        fresh = [(b, e) for b in range(len(table)) if wanted[b] >= 0 for e in range(min(-(-wanted[b] // page), len(table[b])))
                 if e >= held[b] or (b, e) in leave]
        missing = max(0, len(fresh) - len(free))
        if missing == 0:
            for (b, e), p in zip(fresh, free):
                if (b, e) in leave:
                    holders[table[b][e]] -= 1
                    if e == start[b] // page and start[b] % page:
                        moves.append((table[b][e], p, start[b] % page))
                table[b][e], holders[p] = p, 1
                held[b] = max(held[b], e + 1)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    out = [i32(table), i32(held), i32(holders), i32([list(m) for m in moves] + [[-1] * 3] * (s["moves"].shape[0] - len(moves))),
           i32([len(moves)]), i32([missing])]
    if c["kind"] == "compact":
        pools = [s["k"].clone(), s["v"].clone()]
        for t in pools:
            for f, to, _ in moves:
                t[to] = s["k" if t is pools[0] else "v"][f]
        out += [t.double() for t in pools]
    elif c["kind"] == "fork":
        for side in s["pool"]:
            held_ = _exact_values(*side)
            for f, to, n in moves:
                held_[to, :, :n] = held_[f, :, :n].clone()
            rows = []
            for b, n in enumerate((s["tail"][1:] - s["tail"][:-1]).tolist()):
                p = int(s["tail_from"][b])
                if n:
                    rows.append(held_[table[b][p // page], :, :n].permute(1, 0, 2))
            outs = torch.cat(rows) if rows else torch.zeros(0, c["kv_heads"], c["dim"], dtype=torch.float64, device=DEV)
            out.append(outs)
    return out
