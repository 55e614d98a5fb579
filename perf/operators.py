"""What is measured of the operators around a paged, quantised key/value cache that serves drafted tokens:

  cache    new keys and values are quantised into the pages of the cache, accepted ones are moved together, tokens are read back
  attend   attention of a step's tokens (one per request, a chain, or a tree of drafts) over that cache
  verify   which drafted tokens the target's probabilities keep, and the token that follows them

`run` computes each with elementary torch operations, or, where `own` is true, through the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
FORMATS = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}


# ------------------------------------------------------------------------------------------------------ cases

def attend_case(name, requests, tokens, ctx, q_heads, kv_heads, dim, fmt, page, tree):
    return {"name": name, "op": "attend", "requests": requests, "tokens": tokens, "ctx": ctx, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "format": fmt, "page": page, "tree": tree}


def cache_case(name, kind, requests, tokens, ctx, kv_heads, dim, fmt, page):
    return {"name": name, "op": "cache", "kind": kind, "requests": requests, "tokens": tokens, "ctx": ctx,
            "kv_heads": kv_heads, "dim": dim, "format": fmt, "page": page}


def verify_case(name, requests, tokens, branch, vocab, drafts):
    return {"name": name, "op": "verify", "requests": requests, "tokens": tokens, "branch": branch, "vocab": vocab,
            "drafts": drafts}


def listed():
    return [
        # one user at the start of a conversation, no drafts: the latency of a single token (Qwen-3 heads, 4 KB pages per head)
        attend_case("attend 1x1 short", 1, 1, 407, 32, 4, 128, "bf16", 16, False),
        # ordinary decoding of a batch, one token per request (Llama-3.1 70B heads, pages of 4 KB per head)
        attend_case("attend 32x1", 32, 1, 4100, 64, 8, 128, "e4m3", 32, False),
        # a chain of four drafts behind the last token, small batch
        attend_case("attend 8x5 chain", 8, 5, 2900, 64, 8, 128, "int8", 32, False),
        # odd sizes: three query heads per key head, 64-wide heads, a ragged tree
        attend_case("attend 4x13 tree d64", 4, 13, 1531, 24, 8, 64, "e4m3", 64, True),
        # trees of 32 drafts, contexts of a few thousand tokens
        attend_case("attend 8x32 tree", 8, 32, 8000, 64, 8, 128, "e4m3", 32, True),
        # one user with a very long context and a wide tree, unquantised cache
        attend_case("attend 1x64 tree long", 1, 64, 100000, 64, 8, 128, "bf16", 16, True),
        # trees of 16 drafts in a large batch: the largest
        attend_case("attend 48x16 tree", 48, 16, 6000, 64, 8, 128, "int8", 64, True),
        # one step's bookkeeping at a small batch: write the tree, keep the accepted path, read it back
        cache_case("cache step 4x7", "step", 4, 7, 1000, 4, 128, "e4m3", 32),
        # a prompt's chunk quantised on its way in, and the whole context read back (for a chunk that follows)
        cache_case("cache fill 4x2048", "fill", 4, 2048, 6000, 8, 128, "int8", 32),
        # a chain of four drafts for one request
        verify_case("verify 1x5 chain", 1, 5, 1, 32000, True),
        # trees of 16 nodes with up to three alternatives each, a batch
        verify_case("verify 32x16 tree", 32, 16, 3, 128256, True),
        # drafts chosen without a distribution (the likeliest continuations), ragged vocabulary
        verify_case("verify 16x24 given", 16, 24, 4, 100003, False),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["attend", "attend", "attend", "cache", "verify"])
        if op == "attend":
            kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 8, 16])
            tree = rng.random() < 0.6
            c = attend_case("", _spread(rng, 1, 64), _spread(rng, 1, 64), _spread(rng, 1, 100000), kv * group, kv,
                            rng.choice([64, 128, 128, 256]), rng.choice(["bf16", "e4m3", "int8"]), rng.choice([16, 32, 64, 128]), tree)
        elif op == "cache":
            kind = rng.choice(["step", "fill"])
            c = cache_case("", kind, _spread(rng, 1, 64), _spread(rng, 1, 64) if kind == "step" else _spread(rng, 1, 4096),
                           _spread(rng, 1, 8000), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256]),
                           rng.choice(["bf16", "e4m3", "int8"]), rng.choice([16, 32, 64, 128]))
        else:
            c = verify_case("", _spread(rng, 1, 32), _spread(rng, 1, 24), rng.randint(1, 4), _spread(rng, 1000, 128256),
                            rng.random() < 0.6)
        c.pop("name")
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and _plain_floats(c) <= 1.2e9:
            return c


def _plain_floats(c):
    """The largest intermediate of the plain form, in values: it bounds what a drawn case may hold."""
    if c["op"] != "attend":
        return c["requests"] * c["tokens"] * c.get("vocab", 1)
    return c["requests"] * c["ctx"] * (c["tokens"] * c["q_heads"] + 2 * c["kv_heads"] * c["dim"])


def contexts(c):
    """Tokens in the cache before the step, request by request: from half of ctx to all of it, one request with all."""
    return [max(0, int(c["ctx"] * (1.0 - 0.5 * ((0.6180339887 * b) % 1.0)))) for b in range(c["requests"])]


def counts(c):
    """The step's tokens, request by request: trees and steps are ragged, the first request has the most."""
    if c["op"] == "cache" and c["kind"] == "fill" or c["op"] == "attend" and not c["tree"]:
        return [c["tokens"]] * c["requests"]
    return [max(1, int(c["tokens"] * (1.0 - 0.4 * ((0.7548776662 * b) % 1.0)))) for b in range(c["requests"])]


def kept(c):
    """How many of a request's tokens are accepted in a `cache step` case (the first always is)."""
    return [1 + (3 * b + 2) % min(n, 6) if n > 1 else 1 for b, n in enumerate(counts(c))]


def work(c):
    n, total = counts(c), sum(counts(c))
    if c["op"] == "verify":
        # a row of the target's probabilities per request, and one of the drafter's where it has one (a request whose
        # drafts are all kept needs the first alone; one whose early draft is refused needs more than one of each)
        rows = 2 if c["drafts"] else 1
        return {"bytes": 4.0 * c["requests"] * rows * c["vocab"] + 24.0 * total, "flops": 2.0 * c["requests"] * rows * c["vocab"]}
    item = 2 if c["format"] == "bf16" else 1
    row = 2 * c["kv_heads"] * (c["dim"] * item + (0 if c["format"] == "bf16" else 4))        # a token's keys and values
    if c["op"] == "cache":
        wide = 2 * c["kv_heads"] * c["dim"] * 2                                              # the same in bf16
        if c["kind"] == "step":
            k = sum(kept(c))
            return {"bytes": float(total * (wide + row) + 2 * k * row + k * (row + wide)), "flops": 4.0 * total * row}
        back = sum(contexts(c)) + total
        return {"bytes": float(total * (wide + row) + back * (row + wide)), "flops": 4.0 * (total + back) * row}
    q = 2 * c["q_heads"] * c["dim"] * 2
    # every token sees the whole context, its own chain or branch behind that
    pairs = sum((x + (m + 1) / 2 if not c["tree"] else x + math.log2(m + 1)) * m for x, m in zip(contexts(c), n))
    return {"bytes": float(sum(x + m for x, m in zip(contexts(c), n)) * row + total * q),
            "flops": 4.0 * pairs * c["q_heads"] * c["dim"]}


# ----------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 11)
    return g


def _quantise(x, fmt):
    """x [..., dim] (fp32) -> codes and one scale per row, as the cache holds them."""
    if fmt == "bf16":
        return x.to(torch.bfloat16), None
    scale = x.abs().amax(-1) / TOP[fmt]
    y = x / scale.clamp_min(1e-30).unsqueeze(-1)
    return (y.round() if fmt == "int8" else y).clamp(-TOP[fmt], TOP[fmt]).to(FORMATS[fmt]), scale


def _offsets(n):
    return torch.tensor([0] + n, device=DEV).cumsum(0).to(torch.int32)


def _parents(n, branch, g_host):
    """Trees by request (node 0 is the root, parents before children, at most `branch` children of one node), in one list."""
    out = []
    for m in n:
        own_, used = [-1], [0]
        for i in range(1, m):
            if branch == 1:
                p = i - 1
            else:
                free = [j for j in range(i) if used[j] < branch]
                p = free[max(0, len(free) - 1 - int(g_host.expovariate(0.5)))]      # mostly recent nodes: trees grow deep
            used[p] += 1
            own_.append(p)
            used.append(0)
        out.append(own_)
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


def _pages(c, n, g):
    """A shuffled page table wide enough for every request, and how many pages there are."""
    per = [-(-(x + m) // c["page"]) for x, m in zip(contexts(c), n)]
    width = max(per)
    order = torch.randperm(sum(per) + 3, generator=g, device=DEV).to(torch.int32)
    at = torch.tensor([0] + per, device=DEV).cumsum(0)
    col = torch.arange(width, device=DEV)
    real = col[None] < torch.tensor(per, device=DEV)[:, None]
    return torch.where(real, order[(at[:-1, None] + col).clamp_max(order.numel() - 1)], 0).to(torch.int32).contiguous(), order.numel()


def _filled(c, pages, g):
    """A cache of `pages` pages with keys and values in it, some channels larger than the others as in trained models."""
    shape = (pages, c["kv_heads"], c["page"], c["dim"])
    wide = torch.ones(c["dim"], device=DEV)
    wide[:: 16] = 2.5
    out = []
    for spread in (wide, torch.ones_like(wide)):
        codes, scales = torch.empty(shape, dtype=FORMATS[c["format"]], device=DEV), None
        if c["format"] != "bf16":
            scales = torch.empty(shape[:3], device=DEV)
        for a in range(0, pages, 4096):
            x = torch.randn((min(4096, pages - a),) + shape[1:], generator=g, device=DEV) * spread
            q, s = _quantise(x, c["format"])
            codes[a:a + 4096] = q
            if s is not None:
                scales[a:a + 4096] = s
        out += [codes, scales]
    return out[0], out[2], out[1], out[3]


def prepare(case, seed):
    import random
    g, n = _gen(seed), counts(case)
    host = random.Random(int(seed))
    s = {"case": case, "offsets": _offsets(n), "total": sum(n), "most": max(n)}
    if case["op"] == "verify":
        B, V = case["requests"], case["vocab"]
        trees = _parents(n, case["branch"], host)
        N = s["total"]
        z = torch.randn(N, V, generator=g, device=DEV) * 2.5
        p = torch.softmax(z, -1)
        z += torch.randn(N, V, generator=g, device=DEV) * 0.6
        q = torch.softmax(z, -1)
        first = s["offsets"].tolist()
        parent_row = torch.tensor([first[b] + max(v, 0) for b, t in enumerate(trees) for v in t], device=DEV)
        if case["drafts"]:      # each draft is drawn from the drafter's distribution at its parent
            race = torch.empty(N, V, device=DEV).exponential_(generator=g)
            token = (q[parent_row] / race).argmax(-1)
        else:                   # siblings are the drafter's likeliest tokens, in order
            place, seen = [], {}
            for b, t in enumerate(trees):
                for v in t:
                    seen[b, v] = seen.get((b, v), -1) + 1
                    place.append(seen[b, v])
            best = q.topk(max(place) + 1, -1).indices
            token = best[parent_row, torch.tensor(place, device=DEV)]
        words = -(-s["most"] // 32)
        s.update(target=p, drafts=q if case["drafts"] else None, tokens=token.to(torch.int32),
                 parents=torch.tensor([v for t in trees for v in t], dtype=torch.int32, device=DEV), mask=_mask(trees, words),
                 accept=torch.rand(N, generator=g, device=DEV), sample=torch.rand(B, generator=g, device=DEV),
                 rounds=case["branch"], accepted=torch.empty(B, s["most"], dtype=torch.int32, device=DEV),
                 n_accepted=torch.empty(B, dtype=torch.int32, device=DEV), next=torch.empty(B, dtype=torch.int32, device=DEV))
        return s
    s["ctx"] = torch.tensor(contexts(case), dtype=torch.int32, device=DEV)
    s["longest"] = max(x + m for x, m in zip(contexts(case), n))
    s["table"], pages = _pages(case, n, g)
    s["k"], s["v"], s["ks"], s["vs"] = _filled(case, pages, g)
    kv, dim, heads = case["kv_heads"], case["dim"], case.get("q_heads", case["kv_heads"])
    # the product that gives queries, keys and values of the step: one row per token
    qkv = torch.randn(s["total"], (heads + 2 * kv) * dim, generator=g, device=DEV).to(torch.bfloat16)
    s["q"] = qkv[:, :heads * dim].view(-1, heads, dim)
    s["new_k"] = qkv[:, heads * dim:(heads + kv) * dim].view(-1, kv, dim)
    s["new_v"] = qkv[:, (heads + kv) * dim:].view(-1, kv, dim)
    if case["op"] == "attend":
        s["scale"] = 1.0 / math.sqrt(dim)
        s["out"] = torch.empty(s["total"], heads, dim, dtype=torch.bfloat16, device=DEV)
        s["mask"] = _mask(_parents(n, 4, host), -(-s["most"] // 32)) if case["tree"] else None
    else:
        back = kept(case) if case["kind"] == "step" else [x + m for x, m in zip(contexts(case), n)]
        s["back"], s["back_total"], s["back_most"] = _offsets(back), sum(back), max(back)
        s["back_from"] = s["ctx"] if case["kind"] == "step" else torch.zeros_like(s["ctx"])
        path = [sorted([0] + host.sample(range(1, m), k - 1)) for m, k in zip(n, kept(case))] if case["kind"] == "step" else []
        s["accepted"] = torch.tensor([p + [-1] * (s["most"] - len(p)) for p in path], dtype=torch.int32, device=DEV)
        s["n_accepted"] = torch.tensor(back, dtype=torch.int32, device=DEV)
        s["new_len"] = torch.empty_like(s["ctx"])
        s["k_back"] = torch.empty(s["back_total"], kv, dim, dtype=torch.bfloat16, device=DEV)
        s["v_back"] = torch.empty_like(s["k_back"])
    if own:
        from paper_2607_04031_b200 import binding as tl
        s["cache"] = tl.kv_cache(s["k"], s["v"], s["ks"], s["vs"])
        s["batch"] = tl.kv_batch(s["table"], s["ctx"], s["offsets"], s["total"])
        if case["op"] == "cache":
            s["reads"] = tl.kv_batch(s["table"], s["back_from"], s["back"], s["back_total"])
    return s


# ------------------------------------------------------------------------------------------------------- runs

def run(s):
    return {"attend": _attend, "cache": _cache, "verify": _verify}[s["case"]["op"]](s)


def _rows(offsets, start, total):
    """For every row of a ragged batch: its request, and its place in the cache."""
    row = torch.arange(total, device=DEV)
    b = torch.searchsorted(offsets[1:].long(), row, right=True)
    return b, row - offsets[b] + start[b]


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
    at = s["table"].long()[:, pos // page]
    live = pos < (ctx + n)[:, None]
    k, v = s["k"][at, :, pos % page].float(), s["v"][at, :, pos % page].float()              # B, pos, kv, dim
    if s["ks"] is not None:
        k = k * s["ks"][at, :, pos % page].unsqueeze(-1)
        v = v * s["vs"][at, :, pos % page].unsqueeze(-1)
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
        tl.kv_append(s["cache"], s["batch"], s["new_k"], s["new_v"])
        if c["kind"] == "step":
            tl.kv_commit(s["cache"], s["batch"], s["accepted"], s["n_accepted"], s["new_len"])
        tl.kv_read(s["cache"], s["reads"], s["k_back"], s["v_back"])
        return [s["k_back"], s["v_back"]] + ([s["new_len"]] if c["kind"] == "step" else [])
    page = c["page"]
    b, pos = _rows(s["offsets"], s["ctx"], s["total"])
    at = s["table"][b, pos // page].long()
    back, from_ = _rows(s["back"], s["back_from"], s["back_total"])
    back_at = s["table"][back, from_ // page].long()
    if c["kind"] == "step":
        src = from_ - s["ctx"][back]
        src = s["ctx"][back] + s["accepted"][back, src]
        src_at = s["table"][back, src // page].long()
    out = []
    for new, codes, scales in ((s["new_k"], s["k"], s["ks"]), (s["new_v"], s["v"], s["vs"])):
        x, scale = _quantise(new.float(), c["format"])
        codes[at, :, pos % page] = x
        if scale is not None:
            scales[at, :, pos % page] = scale
        if c["kind"] == "step":
            codes[back_at, :, from_ % page] = codes[src_at, :, src % page]
            if scale is not None:
                scales[back_at, :, from_ % page] = scales[src_at, :, src % page]
        y = codes[back_at, :, from_ % page].float()
        out.append((y if scale is None else y * scales[back_at, :, from_ % page].unsqueeze(-1)).to(torch.bfloat16))
    return out + ([s["ctx"] + s["n_accepted"]] if c["kind"] == "step" else [])


def _verify(s):
    c = s["case"]
    if own:
        from paper_2607_04031_b200 import binding as tl
        tl.tree_verify(s["target"], s["drafts"], s["tokens"], s["parents"], s["offsets"], s["accept"], s["sample"],
                       s["accepted"], s["n_accepted"], s["next"])
        return [s["accepted"], s["n_accepted"], s["next"]]
    # Sums over the vocabulary decide which whole numbers come out: they are taken in 64 bits, so that their rounding
    # does not. Every node of every tree is looked at side by side; the loop is over the alternatives of a node.
    N, most = s["total"], s["most"]
    b, place = _rows(s["offsets"], torch.zeros_like(s["offsets"][:-1]), N)
    first = s["offsets"][b].long()
    parent = s["parents"].long()
    parent_row = first + parent.clamp_min(0)
    row = torch.arange(N, device=DEV)
    sibling = (parent_row[:, None] == parent_row) & (parent >= 0)[:, None] & (parent >= 0)
    order = (sibling & (row[None] < row[:, None])).sum(1)                                   # place among the siblings
    u, token = s["accept"].double(), s["tokens"].long()
    r, mass = s["target"].double(), torch.ones(N, dtype=torch.float64, device=DEV)
    chosen, open_ = torch.full((N,), -1, device=DEV), torch.ones(N, dtype=torch.bool, device=DEV)
    for k in range(s["rounds"]):
        child = torch.full((N + 1,), -1, device=DEV).scatter(0, torch.where((order == k) & (parent >= 0), parent_row, N), row)[:N]
        there, at = (child >= 0) & open_, child.clamp_min(0)
        x = token[at]
        rx = r.gather(1, x[:, None])[:, 0]
        qx = s["drafts"].gather(1, x[:, None])[:, 0].double() if s["drafts"] is not None else 1.0
        ok = there & (u[at] * qx * mass < rx)
        chosen, no = torch.where(ok, at, chosen), there & ~ok
        if s["drafts"] is not None:
            less = (r - mass[:, None] * s["drafts"]).clamp_min(0)
            rest = less.sum(1)
        else:
            less = r.scatter(1, x[:, None], 0.0)
            rest = mass - torch.minimum(rx, mass)
        empty = no & (rest <= 0)
        r = torch.where((no & ~empty)[:, None], less, r)
        r = torch.where(empty[:, None], s["target"], r)
        mass = torch.where(no, rest, mass)
        open_ = open_ & ~ok & ~empty
    taken = (parent < 0) | (chosen[parent_row] == row)
    bits = (s["mask"].long()[:, torch.arange(most, device=DEV) // 32] >> (torch.arange(most, device=DEV) % 32) & 1).bool()
    inside = taken[(first[:, None] + torch.arange(most, device=DEV)).clamp_max(N - 1)]
    path = (inside | ~bits).all(1)                                                          # the node and all before it were taken
    slot = torch.where(path, place, most)
    grid = torch.full((c["requests"], most), most, device=DEV)
    grid[b, place] = slot
    grid = grid.sort(1).values
    length = (grid < most).sum(1)
    last = s["offsets"][:-1].long() + grid.gather(1, length[:, None] - 1)[:, 0]
    r = r[last]
    cum = r.cumsum(1)
    nth = (cum <= s["sample"].double()[:, None] * cum[:, -1:]).sum(1)
    top = torch.where(r > 0, torch.arange(r.shape[1], device=DEV), -1).amax(1)
    return [torch.where(grid < most, grid, -1).to(torch.int32), length.to(torch.int32), torch.minimum(nth, top).to(torch.int32)]


# ------------------------------------------------------------------------------------------------------ exact

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "cache": _exact_cache, "verify": _exact_verify}[case["op"]](s)


def _request(s, b):
    first, end = s["offsets"][b:b + 2].tolist()
    return first, end - first


def _exact_attend(s):
    c = s["case"]
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
            key, value = s["k"][pg, h, line].double(), s["v"][pg, h, line].double()
            if s["ks"] is not None:
                key, value = key * s["ks"][pg, h, line].double()[:, None], value * s["vs"][pg, h, line].double()[:, None]
            for e in range(h * group, (h + 1) * group):
                z = s["q"][first:first + m, e].double() @ key.T * s["scale"]
                z = z.masked_fill(~seen, -math.inf)
                out[first:first + m, e] = torch.nan_to_num(torch.softmax(z, -1)) @ value
    return out


def _exact_cache(s):
    c = s["case"]
    outs = []
    for new, codes, scales in ((s["new_k"], s["k"], s["ks"]), (s["new_v"], s["v"], s["vs"])):
        if c["format"] == "bf16":
            held = new.double()
        else:
            scale = new.double().abs().amax(-1, keepdim=True) / TOP[c["format"]]
            y = torch.where(scale > 0, new.double() / scale, 0.0)
            held = scale * (y.round() if c["format"] == "int8" else y.to(torch.float8_e4m3fn).double())
        rows = []
        for b in range(c["requests"]):
            first, m = _request(s, b)
            if c["kind"] == "step":
                k = int(s["n_accepted"][b])
                rows.append(held[first + s["accepted"][b, :k].long()])
                continue
            where = torch.arange(int(s["ctx"][b]), device=DEV)
            pg, line = s["table"][b].long()[where // c["page"]], where % c["page"]
            old = codes[pg, :, line].double()
            rows += [old if scales is None else old * scales[pg, :, line].double().unsqueeze(-1), held[first:first + m]]
        outs.append(torch.cat(rows))
    return outs + ([(s["ctx"] + s["n_accepted"]).to(torch.int32)] if c["kind"] == "step" else [])


def _exact_verify(s):
    c = s["case"]
    parents, tokens, accept = s["parents"].tolist(), s["tokens"].tolist(), s["accept"].tolist()
    paths, lengths, nexts = [], [], []
    for b in range(c["requests"]):
        first, m = _request(s, b)
        path, node = [0], 0
        while True:
            r, mass, went = s["target"][first + node].double(), 1.0, None
            for child in [i for i in range(node + 1, m) if parents[first + i] == node]:
                x, u = tokens[first + child], accept[first + child]
                q = s["drafts"][first + node].double() if s["drafts"] is not None else None
                if u * (1.0 if q is None else float(q[x])) * mass < float(r[x]):
                    went = child
                    break
                if q is None:
                    mass -= min(float(r[x]), mass)
                    less = r.clone()
                    less[x] = 0
                else:
                    less = torch.relu(r - mass * q)
                    mass = float(less.sum())
                if mass <= 0:
                    r = s["target"][first + node].double()
                    break
                r = less
            if went is None:
                break
            path.append(went)
            node = went
        cum = torch.cumsum(r, 0)
        at = int(torch.searchsorted(cum, cum[-1:] * float(s["sample"][b]), right=True))
        nexts.append(min(at, int(torch.nonzero(r > 0)[-1])))
        lengths.append(len(path))
        paths.append(path + [-1] * (s["most"] - len(path)))
    return [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (paths, lengths, nexts)]
