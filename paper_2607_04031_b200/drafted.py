"""Decoding with drafted trees: one attention layer, run through the library as a serving loop would run it.

    python -m paper_2607_04031_b200.drafted [--cache bf16|e4m3|int8|e2m1] [--branches 3] [--depth 4] [--temperature 1.0]
                                            [--rotary] [--samples 1]

Every step drafts a tree of tokens per request (`branches` children of the last certain token, each carried on as a chain
of `depth` tokens), and one pass checks all of them: tl_gemm_bf16 (queries, keys and values in one product, on tile-major
weights), tl_kv_append, tl_tree_mask and tl_tree_attention, tl_gemm_bf16 and tl_gemm for the output and the vocabulary,
tl_tree_verify, tl_kv_commit.  With rotary positions tl_tree_positions and tl_rope_append stand in the place of tl_kv_append.  Pages
can be the requests' own from the start, or taken from a common pool as sequences grow (tl_page_reserve) and given back where drafts
are dropped (tl_page_release); then several continuations of a prompt share its pages (tl_page_fork) until they write them, and the pages
in use can be moved together (tl_page_compact, tl_page_copy).  The draft comes from the same layer without its attention.  Weights are
random: the loop shows the calls and their order, not a language model.
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass

import torch

from . import binding as tl
from . import inputs

CACHES = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8, "e2m1": torch.uint8}


@dataclass
class Step:
    """What one step computed (tensors on the device)."""
    tokens: torch.Tensor         # int32 [rows]
    parents: torch.Tensor        # int32 [rows]
    token_offsets: torch.Tensor  # int32 [requests + 1]
    start: torch.Tensor          # int32 [requests]: cached positions before the step
    mask: torch.Tensor | None
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    out: torch.Tensor
    logits: torch.Tensor
    target: torch.Tensor | None = None
    draft: torch.Tensor | None = None
    accept: torch.Tensor | None = None
    sample: torch.Tensor | None = None
    accepted: torch.Tensor | None = None
    n_accepted: torch.Tensor | None = None
    next_token: torch.Tensor | None = None


class Decoder:
    def __init__(self, requests: int, cache: str = "bf16", vocab: int = 1024, hidden: int = 512, q_heads: int = 8, heads: int = 2,
                 head_dim: int = 128, page_tokens: int = 32, room: int = 1024, temperature: float = 1.0, seed: int = 0,
                 device: str = "cuda:0", rotary: float | None = None, pool_pages: int | None = None):
        """rotary: base of the rotary positions, half layout (None: no positions).  pool_pages: pages that all requests take from and
        give back to (None: every request owns room / page_tokens pages)."""
        self.requests, self.vocab, self.hidden, self.temperature, self.device = requests, vocab, hidden, temperature, device
        self.q_heads, self.heads, self.head_dim = q_heads, heads, head_dim
        self.wide_q, self.wide_kv = q_heads * head_dim, heads * head_dim
        self.embedding = inputs.bf16_normal((vocab, hidden), 1.0, seed).to(device)
        self.w_qkv = self._tile_major(inputs.bf16_normal((hidden, self.wide_q + 2 * self.wide_kv), hidden ** -0.5, seed + 1))
        self.w_o = self._tile_major(inputs.bf16_normal((self.wide_q, hidden), self.wide_q ** -0.5, seed + 2))
        self.w_vocab = self._tile_major(inputs.bf16_normal((hidden, vocab), 2.0 * hidden ** -0.5, seed + 3))
        pages = -(-room // page_tokens)
        pool, scales = (pool_pages or requests * pages, heads, page_tokens, head_dim // 2 if cache == "e2m1" else head_dim), None
        if cache != "bf16":
            scales = [torch.zeros(pool[:3], device=device) for _ in range(2)]
        if cache == "e2m1":
            scales += [torch.zeros(*pool[:3], head_dim // 16, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)]
        self.pool = [torch.zeros(pool, dtype=torch.uint8 if cache != "bf16" else torch.bfloat16, device=device).view(CACHES[cache])
                     for _ in range(2)]
        self.cache = tl.kv_cache(*self.pool, *(scales or ()))
        # pages as they would be after some traffic: a request's are not neighbours
        self.generator = torch.Generator(device=device).manual_seed(seed)
        self.tables = None
        if pool_pages is None:
            self.page_table = torch.randperm(requests * pages, generator=self.generator, device=device).to(torch.int32).view(requests, pages)
        else:
            counts = lambda n: torch.zeros(n, dtype=torch.int32, device=device)  # noqa: E731
            self.page_table = torch.full((requests, pages), -1, dtype=torch.int32, device=device)
            self.held = counts(requests)
            self.tables = tl.page_tables(self.page_table, self.held, counts(pool_pages), page_tokens)
            self.moves, self.n_moves, self.missing = torch.zeros(max(requests, pool_pages), 3, dtype=torch.int32, device=device), counts(1), counts(1)
        self.rope = None
        if rotary is not None:
            self.rope = tl.rope(tl.rope_turns(head_dim, rotary).to(device))
        self.start = torch.zeros(requests, dtype=torch.int32, device=device)
        self.last = None                                     # int64 [requests]: the last certain token, not cached yet

    def _tile_major(self, w: torch.Tensor) -> torch.Tensor:
        w = w.to(self.device)
        out = torch.empty_like(w)
        tl.relayout(w, out, w.shape[0], w.shape[1], 2, inputs.DEFAULT_G, *inputs.DEFAULT_BLOCK, tl.TO_TILE_MAJOR)
        return out

    def _product(self, x: torch.Tensor, w: torch.Tensor, dtype=torch.bfloat16) -> torch.Tensor:
        y = torch.empty(x.shape[0], w.shape[1], dtype=dtype, device=self.device)
        (tl.gemm_bf16 if dtype is torch.bfloat16 else tl.gemm)(x, w, y, x.shape[0], w.shape[1], w.shape[0])
        return y

    def _probabilities(self, logits: torch.Tensor) -> torch.Tensor:
        if self.temperature == 0:
            return torch.nn.functional.one_hot(logits.argmax(-1), self.vocab).float()
        return torch.softmax(logits / self.temperature, -1)

    def _offsets(self, counts) -> torch.Tensor:
        return torch.tensor([0, *counts], dtype=torch.int32).cumsum(0).to(torch.int32).to(self.device)

    def forward(self, tokens: torch.Tensor, parents: torch.Tensor, offsets: torch.Tensor, tree: bool, most: int) -> Step:
        """tokens: int32 [rows]; most: the most rows of a request.  Their keys and values are in the cache afterwards."""
        rows = tokens.shape[0]
        x = self.embedding[tokens.long()]
        qkv = self._product(x, self.w_qkv)
        q = qkv[:, :self.wide_q].view(rows, self.q_heads, self.head_dim)
        k = qkv[:, self.wide_q:self.wide_q + self.wide_kv].view(rows, self.heads, self.head_dim)
        v = qkv[:, self.wide_q + self.wide_kv:].view(rows, self.heads, self.head_dim)
        if self.tables is not None:
            self._reserve(self.start + offsets[1:] - offsets[:-1])
        batch = tl.kv_batch(self.page_table, self.start, offsets, rows)
        if self.rope is None:
            tl.kv_append(self.cache, batch, k, v)
        else:
            positions = None
            if tree:
                positions = torch.empty(rows, dtype=torch.int32, device=self.device)
                tl.tree_positions(parents, offsets, self.start, positions)
            tl.rope_append(self.cache, batch, self.rope, q, q, k, v, positions=positions)
        mask = None
        if tree:
            mask = torch.empty(rows, -(-most // 32), dtype=torch.int32, device=self.device)
            tl.tree_mask(parents, offsets, mask)
        out = torch.empty(rows, self.q_heads, self.head_dim, dtype=torch.bfloat16, device=self.device)
        tl.tree_attention(self.cache, batch, q, out, mask=mask)
        h = x + self._product(out.view(rows, self.wide_q), self.w_o)
        return Step(tokens, parents, offsets, self.start.clone(), mask, q, k, v, out, self._product(h, self.w_vocab, torch.float32))

    def _reserve(self, lengths: torch.Tensor):
        """Pages of its own for the positions that every request is about to write; raises where the pool has too few."""
        tl.page_reserve(self.tables, self.start, lengths, self.moves, self.n_moves, self.missing)
        tl.page_copy(self.cache, self.moves, self.n_moves)
        if self.missing.item():
            raise RuntimeError(f"the pool has {self.missing.item()} pages too few")

    def _continuations(self, samples: int) -> torch.Tensor:
        """The requests that fork(samples) makes continuations of; raises where they cannot be."""
        if samples < 1:
            raise ValueError(f"samples: expected 1 or more, got {samples}")
        to = torch.tensor([r for r in range(self.requests) if r % samples], dtype=torch.int32, device=self.device)
        if to.numel():
            if self.tables is None:
                raise ValueError("continuations share pages: the decoder needs a pool (pool_pages)")
            if bool((self.held[to.long()] != 0).any()):
                raise ValueError("a request that holds pages cannot become another's continuation")
        return to

    def fork(self, samples: int):
        """Request i * samples + j (j > 0), which must hold nothing, continues what request i * samples has so far, on the same pages
        until it writes them."""
        to = self._continuations(samples)
        if to.numel() == 0:
            return
        if self.last is None:
            raise ValueError("nothing to continue: prefill comes first")
        from_ = to // samples * samples
        self.start[to.long()] = self.start[from_.long()]
        self.last[to.long()] = self.last[from_.long()]
        tl.page_fork(self.tables, from_, to, self.start[from_.long()].contiguous())

    def compact(self) -> int:
        """Moves the pages in use to the front of the pool and says how many they are."""
        if self.tables is None:
            raise ValueError("only a decoder with a pool (pool_pages) moves pages")
        tl.page_compact(self.tables, self.moves, self.n_moves, self.missing)
        tl.page_copy(self.cache, self.moves, self.n_moves)
        return int(self.missing.item())

    def prefill(self, prompts) -> Step | None:
        """prompts: one list of token ids per request, none empty (a request without one, None, is left for a fork).  All but their last
        tokens go through the layer."""
        if len(prompts) != self.requests:
            raise ValueError(f"expected {self.requests} prompts, one per request, got {len(prompts)}")
        self.last = torch.tensor([p[-1] if p else 0 for p in prompts], device=self.device)
        counts = [len(p) - 1 if p else 0 for p in prompts]
        prompts = [p or [0] for p in prompts]
        if sum(counts) == 0:
            return None
        tokens = torch.tensor([t for p in prompts for t in p[:-1]], dtype=torch.int32, device=self.device)
        offsets = self._offsets(counts)
        step = self.forward(tokens, tokens, offsets, False, max(counts))
        self.start += offsets[1:] - offsets[:-1]
        return step

    def _draft(self, branches: int, depth: int):
        """Trees in the order root, first children, their children, ...: tokens and distributions, [requests, rows]."""
        def distribution(tokens):
            flat = self._product(self.embedding[tokens.flatten()], self.w_vocab, torch.float32)
            return self._probabilities(flat).view(*tokens.shape, self.vocab), flat.view(*tokens.shape, self.vocab)

        tokens = [self.last.view(-1, 1)]
        rows = []
        for level in range(depth if branches else 0):
            p, logits = distribution(tokens[-1])
            rows.append(p)
            width = branches if level == 0 else 1
            if self.temperature == 0:
                new = logits.topk(width, -1).indices
            else:
                new = torch.multinomial(p.flatten(0, 1), width, True, generator=self.generator).view(*p.shape[:2], width)
            tokens.append(new.flatten(1))
        rows.append(distribution(tokens[-1])[0] if len(tokens) > 1 else torch.zeros(self.requests, 1, self.vocab, device=self.device))
        parents = [-1] + [0 if level == 0 else 1 + (level - 1) * branches + i for level in range(len(tokens) - 1) for i in range(branches)]
        return torch.cat(tokens, 1), torch.cat(rows, 1), parents

    def step(self, branches: int, depth: int) -> Step:
        """One pass over a drafted tree per request; the kept tokens' rows stay in the cache."""
        tokens, draft, parents = self._draft(branches, depth)
        n = tokens.shape[1]
        flat = tokens.flatten().to(torch.int32)
        up = torch.tensor(parents * self.requests, dtype=torch.int32, device=self.device)
        offsets = self._offsets([n] * self.requests)
        s = self.forward(flat, up, offsets, True, n)
        s.target = self._probabilities(s.logits)
        # at temperature 0 the children are the likeliest ones, not drawn
        s.draft = None if self.temperature == 0 else draft.flatten(0, 1).contiguous()
        s.accept = torch.rand(flat.shape[0], generator=self.generator, device=self.device)
        s.sample = torch.rand(self.requests, generator=self.generator, device=self.device)
        s.accepted = torch.empty(self.requests, n, dtype=torch.int32, device=self.device)
        s.n_accepted = torch.empty(self.requests, dtype=torch.int32, device=self.device)
        s.next_token = torch.empty_like(s.n_accepted)
        tl.tree_verify(s.target, s.draft, flat, up, offsets, s.accept, s.sample, s.accepted, s.n_accepted, s.next_token)
        batch = tl.kv_batch(self.page_table, self.start, offsets, flat.shape[0])
        tl.kv_commit(self.cache, batch, s.accepted, s.n_accepted, self.start)
        if self.tables is not None:
            tl.page_release(self.tables, self.start)             # what only dropped drafts needed
        self.last = s.next_token.long()
        return s

    def generate(self, prompts, new_tokens: int, branches: int = 3, depth: int = 4, samples: int = 1):
        """Lists of new token ids, `new_tokens` per request, and the number of passes that gave them.  samples: continuations of each
        prompt, neighbours among the requests (there are len(prompts) * samples)."""
        self._continuations(samples)                         # (what stands against them is said before anything has changed)
        self.prefill([p if j == 0 else None for p in prompts for j in range(samples)])
        if samples > 1:
            self.fork(samples)
        made, passes = [[] for _ in range(self.requests)], 0
        while min(map(len, made)) < new_tokens:
            s = self.step(branches, depth)
            passes += 1
            tokens = s.tokens.view(self.requests, -1).cpu()
            for b, (path, n, nxt) in enumerate(zip(s.accepted.cpu(), s.n_accepted.tolist(), s.next_token.tolist())):
                made[b] += tokens[b][path[1:n].long()].tolist() + [nxt]
        tl.device_status()
        return [m[:new_tokens] for m in made], passes


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--cache", choices=CACHES, default="e4m3")
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--branches", type=int, default=3)
    ap.add_argument("--depth", type=int, default=4)
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--rotary", action="store_true", help="rotary positions, base 10000")
    ap.add_argument("--samples", type=int, default=1, help="continuations of each prompt, sharing its pages")
    a = ap.parse_args()
    prompts = [[(17 * b + 5 * i) % 1024 for i in range(20 + 13 * b)] for b in range(a.requests)]
    for branches, depth in ((0, 0), (a.branches, a.depth)):
        # a request may run ahead of the slowest by a whole tree per pass
        room = max(map(len, prompts)) + (a.tokens + 1) * (1 + depth) + branches * depth + 1
        requests = a.requests * a.samples
        pool = requests * -(-room // 32) if a.samples > 1 else None
        d = Decoder(requests, a.cache, temperature=a.temperature, room=room, rotary=10000.0 if a.rotary else None, pool_pages=pool)
        made, passes = d.generate(prompts, a.tokens, branches, depth, a.samples)
        pages = f", {d.compact()} pages in use" if pool else ""
        print(f"{branches} branches of {depth}: {a.tokens} tokens for {requests} requests in {passes} passes{pages}; the first: {made[0][:8]}")


if __name__ == "__main__":
    main()
