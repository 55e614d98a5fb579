"""The decoding loop with drafted trees, stage by stage: every stage of every step against the plain form in 64 bits of what
that stage was given, and the cache at the end against the rows of the tokens that were kept."""
import os
import subprocess
import sys

import pytest
import torch

from tests import kv_util as ref

pytestmark = pytest.mark.gpu


def held_rows(d):
    """The whole cache in fp32, [requests, room, heads, dim], keys and values."""
    from paper_2607_04031_b200 import binding as tl
    room = d.page_table.shape[1] * d.cache.page_tokens
    rows = d.requests * room
    offsets = torch.arange(0, rows + 1, room, dtype=torch.int32, device=d.device)
    batch = tl.kv_batch(d.page_table, torch.zeros_like(d.start), offsets, rows)
    k, v = (torch.empty(rows, d.heads, d.head_dim, device=d.device) for _ in range(2))
    tl.kv_read(d.cache, batch, k, v)
    tl.device_status()
    return [t.cpu().view(d.requests, room, d.heads, d.head_dim) for t in (k, v)]


def rows_of(s, b):
    return slice(int(s.token_offsets[b]), int(s.token_offsets[b + 1]))


def check_attention(d, fmt, s, held, parents):
    for b in range(d.requests):
        at, ctx = rows_of(s, b), int(s.start[b])
        n = at.stop - at.start
        if n == 0:
            continue
        k, v = (h[b, :ctx + n].double() for h in held)
        if s.mask is None:
            sees = torch.ones(n, n, dtype=torch.bool).tril()
        else:
            sees = torch.eye(n, dtype=torch.bool)
            for i, p in enumerate(parents):
                if p >= 0:
                    sees[i] |= sees[p]
        out = s.out[at].double().cpu()
        want, _, mass, big = ref.attention(s.q[at].cpu(), k, v, ctx, sees, d.head_dim ** -0.5)
        bound = ref.attention_bound(want, mass, big, v, fmt, d.head_dim, d.head_dim ** -0.5, ctx + n)
        assert bool(((out - want).abs() <= bound).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
@pytest.mark.parametrize("branches,depth", [(0, 0), (1, 3), (3, 4), (8, 5)])
def test_every_stage_of_every_step(fmt, temperature, branches, depth):
    from paper_2607_04031_b200 import binding as tl
    from paper_2607_04031_b200.drafted import Decoder
    d = Decoder(3, fmt, temperature=temperature, room=256, vocab=512, seed=branches + depth)
    prompts = [[(7 * i + b) % 512 for i in range(n)] for b, n in enumerate((1, 20, 70))]
    kept = [[] for _ in prompts]                              # (keys, values) of every token that should be cached
    s = d.prefill(prompts)
    check_attention(d, fmt, s, held_rows(d), None)
    for b in range(3):
        kept[b] += list(zip(s.k[rows_of(s, b)].cpu(), s.v[rows_of(s, b)].cpu()))
    assert d.start.tolist() == [0, 19, 69]
    most = 0
    for _ in range(6):
        before, root = d.start.clone(), d.last.clone()
        # the step in two halves, so that the cache can be looked at before rows are moved
        commit = tl.kv_commit
        seen = []
        tl.kv_commit = lambda *a, **kw: (seen.append(held_rows(d)), commit(*a, **kw))[1]
        try:
            s = d.step(branches, depth)
        finally:
            tl.kv_commit = commit
        tl.device_status()
        assert torch.equal(s.start, before)
        n = 1 + branches * depth
        parents = s.parents[:n].tolist()
        check_attention(d, fmt, s, seen[0], parents)
        for b in range(3):
            at = rows_of(s, b)
            assert int(s.tokens[at.start]) == int(root[b])
            path, nxt = ref.verify(s.target[at].double().cpu().numpy(), None if s.draft is None else s.draft[at].double().cpu().numpy(),
                                   s.tokens[at].tolist(), parents, s.accept[at].double().cpu().numpy(), float(s.sample[b]), n)
            got = s.accepted[b][:int(s.n_accepted[b])].tolist()
            assert got == path and int(s.next_token[b]) == nxt
            kept[b] += [(s.k[at][i].cpu(), s.v[at][i].cpu()) for i in path]
            most = max(most, len(path))
        assert d.start.tolist() == [len(x) for x in kept]
    for held, which in zip(held_rows(d), (0, 1)):
        for b in range(3):
            rows = torch.stack([x[which] for x in kept[b]])
            want = rows.float() if fmt == "bf16" else ref.held(*ref.quantise(rows, fmt)).float()
            assert torch.equal(held[b, :len(kept[b])], want)
    assert branches == 0 or most > 1, "no draft was kept: nothing was moved"


def test_the_command():
    run = subprocess.run([sys.executable, "-m", "paper_2607_04031_b200.drafted", "--tokens", "24"], capture_output=True, text=True, timeout=300,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert run.returncode == 0, run.stderr
    lines = run.stdout.strip().splitlines()
    assert len(lines) == 2 and "in 24 passes" in lines[0]
