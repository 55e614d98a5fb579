"""The decoding loop with rotary positions, a 4-bit cache and pages from a common pool: against 64-bit attention over what the cache
holds, and against itself with drafts and without, with pages of its own and from the pool."""
import math

import pytest
import torch

import kv_util
import serve_util

pytestmark = pytest.mark.gpu
PROMPTS = [[3, 1, 4, 1, 5], list(range(40)), [7] * 33]


def _decoder(**kw):
    from paper_2607_04031_b200.drafted import Decoder
    return Decoder(**{**dict(requests=3, cache="e2m1", temperature=1.0, rotary=10000.0, page_tokens=16, room=256), **kw})


def _rows(d, b, n):
    """fp64 keys and values of request b's first n positions, from the pool's bits."""
    k, v, ks, vs, kg, vg = (t.cpu() for t in d.cache._tensors)
    pg, line = d.page_table[b].cpu().long()[torch.arange(n) // 16], torch.arange(n) % 16
    return [serve_util.held4(c[pg, :, line], g.view(torch.uint8)[pg, :, line], s[pg, :, line]) for c, g, s in ((k, kg, ks), (v, vg, vs))]


@pytest.mark.parametrize("pool", [None, 60])
def test_every_row_attends_over_what_its_branch_holds(pool):
    from paper_2607_04031_b200 import binding as tl
    d = _decoder(pool_pages=pool)
    d.prefill(PROMPTS)
    for _ in range(3):
        s = d.step(3, 3)
        tl.device_status()
        start, offs, parents = s.start.tolist(), s.token_offsets.tolist(), s.parents.tolist()
        # the pool still holds the step's rows, behind those that were kept where these lie further on: look at kept paths
        for b in range(3):
            n, first = int(s.n_accepted[b]), offs[b]
            path = s.accepted[b, :n].tolist()
            k, v = _rows(d, b, start[b] + n)
            rows = torch.tensor([first + i for i in path])
            want, _, mass, big = kv_util.attention(s.q[rows.cuda()].cpu(), k, v, start[b], torch.ones(n, n, dtype=torch.bool).tril(), 128 ** -0.5)
            bound = kv_util.attention_bound(want, mass, big, v, "e2m1", 128, 128 ** -0.5, start[b] + n)
            assert bool(((s.out[rows.cuda()].double().cpu() - want).abs() <= bound).all())
            assert all(parents[first + i] == (path[j - 1] if j else -1) for j, i in enumerate(path))


def test_queries_are_turned_by_their_depth():
    from paper_2607_04031_b200 import binding as tl
    d, plain = _decoder(), _decoder(rotary=None)
    d.prefill(PROMPTS), plain.prefill(PROMPTS)
    tokens, draft, parents = d._draft(2, 3)
    flat, up = tokens.flatten().to(torch.int32), torch.tensor(parents * 3, dtype=torch.int32, device="cuda:0")
    offsets = d._offsets([tokens.shape[1]] * 3)
    a, b = d.forward(flat, up, offsets, True, tokens.shape[1]), plain.forward(flat, up, offsets, True, tokens.shape[1])
    tl.device_status()
    depth = []
    for p in parents:
        depth.append(0 if p < 0 else depth[p] + 1)
    pos = torch.tensor([int(s) + x for s in d.start for x in depth])
    want, size = serve_util.turned(b.q.cpu(), tl.rope_turns(128), pos, 0)
    assert bool(((a.q.double().cpu() - want).abs() <= serve_util.turned_bound(want, size, 1.0, torch.bfloat16)).all())


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "e2m1"])
def test_pages_from_a_pool_change_no_token(cache):
    own, pool = _decoder(cache=cache), _decoder(cache=cache, pool_pages=40)
    pool.generator.set_state(own.generator.get_state())      # (the pages of its own were drawn from it)
    a, passes_a = own.generate(PROMPTS, 24, 3, 4)
    b, passes_b = pool.generate(PROMPTS, 24, 3, 4)
    assert a == b and passes_a == passes_b
    in_use = int((pool.tables._tensors[2] > 0).sum())
    assert in_use == sum(-(-n // 16) for n in pool.start.tolist())
    # moved together, they go on as before
    assert pool.compact() == in_use and bool((pool.tables._tensors[2][:in_use] > 0).all())
    for _ in range(3):
        x, y = own.step(3, 4), pool.step(3, 4)
        assert torch.equal(x.logits.view(torch.int32), y.logits.view(torch.int32)) and torch.equal(x.next_token, y.next_token)


def test_continuations_of_a_prompt_share_its_pages_and_go_their_own_ways():
    from paper_2607_04031_b200 import binding as tl
    samples = 4
    d = _decoder(requests=3 * samples, pool_pages=120)
    d.prefill([p if j == 0 else None for p in PROMPTS for j in range(samples)])
    before = int((d.tables._tensors[2] > 0).sum())
    d.fork(samples)
    tl.device_status()
    assert int((d.tables._tensors[2] > 0).sum()) == before
    s = d.step(2, 3)
    # all continuations see one prompt: the roots' logits are the same bits (their rows are of one shape and their pages hold one content)
    roots = s.logits[s.token_offsets[:-1].long()]
    for i in range(3):
        for j in range(1, samples):
            assert torch.equal(roots[i * samples].view(torch.int32), roots[i * samples + j].view(torch.int32))
    for _ in range(4):
        d.step(2, 3)
    tl.device_status()
    holders, held, table = (t.cpu() for t in (d.tables._tensors[2], d.tables._tensors[1], d.page_table))
    count = torch.zeros_like(holders)
    for b in range(3 * samples):
        for p in table[b, :int(held[b])].tolist():
            count[p] += 1
    assert torch.equal(count, holders)
    assert held.tolist() == [-(-n // 16) for n in d.start.tolist()]
    # what lies behind the prompts' whole pages is everybody's own
    whole = [(len(PROMPTS[b // samples]) - 1) // 16 for b in range(3 * samples)]
    for b in range(3 * samples):
        assert all(int(holders[p]) == samples for p in table[b, :whole[b]].tolist())
        assert all(int(holders[p]) == 1 for p in table[b, whole[b]:int(held[b])].tolist())


def test_a_pool_that_is_too_small_says_so():
    d = _decoder(pool_pages=5)
    with pytest.raises(RuntimeError, match="too few"):
        d.generate(PROMPTS, 24, 3, 4)


def test_drafts_change_no_likeliest_token():
    """Temperature 0: drafted decoding gives the tokens of decoding one by one, up to where two are as likely within rounding."""
    one, plain, lead = _decoder(temperature=0.0, requests=2), [], []
    one.prefill(PROMPTS[:2])
    for _ in range(8):
        s = one.step(0, 0)
        top = s.logits.topk(2, -1).values
        plain.append(s.next_token.clone())
        lead.append(top[:, 0] - top[:, 1])
    tree, passes = _decoder(temperature=0.0, requests=2, pool_pages=30).generate(PROMPTS[:2], 8, 3, 4)
    assert passes <= 8
    for a, b, by in zip(torch.stack(plain, 1).tolist(), tree, torch.stack(lead, 1).tolist()):
        at = next((i for i in range(8) if a[i] != b[i]), 8)
        assert at == 8 or by[at] <= 0.1
