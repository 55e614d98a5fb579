"""Verification of draft trees on the GPU against the rule stated in 64 bits; whole numbers have to be equal."""
import math

import numpy as np
import pytest
import torch

import kv_util as ref

pytestmark = pytest.mark.gpu


def _run(target, draft, tokens, trees, accept, sample, most):
    from paper_2607_04031_b200 import binding as tl
    dev = "cuda:0"
    counts = [len(t) for t in trees]
    offs = torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(dev)
    parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device=dev)
    accepted = torch.full((len(trees), most), 99, dtype=torch.int32, device=dev)
    n, nxt = (torch.full((len(trees),), 99, dtype=torch.int32, device=dev) for _ in range(2))
    move = lambda x: None if x is None else x.to(dev)  # noqa: E731
    tl.tree_verify(move(target), move(draft), torch.as_tensor(tokens, dtype=torch.int32).to(dev), parents, offs,
                   torch.as_tensor(accept).to(dev), torch.as_tensor(sample).to(dev), accepted, n, nxt)
    tl.device_status()
    return accepted.cpu().numpy(), n.cpu().numpy(), nxt.cpu().numpy()


def _check(target, draft, tokens, trees, accept, sample, most):
    got = _run(target, draft, tokens, trees, accept, sample, most)
    at = 0
    for b, t in enumerate(trees):
        m = len(t)
        if m == 0:
            want_path, want_next = [], -1
        else:
            want_path, want_next = ref.verify(target[at:at + m].numpy(), None if draft is None else draft[at:at + m].numpy(),
                                              list(tokens[at:at + m]), t, accept[at:at + m], sample[b], most)
        assert got[0][b].tolist() == want_path + [-1] * (most - len(want_path)), b
        assert got[1][b] == len(want_path) and got[2][b] == want_next, (b, got[2][b], want_next)
        at += m
    return got


def _case(counts, branch, vocab, drafts, seed, near=0.6):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    trees = [ref.random_tree(n, branch, rng) if n else [] for n in counts]
    N = sum(counts)
    z = torch.randn(N, vocab, generator=g) * 2
    p, q = torch.softmax(z, -1), torch.softmax(z + near * torch.randn(N, vocab, generator=g), -1)
    tokens, at = [], 0
    for t in trees:
        seen = {}
        for i, par in enumerate(t):
            row = at + max(par, 0)
            k = seen[par] = seen.get(par, -1) + 1
            tokens.append(int(torch.multinomial(q[row], 1, generator=g)) if drafts else int(q[row].topk(k + 1).indices[k]) if k < vocab else 0)
        at += len(t)
    return p, q if drafts else None, tokens, trees, rng.random(N, dtype=np.float32), rng.random(len(counts), dtype=np.float32)


@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("counts,branch", [([1], 1), ([5], 1), ([6, 0, 1, 9], 1), ([24, 1, 16, 30], 4), ([64] * 3, 8), ([17] * 40, 3)])
@pytest.mark.parametrize("vocab", [1, 33, 1000, 4099, 32768, 100003])
def test_matches_the_rule(drafts, counts, branch, vocab):
    if sum(counts) * vocab > 3e7:
        counts = counts[:2]
    _check(*_case(counts, branch, vocab, drafts, seed=vocab + len(counts) + branch), most=max(max(counts), 1))


@pytest.mark.parametrize("drafts", [True, False])
def test_many_requests_use_fewer_ctas_each(drafts):
    for n in (30, 100, 400):
        _check(*_case([4] * n, 2, 5000, drafts, seed=n), most=4)


def test_trees_wider_and_longer_than_what_is_kept_on_chip():
    # 1500 nodes: rows past the first 1024 are looked up in memory; a chain deep, then a star
    vocab, n = 64, 1500
    rng = np.random.default_rng(0)
    chain = [-1] + list(range(n - 1))
    star = [-1] + [0] * 400
    p = torch.full((n + 401, vocab), 1.0 / vocab)
    q = p.clone()
    tokens = rng.integers(0, vocab, n + 401).tolist()
    accept = np.full(n + 401, 0.5, dtype=np.float32)        # p == q: every child is kept
    got = _check(p, q, tokens, [chain, star], accept, np.array([0.3, 0.9], dtype=np.float32), most=n)
    assert got[1].tolist() == [n, 2]
    # without a draft distribution most children of the star are refused
    accept[:] = 0.999
    _check(p[:401], None, tokens[:401], [star], accept[:401], np.array([0.5], dtype=np.float32), most=8)


def test_a_path_ends_where_the_answer_is_full():
    p = torch.full((6, 50), 0.02)
    got = _check(p, p.clone(), [1] * 6, [[-1, 0, 1, 2, 3, 4]], np.zeros(6, dtype=np.float32), np.array([0.5], dtype=np.float32), most=3)
    assert got[1].tolist() == [3]


def test_edges_of_the_distributions():
    vocab = 300
    # all mass on one id; a residual that is empty (p == q and a draft of zero probability); zeros everywhere; NaN and
    # negative entries; ids outside the vocabulary; the largest random number below 1
    one = torch.zeros(vocab); one[17] = 1.0                                           # noqa: E702
    flat = torch.full((vocab,), 1.0 / vocab)
    holes = flat.clone(); holes[::2] = 0                                              # noqa: E702
    dirty = flat.clone(); dirty[3] = math.nan; dirty[4] = -1.0                        # noqa: E702
    zero = torch.zeros(vocab)
    top = np.float32(1 - 2.0 ** -24)
    for p, q, tok in ((one, flat, 17), (one, flat, 16), (one, one, 16), (flat, flat, 5), (holes, holes, 2), (holes, flat, 2), (dirty, flat, 3),
                      (dirty, dirty, 4), (zero, flat, 1), (flat, zero, 1), (flat, flat, -1), (flat, flat, vocab), (flat, flat, 2 ** 31 - 1)):
        target, draft = torch.stack([p] * 3), torch.stack([q] * 3)
        for u in (0.0, 0.5, top):
            for d in (draft, None):
                _check(target, d, [0, tok, tok], [[-1, 0, 0]], np.array([0, u, u], dtype=np.float32), np.array([u], dtype=np.float32), most=3)


def test_strided_rows():
    from paper_2607_04031_b200 import binding as tl
    p, q, tokens, trees, accept, sample = _case([9, 4], 2, 1001, True, seed=2)
    wide = torch.zeros(13, 1111, device="cuda")
    wide[:, 5:1006] = p.cuda()
    other = torch.zeros(13, 1500, device="cuda")
    other[:, 1:1002] = q.cuda()
    offs = torch.tensor([0, 9, 13], dtype=torch.int32, device="cuda")
    parents = torch.tensor([x for t in trees for x in t], dtype=torch.int32, device="cuda")
    acc, n, nxt = torch.empty(2, 9, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    tl.tree_verify(wide[:, 5:1006], other[:, 1:1002], torch.tensor(tokens, dtype=torch.int32, device="cuda"), parents, offs,
                   torch.tensor(accept).cuda(), torch.tensor(sample).cuda(), acc, n, nxt)
    want = _run(p, q, tokens, trees, accept, sample, 9)
    assert np.array_equal(acc.cpu().numpy(), want[0]) and np.array_equal(n.cpu().numpy(), want[1]) and np.array_equal(nxt.cpu().numpy(), want[2])


@pytest.mark.parametrize("drafts", [True, False])
def test_the_next_token_has_the_targets_distribution(drafts):
    # One root with three alternatives, 60000 requests: the token after the root (the kept child's, else the drawn one)
    # has frequency p, to five standard deviations of a binomial.
    from paper_2607_04031_b200 import binding as tl
    B, vocab = 60000, 12
    g = torch.Generator(device="cuda").manual_seed(3)
    p = torch.softmax(torch.randn(vocab, generator=g, device="cuda"), 0)
    q = torch.softmax(torch.randn(vocab, generator=g, device="cuda"), 0)
    toks = torch.zeros(B, 4, dtype=torch.int32, device="cuda")
    if drafts:
        toks[:, 1:] = torch.multinomial(q.expand(B, vocab), 3, replacement=True, generator=g).int()
    else:
        toks[:, 1:] = q.topk(3).indices.int()
    parents = torch.tensor([-1, 0, 0, 0], dtype=torch.int32, device="cuda").repeat(B)
    offs = torch.arange(B + 1, dtype=torch.int32, device="cuda") * 4
    acc, n, nxt = torch.empty(B, 4, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    rows = p.expand(4 * B, vocab).contiguous()
    tl.tree_verify(rows, q.expand(4 * B, vocab).contiguous() if drafts else None, toks.view(-1), parents, offs,
                   torch.rand(4 * B, generator=g, device="cuda"), torch.rand(B, generator=g, device="cuda"), acc, n, nxt)
    first = torch.where(n > 1, toks.gather(1, acc[:, 1:2].clamp_min(0).long())[:, 0], nxt)
    freq = torch.bincount(first.long(), minlength=vocab).double() / B
    sd = (p.double() * (1 - p.double()) / B).sqrt()
    assert bool(((freq - p.double()).abs() <= 5 * sd).all())
