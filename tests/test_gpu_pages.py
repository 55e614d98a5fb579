"""Page bookkeeping on the GPU against tables worked on entry by entry; copies bit by bit."""
import random

import pytest
import torch

import kv_util
import serve_util as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Both:
    """Tables on the GPU and the plain ones beside them."""

    def __init__(self, requests, width, pages, page=16):
        from paper_2607_04031_b200 import binding as tl
        self.tl, self.plain = tl, ref.Tables(requests, width, pages, page)
        self.table, self.held, self.holders = i32(self.plain.table).view(requests, width), i32(self.plain.held), i32(self.plain.holders)
        self.t = tl.page_tables(self.table, self.held, self.holders, page)
        self.moves = torch.full((max(requests, pages, 1), 3), -9, dtype=torch.int32, device=DEV)
        self.n, self.m = i32([-9]), i32([-9])

    def same(self):
        assert self.held.tolist() == self.plain.held
        assert self.holders.tolist() == self.plain.holders
        assert self.table.tolist() == self.plain.table

    def moved(self, want):
        assert self.n.item() == len(want)
        assert self.moves[:len(want)].tolist() == [list(m) for m in want]
        assert bool((self.moves[len(want):] == -9).all())
        self.moves.fill_(-9)

    def reserve(self, start, tokens):
        self.tl.page_reserve(self.t, i32(start), i32(tokens), self.moves, self.n, self.m)
        moves, missing = self.plain.reserve(start, tokens)
        assert self.m.item() == missing
        self.moved(moves)
        self.same()
        return missing

    def release(self, tokens=None):
        self.tl.page_release(self.t, None if tokens is None else i32(tokens))
        self.plain.release(tokens)
        self.same()

    def fork(self, from_, to, tokens):
        self.tl.page_fork(self.t, i32(from_), i32(to), i32(tokens))
        out = self.plain.fork(from_, to, tokens)
        self.same()
        return out

    def compact(self, most=None):
        rows = self.moves if most is None else self.moves[:most]
        self.tl.page_compact(self.t, rows, self.n, self.m)
        moves, in_use = self.plain.compact(rows.shape[0])
        assert self.m.item() == in_use
        self.moved(moves)
        self.same()


def test_a_first_reservation_takes_pages_in_order():
    b = Both(3, 8, 40)
    assert b.reserve([0, 0, 0], [33, -1, 16]) == 0
    assert b.table[0, :3].tolist() == [0, 1, 2] and b.table[2, 0].item() == 3
    b.reserve([33, 0, 16], [34, 1, 17])
    b.tl.device_status()


def test_nothing_changes_without_enough_pages():
    b = Both(2, 8, 6)
    b.reserve([0, 0], [64, 0])
    assert b.reserve([64, 0], [80, 40]) == 2
    assert b.reserve([64, 0], [80, 16]) == 0
    assert b.reserve([80, 16], [81, 17]) == 2
    b.tl.device_status()


def test_positions_past_the_table_are_left_out_and_reported():
    b = Both(2, 3, 20)
    b.reserve([0, 0], [5, 100])
    with pytest.raises(b.tl.TileLensError, match="0xa00"):
        b.tl.device_status()


def test_forks_share_until_one_writes():
    b = Both(5, 8, 40)
    b.reserve([0] * 5, [40, 20, -1, -1, -1])
    assert b.fork([0, 0, 1], [2, 3, 4], [40, 33, 20]) == 0
    # two of three holders write: both leave, the page stays with the third; in request 1 and 4 all holders write: the first keeps it
    b.reserve([-1, 20, 40, 33, 20], [-1, 21, 41, 34, 21])
    b.reserve([40, 21, 41, 34, 21], [60, 30, 60, 60, 60])
    # back into a page that is shared: more than one page is taken over, and the rest of a page is copied
    b.release([35, -1, -1, 20, -1])
    b.reserve([5, 0, 17, 16, 3], [35, 30, 60, 20, 60])
    b.release()
    assert b.holders.sum().item() == 0
    b.tl.device_status()


@pytest.mark.parametrize("from_,to,tokens,out", [([0, 0], [2, 2], [20, 5], 1), ([0, 1], [1, 2], [5, 5], 1), ([0, 5], [5, 2], [5, 5], 2),
                                                 ([-1, 0], [2, -1], [5, 5], 2), ([0, 2], [2, 3], [20, 20], 0), ([3, 0], [2, 3], [20, 20], 0),
                                                 ([2], [2], [5], 0), ([0], [2], [0], 0), ([0], [2], [-3], 0), ([0], [3], [1000], 0)])
def test_forks_that_are_left_out(from_, to, tokens, out):
    b = Both(4, 8, 40)
    b.reserve([0] * 4, [40, 20, -1, -1])
    assert b.fork(from_, to, tokens) == out
    if out:
        with pytest.raises(b.tl.TileLensError, match="0xd00"):
            b.tl.device_status()
    else:
        b.tl.device_status()


@pytest.mark.parametrize("most", [None, 0, 1, 3])
def test_compacting(most):
    b = Both(6, 8, 60)
    b.reserve([0] * 6, [100, 40, 16, 90, 5, -1])
    b.fork([3], [5], [50])
    b.release([-1, 0, 0, -1, -1, -1])
    b.release([20, -1, -1, -1, 0, -1])
    b.compact(most)
    b.compact()
    in_use = b.m.item()
    assert bool((b.holders[:in_use] > 0).all()) and bool((b.holders[in_use:] == 0).all())
    b.compact()                                              # nothing is left to move
    assert b.n.item() == 0
    b.release()
    b.compact()
    assert b.m.item() == 0
    b.tl.device_status()


@pytest.mark.parametrize("requests,width,pages,page,seed", [(1, 1, 1, 16, 0), (3, 4, 7, 16, 1), (17, 20, 200, 32, 2), (64, 12, 500, 16, 3),
                                                            (300, 9, 2500, 64, 4), (1500, 6, 9001, 16, 5), (40, 300, 40007, 16, 6),
                                                            (60, 300, 140003, 16, 7), (9000, 2, 131073, 16, 8)])
def test_long_traffic(requests, width, pages, page, seed):
    """Random reservations, forks, releases and compactions, the tables compared after each."""
    rng = random.Random(seed)
    b = Both(requests, width, pages, page)
    length = [0] * requests
    room = width * page
    for turn in range(30 if pages < 10 ** 5 and requests < 100 else 10):
        kind = rng.choice(["grow", "grow", "back", "fork", "release", "compact"])
        if kind in ("grow", "back"):
            start, tokens = [], []
            for r in range(requests):
                at = length[r] if kind == "grow" else rng.randint(0, length[r])
                n = rng.choice([0, 1, 5, page, 3 * page])
                on = rng.random() < 0.7
                start.append(at if on else rng.choice([-1, at]))
                tokens.append(min(room, at + n) if on else -1)
            if b.reserve(start, tokens) == 0:
                length = [max(n, t) for n, t in zip(length, tokens)]
        elif kind == "fork":
            empty = [r for r in range(requests) if b.plain.held[r] == 0]
            to = rng.sample(empty, min(len(empty), 1 + requests // 3))
            from_ = [rng.randrange(requests) for _ in to]
            tokens = [rng.randint(0, max(1, length[f])) for f in from_]
            if to:
                assert b.fork(from_, to, tokens) == 0
                for f, t, n in zip(from_, to, tokens):
                    length[t] = min(n, b.plain.held[t] * page)
        elif kind == "release":
            keep = [rng.choice([-1, -1, 0, rng.randint(0, length[r])]) for r in range(requests)]
            b.release(keep)
            length = [n if k < 0 else min(n, k) for n, k in zip(length, keep)]
        else:
            b.compact(rng.choice([None, 2]) if pages > 2 else None)
    b.tl.device_status()


@pytest.mark.parametrize("pages", [2 ** 15, 2 ** 15 + 1, 2 ** 16, 2 ** 16 + 1, 2 ** 17, 2 ** 17 + 1, 300000])
def test_the_last_pages_of_a_large_pool(pages):
    """One CTA up to 2^15 (compacting) or 2^16 pages, a cluster beyond: all but the last few pages are held, forks write, and everything moves to the front."""
    b = Both(6, pages, pages)
    room = (pages - 20) * 16
    b.reserve([0] * 6, [room, 30, -1, -1, -1, -1])
    b.fork([1, 1, 0], [2, 3, 4], [30, 20, 35])
    assert b.reserve([-1, 30, 30, 20, 35, -1], [-1, 40, 40, 40, 40, 400]) > 0
    assert b.reserve([-1, 30, 30, 20, 35, -1], [-1, 40, 40, 40, 40, 90]) == 0
    b.release([100, -1, -1, 0, -1, -1])
    b.compact()
    b.tl.device_status()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8", "e2m1"])
@pytest.mark.parametrize("dim,heads,page,permuted", [(64, 3, 16, False), (128, 8, 32, False), (256, 1, 64, True), (128, 2, 1024, False)])
def test_copies(fmt, dim, heads, page, permuted):
    from paper_2607_04031_b200 import binding as tl
    make = lambda pages, seed: (ref.Pool4 if fmt == "e2m1" else kv_util.Pool)(fmt, heads, dim, page, [page * pages], seed, spare=0)  # noqa: E731
    pools = [make(9, 1), make(6, 2)]
    g = torch.Generator().manual_seed(5)
    for p in pools:
        for t in (p.k, p.v, p.ks, p.vs) + ((p.kg, p.vg) if fmt == "e2m1" else ()):
            if t is not None:
                t.view(torch.uint8).random_(0, 256, generator=g)
    for to_other in (False, True):
        dev = [p.device(DEV, permuted) for p in pools]
        caches = [tl.kv_cache(*d) for d in dev]
        moves = [[1, 2, page], [0, 3, 1], [5, 0, 0], [4, 5, page - 1], [8, 1, 2 * page]] if to_other else [[1, 2, page], [0, 3, 1], [5, 6, 0], [4, 7, page - 1]]
        n = len(moves)
        # (more rows than are to be done)
        tl.page_copy(caches[0], i32(moves + [[0, 4, page]]), i32([n]), to=caches[1] if to_other else None)
        tl.device_status()
        want = [[None if t is None else t.contiguous().view(torch.uint8).cpu().clone() for t in p.device("cpu")] for p in pools]
        dst = want[1 if to_other else 0]
        for f, t, rows in moves:
            for s, d in zip(want[0], dst):
                if s is not None:
                    s4, d4 = (z.view(z.shape[0], heads, page, -1) for z in (s, d))
                    d4[t, :, :rows] = s4[f, :, :rows]
        for d, w in zip(dev, want):
            for a, z in zip(d, w):
                assert a is None or torch.equal(a.contiguous().view(torch.uint8).cpu(), z)


def test_copies_of_pages_that_do_not_exist_are_left_out_and_reported():
    from paper_2607_04031_b200 import binding as tl
    pool = ref.Pool4("e2m1", 2, 64, 16, [64], 1, spare=0)
    dev = pool.device(DEV)
    tl.page_copy(tl.kv_cache(*dev), i32([[4, 0, 16], [0, -1, 16], [2, 3, -5]]))
    with pytest.raises(tl.TileLensError, match="0xa00"):
        tl.device_status()
    for a, z in zip(dev, pool.device("cpu")):
        assert torch.equal(a.cpu().view(torch.uint8), z.view(torch.uint8))


def test_captured_calls_follow_the_tables():
    """reserve, copy, release and compact of one graph, replayed: what they decide is on the device."""
    from paper_2607_04031_b200 import binding as tl
    b = Both(3, 8, 30)
    pool = ref.Pool4("e2m1", 2, 64, 16, [30 * 16], 1, spare=0)
    dev = pool.device(DEV)
    cache = tl.kv_cache(*dev)
    start, tokens, keep = i32([0, 0, 0]), i32([0, 0, 0]), i32([-1, -1, -1])
    ws = torch.empty(tl.page_workspace_bytes(b.t), dtype=torch.uint8, device=DEV)
    n2, m2, moves2 = i32([0]), i32([0]), torch.zeros(30, 3, dtype=torch.int32, device=DEV)

    def calls():
        tl.page_release(b.t, keep)
        tl.page_reserve(b.t, start, tokens, b.moves, b.n, b.m)
        tl.page_copy(cache, b.moves, b.n)
        tl.page_compact(b.t, moves2, n2, m2)
        tl.page_copy(cache, moves2, n2)
    tl.set_workspace(ws)
    try:
        calls()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            calls()
        for s, t, k in (([0, 0, 0], [40, 70, 5], [-1] * 3), ([40, 70, 5], [60, 71, 30], [40, 0, -1]), ([50, 0, 20], [80, 17, 31], [20, -1, 0])):
            start.copy_(i32(s)), tokens.copy_(i32(t)), keep.copy_(i32(k))
            graph.replay()
            b.plain.release(k)
            moves, missing = b.plain.reserve(s, t)
            assert (b.n.item(), b.m.item()) == (len(moves), missing)
            moves, in_use = b.plain.compact(30)
            assert (n2.item(), m2.item()) == (len(moves), in_use)
            b.same()
        tl.device_status()
    finally:
        tl.set_workspace(None)


def test_a_workspace_that_is_too_small_is_refused():
    from paper_2607_04031_b200 import binding as tl
    b = Both(3, 8, 30)
    small = torch.empty(256, dtype=torch.uint8, device=DEV)
    tl.set_workspace(small)
    try:
        for call in (lambda: b.reserve([0] * 3, [1] * 3), lambda: b.compact(), lambda: b.fork([0], [1], [5])):
            with pytest.raises(tl.TileLensError) as e:
                call()
            assert e.value.status == 6
    finally:
        tl.set_workspace(None)
