"""Positions of more rows than 32-bit thread numbers count warps."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rows", [2 ** 26 + 300, 2 ** 27 + 300])
def test_positions_of_the_last_rows(rows):
    # two requests, each a root that all others hang from, but for a chain at its end
    from paper_2607_04031_b200 import binding as tl
    first = 2 ** 26 - 100
    parents = torch.zeros(rows, dtype=torch.int32, device=DEV)
    want = torch.ones(rows, dtype=torch.int32, device=DEV)
    for a, n in ((0, first), (first, rows - first)):
        chain = torch.arange(n - 40, n, dtype=torch.int32, device=DEV)
        parents[a + n - 40:a + n] = chain - 1
        want[a + n - 40:a + n] = torch.arange(2, 42, dtype=torch.int32, device=DEV)
        parents[a], want[a] = -1, 0
    want[:first] += 5
    want[first:] += 1000
    got = torch.full((rows + 8,), -7, dtype=torch.int32, device=DEV)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    tl.tree_positions(parents, i32([0, first, rows]), i32([5, 1000]), got[:rows])
    tl.device_status()
    assert torch.equal(got[:rows], want)
    assert bool((got[rows:] == -7).all())
