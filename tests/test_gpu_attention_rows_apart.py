"""A row's result depends on what it sees and on nothing else, to the last bit."""
import pytest
import torch

from test_gpu_tree_attention import FORMATS, Step

pytestmark = pytest.mark.gpu

# few rows; 128-row blocks; 256-row blocks (on one multiprocessor)
SHAPES = [(2, 4, [6], None), (1, 8, [4], None), (2, 4, [48], None), (2, 8, [10, 16], None), (4, 4, [60], 1), (2, 8, [40, 33], 1)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
@pytest.mark.parametrize("ctx", [0, 45, 400])
def test_a_token_that_a_row_does_not_see_leaves_its_bits_alone(fmt, dim, heads, group, counts, sms, ctx):
    # token 1's key becomes 50 times as long: its neighbours' maxima grow by hundreds, or fall
    from paper_2607_04031_b200 import binding as tl
    ctxs = [ctx + 7 * b for b in range(len(counts))]
    one, two = (Step(fmt, heads, group, dim, 16, ctxs, counts, seed=40 + dim) for _ in range(2))
    k, v = two.pool.rows(0, ctxs[0] + 2)
    at = torch.tensor([ctxs[0] + 1])
    two.pool.write(0, at, (k[-1:] * 50).float(), -v[-1:].float())
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        a, la = one.run().float().cpu(), one.lse.cpu()
        b, lb = two.run().float().cpu(), two.lse.cpu()
        tl.device_status()
    sees = torch.zeros(sum(counts), dtype=torch.bool)
    sees[:counts[0]] = one.sees[0][:, 1]
    assert bool(sees.any()) and bool((~sees).any())
    assert torch.equal(a[~sees], b[~sees]) and torch.equal(la[~sees], lb[~sees])
    assert not torch.equal(a[sees], b[sees])
