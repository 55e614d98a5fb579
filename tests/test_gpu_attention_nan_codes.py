"""E4M3 codes that stand for NaN at masked positions (memory that nobody wrote, or rows another program quantised)."""
import math

import pytest
import torch

import kv_util as ref
from test_gpu_tree_attention import Step

pytestmark = pytest.mark.gpu


def _pair(heads, group, dim, ctx, counts, seed):
    return [Step("e4m3", heads, group, dim, 16, ctx, counts, seed=seed) for _ in range(2)]


def _spoil(step, b, pos, which, dims):
    """NaN bytes of either sign at one position of a request, its scales finite."""
    pg, line = step.pool.place(b, torch.tensor([pos]))
    codes = (step.pool.k if which == "k" else step.pool.v).view(torch.uint8)
    for i, d in enumerate(dims):
        codes[pg, :, line, d] = 0x7F if i % 2 == 0 else 0xFF


# few rows; 128-row blocks; 256-row blocks (on one multiprocessor)
SHAPES = [(2, 4, [6], None), (2, 8, [3, 2], None), (1, 8, [4], None), (2, 4, [48], None), (2, 8, [10, 16], None), (4, 4, [60], 1), (2, 8, [40, 33], 1)]


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
@pytest.mark.parametrize("ctx", [0, 45, 400])
def test_masked_nan_codes_have_no_influence(dim, heads, group, counts, sms, ctx):
    from paper_2607_04031_b200 import binding as tl
    ctxs = [ctx + 7 * b for b in range(len(counts))]
    clean, dirty = _pair(heads, group, dim, ctxs, counts, seed=21 + dim)
    spoiled = (1, counts[0] - 1)                             # one token in the middle of the tree, and the last
    for j in spoiled:
        _spoil(dirty, 0, ctxs[0] + j, "v", range(dim))
    _spoil(dirty, 0, ctxs[0] + 1, "k", range(0, dim, 3))
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        a, la = clean.run().float().cpu(), clean.lse.cpu()
        b, lb = dirty.run().float().cpu(), dirty.lse.cpu()
        tl.device_status()
    sees = torch.zeros(sum(counts), dtype=torch.bool)
    sees[:counts[0]] = clean.sees[0][:, list(spoiled)].any(1)
    assert bool(sees.any()) and bool((~sees).any())
    assert torch.equal(a[~sees], b[~sees]) and torch.equal(la[~sees], lb[~sees])
    assert bool(b[sees].isnan().all())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,counts,sms", SHAPES)
@pytest.mark.parametrize("where", ["step", "context"])
def test_nan_codes_that_are_seen_spoil_their_dimensions(dim, heads, group, counts, sms, where):
    # value codes alone: the rows that see them have NaN in those dimensions, and elsewhere the bits they had
    from paper_2607_04031_b200 import binding as tl
    ctxs = [45 + 7 * b for b in range(len(counts))]
    clean, dirty = _pair(heads, group, dim, ctxs, counts, seed=33 + dim)
    dims = [0, 7, 31, 32, dim // 2 + 1, dim - 1]
    _spoil(dirty, 0, ctxs[0] + 1 if where == "step" else 20, "v", dims)
    pg, line = clean.pool.place(0, torch.tensor([ctxs[0] + 1 if where == "step" else 20]))
    clean.pool.v.view(torch.uint8)[pg, :, line] = dirty.pool.v.view(torch.uint8)[pg, :, line]
    for d in dims:
        clean.pool.v.view(torch.uint8)[pg, :, line, d] = 0
    with tl.option(tl.OPT_SM_LIMIT, sms or 0):
        a, b = clean.run().float().cpu(), dirty.run().float().cpu()
        tl.device_status()
    sees = torch.zeros(sum(counts), dtype=torch.bool)
    sees[:counts[0]] = clean.sees[0][:, 1] if where == "step" else True
    spoiled = torch.zeros(dim, dtype=torch.bool)
    spoiled[dims] = True
    assert bool(b[sees][..., spoiled].isnan().all())
    assert torch.equal(a[sees][..., ~spoiled], b[sees][..., ~spoiled]) and torch.equal(a[~sees], b[~sees])


@pytest.mark.parametrize("counts", [[6], [48]])
def test_a_pool_that_was_never_written(counts):
    # every byte of the pool 0xFF, scales 1: only the tokens a row sees were written
    from paper_2607_04031_b200 import binding as tl
    n = counts[0]
    s = Step("e4m3", 2, 4, 128, 16, [45], counts, seed=8)
    hidden = [j for j in range(1, n) if j % 3 == 0]
    s.sees[0][:, hidden] = False
    words = torch.zeros(n, s.words, dtype=torch.int64)
    for j in range(n):
        words[:, j // 32] |= s.sees[0][:, j].long() << (j % 32)
    s.mask = ((words + 2 ** 31) % 2 ** 32 - 2 ** 31).to(torch.int32)
    pg, line = s.pool.place(0, 45 + torch.tensor(hidden))
    for codes, scales in ((s.pool.k, s.pool.ks), (s.pool.v, s.pool.vs)):
        codes.view(torch.uint8)[pg, :, line] = 0xFF
        scales[pg, :, line] = 1.0
    out = s.run().double().cpu()
    tl.device_status()
    k, v = s.pool.rows(0, 45 + n)
    k, v = torch.nan_to_num(k), torch.nan_to_num(v)          # (masked ones alone)
    want, _, mass, big = ref.attention(s.q, k, v, 45, s.sees[0], s.scale)
    assert bool(((out - want).abs() <= ref.attention_bound(want, mass, big, v, "e4m3", 128, s.scale, 45 + n)).all())
    assert math.isfinite(float(out.abs().max()))
