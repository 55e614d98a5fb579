"""Prompts and their chunks: several hundred causal rows a request, from position 0 and behind a context."""
import pytest

from test_gpu_tree_attention import FORMATS, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim,heads,group,page", [(64, 1, 2, 16), (128, 1, 3, 128), (256, 1, 1, 32)])
@pytest.mark.parametrize("ctx,counts", [([0], [600]), ([800], [512]), ([0, 333, 1000], [257, 1, 130])])
def test_several_hundred_causal_rows(fmt, dim, heads, group, page, ctx, counts):
    Step(fmt, heads, group, dim, page, ctx, counts, trees="causal", seed=dim + len(ctx)).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
def test_a_prompt_in_blocks_of_256_rows(fmt, dim):
    from paper_2607_04031_b200 import binding as tl
    with tl.option(tl.OPT_SM_LIMIT, 1):
        Step(fmt, 2, 2, dim, 64, [700], [300], trees="causal", seed=dim).check()
