"""Page tables as wide as the longest sequence there may be, as a serving loop keeps them."""
import pytest
import torch

from test_gpu_tree_attention import FORMATS, Step, block_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("ctx,counts,rows", [([300], [26], 128), ([300, 200], [30, 26], 128), ([4000, 2500], [30, 26], 256)])
def test_the_choice_of_blocks_goes_by_the_pool_where_the_table_is_wide(fmt, dim, ctx, counts, rows):
    # 208 rows and more of a head, 4 multiprocessors: 128-row blocks for a few hundred positions, whatever the table has room for
    from paper_2607_04031_b200 import binding as tl
    s = Step(fmt, 4, 8, dim, 16, ctx, counts, seed=dim)
    with tl.option(tl.OPT_SM_LIMIT, 4):
        s.check()
        narrow, out = block_rows(s, 4), s.out.clone()
        s.pool.table = torch.nn.functional.pad(s.pool.table, (0, 8192 - s.pool.table.shape[1]), value=2 ** 31 - 1)
        s.run()
        tl.device_status()
        assert block_rows(s, 4) == narrow == rows
        assert torch.equal(s.out, out)
