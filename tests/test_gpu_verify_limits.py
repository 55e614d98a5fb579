"""How many children of one node tl_tree_verify tries."""
import numpy as np
import pytest
import torch

import kv_util as ref
from test_gpu_tree_verify import _run

pytestmark = pytest.mark.gpu
TRIED = 512                                                  # as the header says


def _star(children, vocab, drafts):
    """A root whose first children are refused: without draft distributions by their random numbers, with them because the target
    gives their tokens nothing."""
    q = torch.full((children + 1, vocab), 1.0 / vocab)
    p = q.clone()
    if drafts:
        p[:, :vocab // 2] = 0
        p[:, vocab // 2:] *= 2
    tokens = [0] + list(range(children))
    accept = np.full(children + 1, 0.9999, dtype=np.float32)
    return p, q if drafts else None, tokens, accept


@pytest.mark.parametrize("drafts", [True, False])
@pytest.mark.parametrize("children,lucky", [(n, c) for n in (511, 512, 513, 600) for c in (None, 511, 512, 513, 514, 600) if c is None or c <= n])
@pytest.mark.parametrize("vocab", [1400, 20002])
def test_the_children_that_are_tried(drafts, children, lucky, vocab):
    p, q, tokens, accept = _star(children, vocab, drafts)
    if lucky is not None:                                    # this child would be kept
        accept[lucky] = 0.0
        tokens[lucky] = vocab - 3
    sample = np.array([0.30037], dtype=np.float32)
    parents = [-1] + [0] * children
    n = min(children, TRIED) + 1
    path, nxt = ref.verify(p[:n].numpy(), None if q is None else q[:n].numpy(), tokens[:n], parents[:n], accept[:n], sample[0], 4)
    assert len(path) == (2 if lucky is not None and lucky <= TRIED else 1)
    got = _run(p, q, tokens, [parents], accept, sample, 4)
    assert got[0][0].tolist() == path + [-1] * (4 - len(path)) and got[1][0] == len(path) and got[2][0] == nxt
