"""GPU: entries among a sequence's that name no block are not its own: freeing what lies behind the window neither writes
them nor ends at them, and the other operators leave them, and the counts, alone."""
import numpy as np
import pytest
import torch

import paper_2602_09323_amd as coopt
from test_gpu_blocks import make

pytestmark = pytest.mark.gpu


def _with_foreign(pool, dev, places):
    """Other numbers in the place of blocks that the sequences held."""
    for s, e, value in places:
        pool.refs[pool.tables[s, e]] -= 1
        pool.tables[s, e] = value
    dev.tables.copy_(torch.from_numpy(pool.tables.astype(np.int32)))
    coopt.kv_blocks_init(*dev.state, dev.shape)
    dev.check(pool, "init")


@pytest.mark.parametrize("window,sinks", [(16, 0), (40, 33), (700, 16)])
def test_behind_a_window(window, sinks):
    lens = [2000, 300, 1040, 0]
    pool, dev = make(51, 4, 400, 140, lens)
    _with_foreign(pool, dev, [(0, 0, 400), (0, 5, 1 << 30), (0, 60, 0x7FFFFFFF), (0, 61, -7), (1, 3, 401), (2, 64, 12345), (2, 20, -(1 << 31))])
    for _ in range(3):
        dev.outside(pool, window, sinks)
        dev.reserve(pool, [0, 30, 70, 75, 80], 80)
    dev.compact(pool)
    dev.free_seqs(pool, [0, 1, 2, 3])
    assert len(pool.free_blocks()) == 400
