"""Operators of the KV pool at the ends of their ranges: rows that are no
numbers, contexts and lists cut into many partitions."""
import numpy as np
import pytest

from paper_2609_13592_amd import binding as bd
from tests.gpu_util import dev_f32, dev_u16, host_u16, stream, sync, to_dev_u16
from tests.test_gpu_kv4 import attention
from tests.test_gpu_sparse import Cache, rand_u16

pytestmark = pytest.mark.gpu
FORMATS = [bd.KV_BF16, bd.KV_FP4]
NAN = 0x7fc0


# Blocks of the one long context (the table is as wide): one partition, several
# that one wavefront merges, many that sixteen do.  A 4-bit context or list is
# cut from 61 blocks on, a bf16 one from 5 (dense) or 9 (list) on.
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hq", [(2, 8), (2, 2), (1, 8)])
@pytest.mark.parametrize("blocks", [4, 70, 300])
def test_nan_shows_in_any_number_of_partitions(gpu_ctx, fmt, H, Hq, blocks):
    """A query head that is not a number, and a run of blocks whose keys are
    none, make their rows NaN however the context is cut; other rows keep
    their bits."""
    rng = np.random.default_rng(blocks)
    G = Hq // H
    lens = np.array([16 * blocks, 16 * blocks - 5, 16 * blocks, 7])
    c = Cache(gpu_ctx, rng, fmt, lens, H, Hq)
    try:
        c.write()
        sel = np.tile(np.arange(blocks, dtype=np.int32), (4, H, 1))
        sel[:, :, 2::5] = -1  # every fifth one is left out

        def rows():
            return [c.attend(sel), attention(gpu_ctx, c.pool, 0, c.q, c.tables, lens)]
        clean = rows()
        c.q[0, 1] = NAN  # one query head
        # whole partitions of request 1, last KV head: a quarter of its blocks
        n = blocks // 64 * 16 or 1
        c.k[1][16 * n:32 * n, H - 1, ::32] = NAN
        c.k[3][:, 0, ::32] = NAN  # all that request 3 has
        c.write()
        want = np.zeros((4, Hq), bool)
        want[0, 1] = True
        want[1, Hq - G:] = True
        want[3, :G] = True
        for o, before in zip(rows(), clean):
            assert np.array_equal(np.isnan(o).all(2), want)
            assert np.array_equal(o[~want].view(np.uint32), before[~want].view(np.uint32))
    finally:
        c.close()
