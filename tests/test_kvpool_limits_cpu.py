"""The KV pool's allocator with long requests (no GPU)."""
import time

import numpy as np

from paper_2609_13592_amd import binding as bd


def test_a_request_grows_block_by_block_in_linear_time():
    """A decoding request takes one block at a time: 300000 of them by one
    request cost about what they cost 1000 requests.  (With the whole list
    copied at each call it would be 180 GB, some 20 seconds.)"""
    n = 300000
    ctx = bd.boost_init(-1)
    pool = bd.boost_kv_pool_create(ctx, 1, 1, 128, n, 2, bd.KV_ALL_HBM)
    try:
        def take(requests):
            t = time.process_time()
            for i in range(n):
                assert len(bd.boost_kv_alloc(pool, i % requests, 1)) == 1
            return time.process_time() - t
        spread = take(1000)
        for r in range(1000):
            bd.boost_kv_free(pool, r)
        one = take(1)
        assert one < 3 * spread + 1
        assert np.array_equal(bd.boost_kv_request_blocks(pool, 0), np.arange(n))
    finally:
        bd.boost_kv_pool_destroy(pool)
        bd.boost_shutdown(ctx)
