"""GPU parity of block copies, and forked requests decoding side by side."""
import numpy as np
import pytest

from oracle import gemv as og
from oracle import kv4
from paper_2609_13592_amd import binding as bd
from tests.gpu_util import dev_f32, dev_u16, host_u16, stream, sync, to_dev_u16

pytestmark = pytest.mark.gpu


def dev_i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def rand_u16(rng, shape):
    return og.f32_to_bf16(rng.standard_normal(shape).astype(np.float32))


def everything(ctx, pool, layers, H, D, nb):
    """Every slot of the pool as it reads back: [layers, 2, nb, 16, H, D]."""
    n = nb * 16
    out = np.empty((layers, 2, nb, 16, H, D), np.uint16)
    slots = dev_i32(np.arange(n))
    k, v = dev_u16(n, H, D), dev_u16(n, H, D)
    for layer in range(layers):
        bd.boost_kv_read(ctx, pool, layer, slots, k, v, n, stream())
        sync()
        out[layer, 0], out[layer, 1] = (host_u16(x).reshape(nb, 16, H, D) for x in (k, v))
    return out


def filled(ctx, rng, fmt, layers, H, D, nb, mode, M):
    pool = bd.boost_kv_pool_create_format(ctx, fmt, layers, H, D, nb, M, mode, q_heads=H, max_batch=4,
                                          max_blocks_per_seq=64)
    nb = bd.boost_kv_pool_info(pool)["nb_pool"]
    for layer in range(layers):
        bd.boost_kv_write(ctx, pool, layer, dev_i32(np.arange(nb * 16)), to_dev_u16(rand_u16(rng, (nb * 16, H, D))),
                          to_dev_u16(rand_u16(rng, (nb * 16, H, D))), nb * 16, stream())
    sync()
    return pool, nb


@pytest.mark.parametrize("fmt,D", [(bd.KV_BF16, 128), (bd.KV_BF16, 64), (bd.KV_FP4, 128)])
@pytest.mark.parametrize("mode,M", [(bd.KV_ALL_HBM, 0), (bd.KV_LPP, 2), (bd.KV_ALL_HOST, 0)])
def test_copies_move_whole_blocks_and_nothing_else(gpu_ctx, fmt, D, mode, M):
    rng = np.random.default_rng(0)
    layers, H = 3, 3
    pool, nb = filled(gpu_ctx, rng, fmt, layers, H, D, 500, mode, M)
    try:
        want = everything(gpu_ctx, pool, layers, H, D, nb)
        order = rng.permutation(nb)
        ends = [0, nb - 1]
        order = np.concatenate([ends, order[~np.isin(order, ends)]])
        for layer0, n_layers, n in ((0, 3, 1), (1, 1, 7), (0, 2, 130), (2, 1, 0)):
            src = order[rng.integers(1, 100, n)]
            dst = order[100:100 + n] if n > 1 else order[:n]
            bd.boost_kv_copy_blocks(gpu_ctx, pool, layer0, n_layers, src, dst, n, stream())
            want[layer0:layer0 + n_layers, :, dst] = want[layer0:layer0 + n_layers, :, src]
            assert np.array_equal(everything(gpu_ctx, pool, layers, H, D, nb), want)
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_more_pairs_than_a_launch_carries(gpu_ctx):
    rng = np.random.default_rng(1)
    pool, nb = filled(gpu_ctx, rng, bd.KV_BF16, 1, 1, 128, 2000, bd.KV_ALL_HBM, 0)
    try:
        want = everything(gpu_ctx, pool, 1, 1, 128, nb)
        order = rng.permutation(nb)
        src, dst = order[:900], order[900:1800]
        bd.boost_kv_copy_blocks(gpu_ctx, pool, 0, 1, src, dst, 900, stream())
        want[:, :, dst] = want[:, :, src]
        assert np.array_equal(everything(gpu_ctx, pool, 1, 1, 128, nb), want)
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("fmt", [bd.KV_BF16, bd.KV_FP4])
def test_summaries_go_with_their_blocks(gpu_ctx, fmt):
    """The copy's scores are the source's, in the layers that were copied."""
    import torch
    rng = np.random.default_rng(2)
    pool, nb = filled(gpu_ctx, rng, fmt, 2, 2, 128, 500, bd.KV_LPP, 3)
    try:
        bd.boost_kv_index_enable(pool)
        every = np.arange(60, dtype=np.int32)[None]
        lens = dev_i32([960])
        q = to_dev_u16(rand_u16(rng, (1, 2, 128)))

        def scores(layer):
            sc, sel = dev_f32(1, 2, 60), dev_i32(np.zeros((1, 2, 4)))
            bd.boost_kv_select(gpu_ctx, pool, layer, q, 1, 2, dev_i32(every), 60, lens, 4, 0, 0, sc, sel, stream())
            sync()
            return sc.cpu().numpy()[0]
        for layer in (0, 1):
            bd.boost_kv_index_update(gpu_ctx, pool, layer, dev_i32(every), 60, dev_i32([0]), lens, 1, 960, stream())
        before = [scores(0), scores(1)]
        bd.boost_kv_copy_blocks(gpu_ctx, pool, 1, 1, [3, 3, 50], [10, 59, 0], 3, stream())
        after = [scores(0), scores(1)]
        want = before[1].copy()
        want[:, [10, 59, 0]] = want[:, [3, 3, 50]]
        assert np.array_equal(after[0], before[0]) and np.array_equal(after[1], want)
        torch.cuda.synchronize()
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_refusals(gpu_ctx):
    pool = bd.boost_kv_pool_create(gpu_ctx, 3, 2, 128, 512, 0, bd.KV_ALL_HBM, q_heads=2, max_batch=1,
                                   max_blocks_per_seq=1)
    try:
        for layer0, n_layers, src, dst in ((-1, 1, [0], [1]), (0, 0, [0], [1]), (0, 4, [0], [1]), (3, 1, [0], [1]),
                                           (0, 1, [512], [1]), (0, 1, [-1], [1]), (0, 1, [0], [512]),
                                           (0, 1, [0], [-1]), (0, 1, [0, 1], [2, 2]), (0, 1, [0, 1], [2, 0]),
                                           (0, 1, [7], [7]), (2 ** 31 - 1, 2, [0], [1]),
                                           (0, 1, [5, 6, 7, 2 ** 31 - 1], [1, 2, 3, 4])):
            with pytest.raises(bd.BoostError) as e:
                bd.boost_kv_copy_blocks(gpu_ctx, pool, layer0, n_layers, src, dst, len(src), stream())
            assert e.value.code == bd.EINVAL
        for n, s in ((-1, 0), (1, None)):
            rc = bd.load().boost_kv_copy_blocks(gpu_ctx, pool, 0, 1, s, None, n, None)
            assert rc == bd.EINVAL
        bd.boost_kv_copy_blocks(gpu_ctx, pool, 0, 1, [], [], 0, stream())
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_a_copy_in_a_graph(gpu_ctx):
    """Captured on another stream and replayed over changing contents."""
    import torch
    rng = np.random.default_rng(3)
    pool, nb = filled(gpu_ctx, rng, bd.KV_FP4, 2, 2, 128, 500, bd.KV_ALL_HBM, 0)
    try:
        src, dst = [4, 9, 4], [100, 200, 300]
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            bd.boost_kv_copy_blocks(gpu_ctx, pool, 0, 2, src, dst, 3, torch.cuda.current_stream().cuda_stream)
        for _ in range(3):
            rows = rand_u16(rng, (32, 2, 128))
            slots = np.concatenate([4 * 16 + np.arange(16), 9 * 16 + np.arange(16)])
            for layer in (0, 1):
                bd.boost_kv_write(gpu_ctx, pool, layer, dev_i32(slots), to_dev_u16(rows), to_dev_u16(rows), 32, stream())
            sync()
            want = everything(gpu_ctx, pool, 2, 2, 128, nb)
            want[:, :, dst] = want[:, :, src]
            graph.replay()
            sync()
            assert np.array_equal(everything(gpu_ctx, pool, 2, 2, 128, nb), want)
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("fmt", [bd.KV_BF16, bd.KV_FP4])
@pytest.mark.parametrize("mode,M", [(bd.KV_ALL_HBM, 0), (bd.KV_LPP, 3)])
def test_forked_requests_decode_side_by_side(gpu_ctx, fmt, mode, M):
    """One prompt, three continuations: fork, unshare and copy the last block,
    append, summarise, select, attend, for several steps, with a truncation and
    a compaction between; every row against its own keys and values."""
    rng = np.random.default_rng(4)
    H, Hq, mb, top, L0 = 4, 16, 40, 8, 300
    pool = bd.boost_kv_pool_create_format(gpu_ctx, fmt, 1, H, 128, 400, M, mode, q_heads=Hq, max_batch=4,
                                          max_blocks_per_seq=mb)
    try:
        bd.boost_kv_index_enable(pool)
        filler = bd.boost_kv_alloc(pool, 99, 60)  # so that compaction has something to do
        bd.boost_kv_alloc(pool, 0, (L0 + 15) // 16)
        bd.boost_kv_truncate(pool, 99, 5)
        assert bd.boost_kv_request_blocks(pool, 99).tolist() == filler[:5]
        k, v = rand_u16(rng, (L0, H, 128)), rand_u16(rng, (L0, H, 128))
        ks, vs = [k], [v]

        def tables(n):
            t = np.full((n, mb), -1, np.int32)
            for r in range(n):
                b = bd.boost_kv_request_blocks(pool, r)
                t[r, :len(b)] = b
            return t
        t = tables(1)
        at = np.arange(L0)
        bd.boost_kv_write(gpu_ctx, pool, 0, dev_i32(t[0, at // 16] * 16 + at % 16), to_dev_u16(k), to_dev_u16(v), L0,
                          stream())
        bd.boost_kv_index_update(gpu_ctx, pool, 0, dev_i32(t), mb, dev_i32([0]), dev_i32([L0]), 1, L0, stream())
        for child in (1, 2):
            bd.boost_kv_fork(pool, 0, child, (L0 + 15) // 16)
            ks.append(k)
            vs.append(v)
        lens = np.full(3, L0)

        def values(x):
            return kv4.stored(x) if fmt == bd.KV_FP4 else og.bf16_to_f32(x).astype(np.float64)
        for turn in range(24):
            if turn == 9:  # request 2 takes back its last eight tokens
                lens[2] -= 8
                ks[2], vs[2] = ks[2][:lens[2]], vs[2][:lens[2]]
                bd.boost_kv_truncate(pool, 2, (int(lens[2]) + 15) // 16)
            pairs = []
            for r in range(3):  # room for the new token, in a block that is the request's own
                held = len(bd.boost_kv_request_blocks(pool, r))
                if lens[r] // 16 >= held:
                    assert bd.boost_kv_alloc(pool, r, 1) != bd.EAGAIN
                else:
                    s, d = bd.boost_kv_unshare(pool, r, int(lens[r]) // 16)
                    if s != d:
                        pairs.append((s, d))
            assert len(pairs) == (2 if turn == 0 else 0)  # the last holder keeps the block
            if pairs:
                bd.boost_kv_copy_blocks(gpu_ctx, pool, 0, 1, *zip(*pairs), len(pairs), stream())
            if turn == 15:
                src, dst = bd.boost_kv_compact(pool, 1000)
                assert len(src) > 0
                bd.boost_kv_copy_blocks(gpu_ctx, pool, 0, 1, src, dst, len(src), stream())
                junk = np.asarray(src)[:, None] * 16 + np.arange(16)  # what was left behind no longer matters
                bad = np.full((junk.size, H, 128), 0x7fc0, np.uint16)
                bd.boost_kv_write(gpu_ctx, pool, 0, dev_i32(junk.ravel()), to_dev_u16(bad), to_dev_u16(bad),
                                  junk.size, stream())
            nk, nv, q = rand_u16(rng, (3, H, 128)), rand_u16(rng, (3, H, 128)), rand_u16(rng, (3, Hq, 128))
            td, pos = dev_i32(tables(3)), dev_i32(lens)
            bd.boost_kv_append(gpu_ctx, pool, 0, td, mb, pos, to_dev_u16(nk), to_dev_u16(nv), 3, stream())
            for r in range(3):
                ks[r], vs[r] = np.concatenate([ks[r], nk[r:r + 1]]), np.concatenate([vs[r], nv[r:r + 1]])
            lens = lens + 1
            ends = dev_i32(lens)
            bd.boost_kv_index_update(gpu_ctx, pool, 0, td, mb, pos, ends, 3, 1, stream())
            sc, sel = dev_f32(3, H, mb), dev_i32(np.zeros((3, H, top)))
            o = dev_f32(3, Hq, 128)
            qd = to_dev_u16(q)
            bd.boost_kv_select(gpu_ctx, pool, 0, qd, 3, Hq, td, mb, ends, top, 1, 1, sc, sel, stream())
            bd.boost_sparse_attn_decode(gpu_ctx, pool, 0, qd, 3, Hq, td, mb, ends, sel, top, 0.0, o, bd.DTYPE_F32,
                                        stream())
            sync()
            sel, o = sel.cpu().numpy(), o.cpu().numpy()
            qf = og.bf16_to_f32(q).astype(np.float64)
            from oracle import select as osel
            for r in range(3):
                kk, vv = values(ks[r]), values(vs[r])
                assert np.array_equal(sel[r], osel.select(osel.scores(qf[r], kk), top, 1, 1)), (turn, r)
                for h in range(Hq):
                    tok = (sel[r, h // 4][:, None] * 16 + np.arange(16)).ravel()
                    tok = tok[tok < lens[r]]
                    want = kv4.attend(qf[r, h][None], kk[tok, h // 4], vv[tok, h // 4])[0]
                    # the bound of tests/test_gpu_sparse.py for 128 tokens: a score
                    # off by 130 * 2^-24 * sum|q k| / sqrt(128) (sum|q k| < 200 here:
                    # 1.4e-4), twice that and 2^-16 times max|v| < 5
                    assert np.abs(o[r, h] - want).max() < 1.5e-3, (turn, r, h)
    finally:
        bd.boost_kv_pool_destroy(pool)
