"""Operators of the KV pool at the ends of their ranges: rows that are no
numbers, contexts and lists cut into many partitions."""
import numpy as np
import pytest

from oracle import gemv as og
from oracle import select as osel
from paper_2609_13592_amd import binding as bd
from paper_2609_13592_amd.step import Dims
from tests.gpu_util import stream, sync, to_dev_u16
from tests.test_gpu_kv4 import attention, check, fill, make, new_pool
from tests.test_gpu_sparse import Cache
from tests.test_gpu_step_cache import Run

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


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hq", [(2, 8), (1, 8)])
@pytest.mark.parametrize("blocks", [4, 70])
@pytest.mark.parametrize("size", [1, 2 ** 15, 2 ** 20, 2 ** 55])
def test_scores_of_any_size(gpu_ctx, fmt, H, Hq, blocks, size):
    """Scores 253 * 32 * size * size * a, a of 0, 1, -6 .., exact in fp32 however they are
    summed: far apart, so that the row is the value of the token with the
    largest, or the mean of the two that have it."""
    rng = np.random.default_rng(blocks)
    c = Cache(gpu_ctx, rng, fmt, [16 * blocks, 16 * blocks - 3], H, Hq)
    try:
        c.q[:] = 0
        d = rng.integers(0, 128, size=Hq)
        c.q[:, np.arange(Hq), d] = og.f32_to_bf16(np.float32(32 * 253 * size))
        best = np.zeros((2, H, 2), int)
        for b in range(2):
            k = rng.choice(np.array([0, 0.5, 1, -1, -6], np.float32), size=c.k[b].shape)
            v = rng.choice(np.array([0, 0.5, 1, -1, -6], np.float32), size=c.k[b].shape)
            best[b] = rng.integers(0, len(k), size=(H, 2))
            for h in range(H):
                k[best[b, h], h] = 6
            c.k[b][:], c.v[b][:] = og.f32_to_bf16(k * np.float32(size)), og.f32_to_bf16(v)
        c.write()
        lists = np.tile(np.arange(blocks, dtype=np.int32), (2, H, 1))
        for o in (c.attend(lists), attention(gpu_ctx, c.pool, 0, c.q, c.tables, c.lens)):
            for b in range(2):
                v = c.meaning(c.v[b])
                for h in range(Hq):
                    g = h // (Hq // H)
                    assert np.array_equal(o[b, h], v[np.unique(best[b, g]), g].mean(0)), (b, h)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("small", [-149 + 54, -101, -120])
def test_summaries_round_outwards_at_any_ratio(gpu_ctx, fmt, small):
    """Keys 2^60 in some dims beside 2^small in the others, of either sign: a
    step of 2^54 (a product of 2^(small - 54) is no fp32 number) still has the
    small ones within [-1, 0] or [0, 1]."""
    rng = np.random.default_rng(1)
    c = Cache(gpu_ctx, rng, fmt, [100, 33, 1], 2, 8)
    try:
        for k in c.k:
            x = rng.choice(np.array([1, -1, 0.5], np.float32), size=k.shape) * np.float32(2.0 ** small)
            for t in range(0, len(k), 16):  # one sign a dim and block: both bounds at 0 and beyond
                x[t:t + 16] = np.abs(x[t:t + 16]) * rng.choice(np.array([1, -1, 1], np.float32), size=x.shape[1:])
            x[:, :, :32] = rng.choice(np.array([1, -1, 0.5], np.float32), size=x[:, :, :32].shape) * np.float32(2.0 ** 60)
            k[:] = og.f32_to_bf16(x)
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        c.check_selection(2)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("top", [1, 2, 3])
def test_a_step_over_the_fewest_blocks(gpu_ctx, fmt, top):
    """The blocks that are always taken by default, as far as the list goes:
    the last two, then the first."""
    dims = Dims(layers=2, d=512, hq=8, hkv=2, hd=128, ffn=384, vocab=500)
    r = Run(gpu_ctx, dims, fmt, [1, 17, 300], top)
    try:
        ids, logits = r.step()
        assert np.all(np.isfinite(logits)) and np.array_equal(ids, logits.argmax(1))
        q, lists = r.model.q.cpu().double().numpy(), r.model.sel.cpu().numpy()
        for b, (k, _) in enumerate(r.held(1)):  # the last layer's
            want = osel.select(osel.scores(q[b], k), top, top > 2, min(top, 2))
            assert np.array_equal(lists[b], want), b
    finally:
        r.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("wide", [2 ** 26 + 5, 2 ** 31 - 1])
def test_tables_as_wide_as_an_int32_goes(gpu_ctx, fmt, wide):
    """A table and scores of up to 8 GiB each: the launches follow what a
    context can have, and block numbers do not overflow at the table's end."""
    import torch
    rng = np.random.default_rng(3)
    c = Cache(gpu_ctx, rng, fmt, [1000], 1, 4)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        table = torch.full((wide,), -1, dtype=torch.int32, device="cuda")
        table[:c.mb] = torch.from_numpy(c.tables[0]).cuda()
        i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        bd.boost_kv_index_update(gpu_ctx, c.pool, 0, table, wide, i32(0), i32(1000), 1, 2 ** 31 - 1, stream())
        scores = torch.full((wide,), 77.0, dtype=torch.float32, device="cuda")
        sel = i32(*[99] * 9)
        bd.boost_kv_select(gpu_ctx, c.pool, 0, to_dev_u16(c.q), 1, 4, table, wide, i32(1000), 9, 1, 2, scores,
                           sel, stream())
        sync()
        want = osel.scores(og.bf16_to_f32(c.q[0]).astype(np.float64), c.meaning(c.k[0]))
        assert np.array_equal(scores[:63].cpu().numpy()[None], want)
        assert bool((scores[63:] == 77.0).all())
        assert np.array_equal(sel.cpu().numpy()[None], osel.select(want, 9, 1, 2))
    finally:
        c.close()


def test_a_copy_of_nothing(gpu_ctx):
    """n = 0 does nothing, with or without arrays; pairs need them."""
    c = Cache(gpu_ctx, np.random.default_rng(0), bd.KV_BF16, [1], 1, 1)
    try:
        call = bd.load().boost_kv_copy_blocks
        some = np.zeros(1, np.int32)
        for src, dst in ((None, None), (some.ctypes.data, None), (some.ctypes.data, some.ctypes.data)):
            assert call(gpu_ctx, c.pool, 0, 1, src, dst, 0, stream()) == bd.OK
        assert call(gpu_ctx, c.pool, 0, 1, None, some.ctypes.data, 1, stream()) == bd.EINVAL
        assert call(gpu_ctx, c.pool, 0, 1, some.ctypes.data, None, 1, stream()) == bd.EINVAL
    finally:
        c.close()


@pytest.mark.parametrize("Hq,H,B,hi,mode,M", [(32, 8, 70, 3000, bd.KV_ALL_HBM, 0), (4, 1, 70, 3000, bd.KV_ALL_HBM, 0),
                                              (16, 2, 130, 2700, bd.KV_LPP, 2), (8, 1, 300, 2600, bd.KV_LPP, 2),
                                              (10, 5, 65, 4000, bd.KV_ALL_HOST, 0)])
def test_4bit_partitions_of_many_requests(gpu_ctx, Hq, H, B, hi, mode, M):
    """More than 64 requests in tables of more than 160 blocks: the one 4-bit
    kernel that searches its items by barriers (to 160 blocks contexts stay
    whole, up to 64 requests wavefronts search), over one and two rounds of 256
    requests, up to four query heads and eight, pages on host and not."""
    rng = np.random.default_rng(B + hi)
    lens = rng.integers(1, hi, size=B, endpoint=True)
    lens[0] = hi
    lens[[2, B - 1]] = 0
    lens[5:9] = [1, 16, 17, 2561]
    mb, nb = (hi + 15) // 16, int(((lens + 15) // 16).sum())
    assert mb > 160
    tables, ks, vs, q = make(rng, lens, H, Hq, nb, mb)
    pool = new_pool(gpu_ctx, H, Hq, nb, M, mode, max_batch=B, max_blocks=mb)
    try:
        if mode != bd.KV_ALL_HBM:
            assert bd.boost_kv_pool_info(pool)["host_pages_per_tensor"] > 0
        fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
        o = attention(gpu_ctx, pool, 0, q, tables, lens)
        check(o, q, ks, vs, lens)
        assert np.array_equal(attention(gpu_ctx, pool, 0, q, tables, lens, bd.DTYPE_BF16), og.f32_to_bf16(o))
        on = attention(gpu_ctx, pool, 0, q, tables, lens, fn=bd.boost_paged_attn_decode_noalloc)
        assert np.array_equal(on.view(np.uint32), o.view(np.uint32))
        # requests one by one, whose items wavefronts search
        for b in (0, 1, 5, 8, B - 2):
            one = attention(gpu_ctx, pool, 0, q[b:b + 1], tables[b:b + 1], lens[b:b + 1])
            check(one, q[b:b + 1], ks[b:b + 1], vs[b:b + 1], lens[b:b + 1])
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("Hq,H,B,hi", [(64, 8, 40, 300), (40, 8, 33, 2560), (7, 1, 300, 90)])
def test_4bit_whole_contexts_of_many_heads(gpu_ctx, Hq, H, B, hi):
    """More than four query heads to a KV head, more (request, KV head) pairs
    than compute units, tables of up to 160 blocks: one workgroup of four
    wavefronts a pair, nothing to merge."""
    rng = np.random.default_rng(B)
    lens = rng.integers(1, hi, size=B, endpoint=True)
    lens[:4] = [hi, 1, 0, 17]
    lens[B - 1] = 0
    mb, nb = (hi + 15) // 16, int(((lens + 15) // 16).sum())
    tables, ks, vs, q = make(rng, lens, H, Hq, nb, mb)
    pool = new_pool(gpu_ctx, H, Hq, nb, max_batch=B, max_blocks=mb)
    try:
        fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
        o = attention(gpu_ctx, pool, 0, q, tables, lens)
        check(o, q, ks, vs, lens)
        assert np.array_equal(attention(gpu_ctx, pool, 0, q, tables, lens, bd.DTYPE_BF16), og.f32_to_bf16(o))
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_pool_for_the_longest_contexts(gpu_ctx, fmt):
    """max_blocks_per_seq 2^27, what int32 tokens fill (16 GiB of scratch for one
    query head): calls over short tables run."""
    rng = np.random.default_rng(2)
    lens = np.array([1000])
    tables, ks, vs, q = make(rng, lens, 1, 1, 63, 63)
    pool = new_pool(gpu_ctx, 1, 1, 63, max_batch=1, max_blocks=2 ** 27, fmt=fmt)
    small = new_pool(gpu_ctx, 1, 1, 63, max_batch=1, max_blocks=63, fmt=fmt)
    try:
        rows = []
        for p in (pool, small):
            fill(gpu_ctx, p, 0, lens, tables, ks, vs)
            rows.append(attention(gpu_ctx, p, 0, q, tables, lens))
        assert np.any(rows[0]) and np.array_equal(rows[0].view(np.uint32), rows[1].view(np.uint32))
    finally:
        bd.boost_kv_pool_destroy(pool)
        bd.boost_kv_pool_destroy(small)
