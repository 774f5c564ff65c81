"""GPU parity of the 4-bit KV pool: storing, reading back and attention."""
import numpy as np
import pytest

from oracle import gemv as og
from oracle import kv4
from paper_2609_13592_amd import binding as bd
from tests.gpu_util import dev_f32, dev_u16, host_u16, stream, sync, to_dev_u16

pytestmark = pytest.mark.gpu


def new_pool(ctx, H, Hq, nb, M=0, mode=bd.KV_ALL_HBM, layers=1, max_batch=64, max_blocks=256,
             budget=0, fmt=bd.KV_FP4, D=128):
    return bd.boost_kv_pool_create_format(ctx, fmt, layers, H, D, nb, M, mode, q_heads=Hq,
                                          max_batch=max_batch, max_blocks_per_seq=max_blocks,
                                          hbm_budget_bytes=budget)


def dev_i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def read(ctx, pool, layer, slots, H, D=128):
    n = len(slots)
    k, v = dev_u16(n, H, D), dev_u16(n, H, D)
    k.fill_(-1), v.fill_(-1)
    bd.boost_kv_read(ctx, pool, layer, dev_i32(slots), k, v, n, stream())
    sync()
    return host_u16(k), host_u16(v)


def same_values(got_u16, want):
    """bf16 bits against fp64 values: equal numbers (zeros of either sign),
    NaN where NaN is expected."""
    got = og.bf16_to_f32(got_u16).astype(np.float64)
    return np.array_equal(np.isnan(got), np.isnan(want)) and \
        np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


def rand_kv(rng, shape, spread=3):
    return og.f32_to_bf16((rng.standard_normal(shape)
                           * np.exp2(rng.integers(-spread, spread + 1, shape[:-1] + (1,))))
                          .astype(np.float32))


def test_every_bf16_value_through_the_pool(gpu_ctx):
    """All 65536 bf16 patterns: in order (groups of neighbours), shuffled
    (groups of every size of value) and shuffled among finite ones only."""
    rng = np.random.default_rng(0)
    every = np.arange(65536, dtype=np.uint16)
    finite = every[(every & 0x7f80) != 0x7f80]
    rows = np.concatenate([every, rng.permutation(every), rng.permutation(finite)[:65024]])
    rows = rows.reshape(-1, 2, 128)  # [768 - 2, 2 heads, 128]
    n = rows.shape[0]
    pool = new_pool(gpu_ctx, 2, 2, 64, max_blocks=64)
    try:
        slots = rng.permutation(64 * 16)[:n]
        other = rows[rng.permutation(n)]
        bd.boost_kv_write(gpu_ctx, pool, 0, dev_i32(slots), to_dev_u16(rows), to_dev_u16(other), n,
                          stream())
        k, v = read(gpu_ctx, pool, 0, slots, 2)
        assert same_values(k, kv4.stored(rows))
        assert same_values(v, kv4.stored(other))
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("mode,M,budget", [(bd.KV_ALL_HBM, 0, 0), (bd.KV_LPP, 3, 0),
                                           (bd.KV_ALL_HOST, 0, 0),
                                           (bd.KV_BUDGET, 0, 4 * 5 * bd.PAGE_BYTES)])
@pytest.mark.parametrize("fmt,D", [(bd.KV_FP4, 128), (bd.KV_BF16, 128), (bd.KV_BF16, 64)])
def test_read_is_the_inverse_of_write(gpu_ctx, fmt, D, mode, M, budget):
    """Tokens of the first, the last and random blocks, two layers, every tier
    mode; skipped slots write nothing and leave their rows as they were."""
    rng = np.random.default_rng(1)
    H, nb = 4, 4000
    pool = new_pool(gpu_ctx, H, H, nb, M, mode, layers=2, budget=budget, fmt=fmt, D=D)
    try:
        nbp = bd.boost_kv_pool_info(pool)["nb_pool"]
        assert nbp % (1920 if fmt == bd.KV_FP4 else 2 ** 20 // (16 * D)) == 0 and nbp >= nb
        slots = np.concatenate([[0, nbp * 16 - 1, 1919 * 16 + 15, 1920 * 16],
                                rng.permutation(np.arange(100, nbp * 16 - 100))[:300]])
        slots = slots[(slots != 7) & (slots != 9)]
        n = len(slots)
        for layer in (1, 0):
            kk, vv = rand_kv(rng, (n, H, D)), rand_kv(rng, (n, H, D))
            bd.boost_kv_write(gpu_ctx, pool, layer, dev_i32(slots), to_dev_u16(kk), to_dev_u16(vv), n,
                              stream())
            junk = rand_kv(rng, (4, H, D))  # none of these is a slot of the pool
            bd.boost_kv_write(gpu_ctx, pool, layer, dev_i32([-1, nbp * 16, -2 ** 31, 2 ** 31 - 1]),
                              to_dev_u16(junk), to_dev_u16(junk), 4, stream())
            ask = np.concatenate([slots, [-1, nbp * 16, 2 ** 31 - 1]])
            k, v = read(gpu_ctx, pool, layer, ask, H, D)
            for got, put in ((k, kk), (v, vv)):
                if fmt == bd.KV_FP4:
                    assert same_values(got[:n], kv4.stored(put))
                else:
                    assert np.array_equal(got[:n], put)
                assert np.all(got[n:] == 0xffff)
        k0, _ = read(gpu_ctx, pool, 1, [7, 9], H, D)
        assert np.all(k0 == 0)  # never written
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("H,Hq,S", [(8, 32, 1), (1, 1, 4), (5, 10, 8)])
def test_append_forms_store_the_bits_of_write(gpu_ctx, H, Hq, S):
    """kv_append, rope_kv_append and its slices form against kv_write of the
    same rows; positions and blocks outside are skipped."""
    import torch
    rng = np.random.default_rng(2)
    B, mb = 9, 6
    pos = np.array([0, 1, 15, 16, 95, 40, -1, 96, 33])
    tables = rng.permutation(1000)[:B * mb].reshape(B, mb).astype(np.int32)
    tables[8, 2] = -1
    live = [0, 1, 2, 3, 4, 5]
    slots = [int(tables[b, pos[b] // 16]) * 16 + int(pos[b]) % 16 for b in live]
    pools = [new_pool(gpu_ctx, H, Hq, 1000, max_batch=B, max_blocks=mb) for _ in range(4)]
    try:
        N = (Hq + 2 * H) * 128
        K = 4096  # divides a page: no cut rows
        parts = torch.from_numpy((rng.standard_normal((S, B, N)) * 2).astype(np.float32)).cuda()
        qkv = torch.zeros((B, N), dtype=torch.float32, device="cuda")
        for s in range(S):
            qkv += parts[s]
        q, k, v = dev_u16(B, Hq, 128), dev_u16(B, H, 128), dev_u16(B, H, 128)
        td, pd = dev_i32(tables), dev_i32(pos)
        bd.boost_rope_qkv(gpu_ctx, qkv, pd, B, Hq, H, 128, 500000.0, q, k, v, stream())
        sync()
        idx = torch.tensor(live, device="cuda")
        ks, vs = k[idx].contiguous(), v[idx].contiguous()
        bd.boost_kv_write(gpu_ctx, pools[0], 0, dev_i32(slots), ks, vs, len(live), stream())
        bd.boost_kv_append(gpu_ctx, pools[1], 0, td, mb, pd, k, v, B, stream())
        q2, q3 = dev_u16(B, Hq, 128), dev_u16(B, Hq, 128)
        bd.boost_rope_kv_append(gpu_ctx, pools[2], 0, qkv, pd, B, Hq, 500000.0, td, mb, q2, stream())
        bd.boost_rope_kv_append_slices(gpu_ctx, pools[3], 0, parts, S, K, pd, B, Hq, 500000.0, td, mb,
                                       q3, stream())
        sync()
        assert torch.equal(q, q2) and torch.equal(q, q3)
        everything = np.arange(1000 * 16)
        want = read(gpu_ctx, pools[0], 0, everything, H)
        assert same_values(want[0][slots], kv4.stored(host_u16(ks)))
        for p in pools[1:]:
            got = read(gpu_ctx, p, 0, everything, H)
            for a, b in zip(got, want):
                assert same_values(a, og.bf16_to_f32(b).astype(np.float64))
    finally:
        for p in pools:
            bd.boost_kv_pool_destroy(p)


def fill(ctx, pool, layer, lens, tables, ks, vs):
    slots, kk, vv = [], [], []
    for b, L in enumerate(lens):
        if L:
            t = np.arange(L)
            slots.append(tables[b, t // 16] * 16 + t % 16)
            kk.append(ks[b])
            vv.append(vs[b])
    if slots:
        s = np.concatenate(slots)
        bd.boost_kv_write(ctx, pool, layer, dev_i32(s), to_dev_u16(np.concatenate(kk)),
                          to_dev_u16(np.concatenate(vv)), len(s), stream())
        sync()


def make(rng, lens, H, Hq, nb, mb):
    tables = np.full((len(lens), mb), -1, np.int32)
    free = rng.permutation(nb)
    at = 0
    for b, L in enumerate(lens):
        n = (int(L) + 15) // 16
        tables[b, :n] = free[at:at + n]
        at += n
    assert at <= nb
    ks = [rand_kv(rng, (int(L), H, 128), 1) for L in lens]
    vs = [rand_kv(rng, (int(L), H, 128), 1) for L in lens]
    q = og.f32_to_bf16(rng.standard_normal((len(lens), Hq, 128)).astype(np.float32))
    return tables, ks, vs, q


def attention(ctx, pool, layer, q, tables, lens, dtype=bd.DTYPE_F32, scale=0.0,
              fn=bd.boost_paged_attn_decode):
    B, Hq, D = q.shape
    out = dev_f32(B, Hq, D) if dtype == bd.DTYPE_F32 else dev_u16(B, Hq, D)
    fn(ctx, pool, layer, to_dev_u16(q), B, Hq, dev_i32(tables), tables.shape[1], dev_i32(lens),
       scale, out, dtype, stream())
    sync()
    return out.cpu().numpy() if dtype == bd.DTYPE_F32 else host_u16(out)


def check(o, q, ks, vs, lens, scale=None, tokens=None):
    """Every row within the bound of its own sums.  A score is an fp32 sum of
    128 exact products (129 roundings with the scaling) of relative size 2^-24
    each, against sum |q k|; exp2 adds 2^-22 of its value, so a probability is
    off by e = 130 * 2^-24 * scale * max sum |q k| + 2^-22 (relative), the
    normalised one by twice that, the parts by at most 2^-16, the sums over L
    tokens and the merge by (L + 200) * 2^-24; all of them times max |v|."""
    B, Hq, D = q.shape
    H = ks[0].shape[1]
    G = Hq // H
    qf = og.bf16_to_f32(q).astype(np.float64)
    sc = 1 / np.sqrt(D) if scale is None else scale
    for b in range(B):
        keep = np.arange(int(lens[b])) if tokens is None else tokens[b]
        if len(keep) == 0:
            assert np.all(o[b] == 0)
            continue
        k, v = kv4.stored(ks[b][keep]), kv4.stored(vs[b][keep])
        for h in range(Hq):
            kh, vh = k[:, h // G], v[:, h // G]
            want = kv4.attend(qf[b, h][None], kh, vh, sc)[0]
            e = 130 * 2.0 ** -24 * sc * (np.abs(qf[b, h]) @ np.abs(kh).T).max() + 2.0 ** -22
            tol = np.abs(vh).max() * (2 * e + 2.0 ** -16 + (len(keep) + 200) * 2.0 ** -24)
            assert np.abs(o[b, h] - want).max() <= tol, (b, h)


LENS = np.array([1, 15, 16, 17, 31, 32, 33, 300, 1000, 0, 2049])


@pytest.mark.parametrize("Hq,H", [(8, 8), (16, 8), (6, 2), (32, 8), (10, 2), (12, 2), (7, 1), (64, 8)])
def test_attention_parity_and_placement_invariance(gpu_ctx, Hq, H):
    """Every number of query heads per KV head from 1 to 8, contexts around
    block borders, the same bits on every tier mode."""
    rng = np.random.default_rng(Hq)
    tables, ks, vs, q = make(rng, LENS, H, Hq, 1920, 130)
    outs = []
    for mode, M in ((bd.KV_ALL_HBM, 0), (bd.KV_LPP, 2), (bd.KV_ALL_HOST, 0)):
        pool = new_pool(gpu_ctx, H, Hq, 1920, M, mode, max_blocks=130)
        try:
            fill(gpu_ctx, pool, 0, LENS, tables, ks, vs)
            outs.append(attention(gpu_ctx, pool, 0, q, tables, LENS))
        finally:
            bd.boost_kv_pool_destroy(pool)
    check(outs[0], q, ks, vs, LENS)
    for o in outs[1:]:
        assert np.array_equal(o.view(np.uint32), outs[0].view(np.uint32))


@pytest.mark.parametrize("Hq,H,B,hi", [(32, 8, 70, 200), (8, 2, 300, 90), (32, 8, 1, 9000),
                                       (64, 8, 3, 2500), (4, 1, 1, 40000), (8, 8, 64, 130)])
def test_attention_sizes(gpu_ctx, Hq, H, B, hi):
    """Both item searches, one request to 300, short contexts to long ones,
    pools over several pages per head; bf16 output and the static scratch give
    the rounded and the same bits."""
    rng = np.random.default_rng(B + hi)
    lens = rng.integers(1, hi, size=B, endpoint=True)
    lens[0] = hi
    lens[3::9] = 0
    mb = (hi + 15) // 16
    nb = int(sum((int(x) + 15) // 16 for x in lens))
    tables, ks, vs, q = make(rng, lens, H, Hq, nb + 30, mb)
    pool = new_pool(gpu_ctx, H, Hq, nb + 30, max_batch=B, max_blocks=mb)
    try:
        fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
        o = attention(gpu_ctx, pool, 0, q, tables, lens)
        check(o, q, ks, vs, lens)
        ob = attention(gpu_ctx, pool, 0, q, tables, lens, bd.DTYPE_BF16)
        assert np.array_equal(ob, og.f32_to_bf16(o))
        on = attention(gpu_ctx, pool, 0, q, tables, lens, fn=bd.boost_paged_attn_decode_noalloc)
        assert np.array_equal(on.view(np.uint32), o.view(np.uint32))
        o2 = attention(gpu_ctx, pool, 0, q, tables, lens, scale=0.31)
        check(o2, q, ks, vs, lens, scale=float(np.float32(0.31)))
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_what_lies_behind_the_context_does_not_matter(gpu_ctx):
    """NaN and infinities behind the last token of a block, in blocks that the
    table does not name, and table entries past the context that name none."""
    rng = np.random.default_rng(5)
    H, Hq, mb = 4, 16, 12
    lens = np.array([1, 20, 33, 160, 0, 7])
    tables, ks, vs, q = make(rng, lens, H, Hq, 1920, mb)
    outs = []
    for poison in (False, True):
        pool = new_pool(gpu_ctx, H, Hq, 1920, max_batch=8, max_blocks=mb)
        try:
            t2 = tables.copy()
            if poison:
                n = 1920 * 16
                bad = np.full((n, H, 128), 0x7f80, np.uint16)
                bad[::2] = 0x7fc0
                bd.boost_kv_write(gpu_ctx, pool, 0, dev_i32(np.arange(n)), to_dev_u16(bad),
                                  to_dev_u16(bad), n, stream())
                for b, L in enumerate(lens):  # entries past the context
                    t2[b, (L + 15) // 16:] = rng.choice([-1, 5, 10 ** 9, -2 ** 31])
            fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
            outs.append(attention(gpu_ctx, pool, 0, q, t2, lens))
        finally:
            bd.boost_kv_pool_destroy(pool)
    check(outs[0], q, ks, vs, lens)
    assert np.array_equal(outs[0].view(np.uint32), outs[1].view(np.uint32))


def test_blocks_outside_the_pool_are_left_out(gpu_ctx):
    rng = np.random.default_rng(6)
    H, Hq, mb = 2, 8, 40
    lens = np.array([640, 100, 16, 33])
    tables, ks, vs, q = make(rng, lens, H, Hq, 1920, mb)
    pool = new_pool(gpu_ctx, H, Hq, 1920, max_batch=8, max_blocks=mb)
    try:
        fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
        bad = tables.copy()
        bad[0, [0, 7, 39]] = [-1, 1920, 2 ** 31 - 1]
        bad[1, 6] = -5           # the partial block
        bad[2, 0] = 1920         # nothing left
        tokens = []
        for b, L in enumerate(lens):
            t = np.arange(L)
            ok = (bad[b, t // 16] >= 0) & (bad[b, t // 16] < 1920)
            tokens.append(t[ok])
        o = attention(gpu_ctx, pool, 0, q, bad, lens)
        check(o, q, ks, vs, lens, tokens=tokens)
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_a_nan_in_the_context_shows(gpu_ctx):
    """A key group that is NaN makes its head's rows NaN, a value group its
    dims, and no other request's or head's row changes."""
    rng = np.random.default_rng(7)
    H, Hq, mb = 2, 8, 4
    lens = np.array([50, 50, 1])
    tables, ks, vs, q = make(rng, lens, H, Hq, 1920, mb)
    pool = new_pool(gpu_ctx, H, Hq, 1920, max_batch=8, max_blocks=mb)
    try:
        fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
        clean = attention(gpu_ctx, pool, 0, q, tables, lens)
        ks[0][20, 1, 5] = 0x7fc0
        vs[1][3, 0, 70] = 0x7f80
        ks[2][0, 0, 127] = 0xff80
        fill(gpu_ctx, pool, 0, lens, tables, ks, vs)
        o = attention(gpu_ctx, pool, 0, q, tables, lens)
        want = np.isnan(o)
        exp = np.zeros_like(want)
        exp[0, 4:] = True
        exp[1, :4, 64:96] = True
        exp[2, :4] = True
        assert np.array_equal(want, exp)
        assert np.array_equal(o[~exp], clean[~exp])
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_refusals(gpu_ctx):
    import torch
    for kw in (dict(fmt=2), dict(fmt=-1), dict(fmt=bd.KV_FP4, D=64)):
        with pytest.raises(bd.BoostError) as e:
            new_pool(gpu_ctx, 8, 32, 100, **kw)
        assert e.value.code == bd.EINVAL
    pool = new_pool(gpu_ctx, 2, 32, 100, max_batch=4, max_blocks=8)
    try:
        assert bd.boost_kv_pool_format(pool) == bd.KV_FP4
        buf = torch.zeros(4 * 32 * 128 + 8, dtype=torch.int16, device="cuda")
        i = torch.zeros(64, dtype=torch.int32, device="cuda")
        off = buf[1:]
        calls = [lambda: bd.boost_kv_read(gpu_ctx, pool, 1, i, buf, buf, 1, stream()),
                 lambda: bd.boost_kv_read(gpu_ctx, pool, 0, i, off, buf, 1, stream()),
                 lambda: bd.boost_kv_read(gpu_ctx, pool, 0, i, buf, off, 1, stream()),
                 lambda: bd.boost_kv_read(gpu_ctx, pool, 0, i, buf, buf, -1, stream()),
                 lambda: bd.boost_kv_read(gpu_ctx, pool, 0, 0, buf, buf, 1, stream()),
                 lambda: bd.boost_kv_write(gpu_ctx, pool, 0, i, off, buf, 1, stream()),
                 lambda: bd.boost_kv_append(gpu_ctx, pool, 0, i, 8, i, buf, off, 1, stream()),
                 lambda: bd.boost_kv_pages(pool, 1, 0), lambda: bd.boost_kv_pages(pool, 0, 2),
                 # 16 query heads per KV head
                 lambda: bd.boost_paged_attn_decode(gpu_ctx, pool, 0, buf, 1, 32, i, 8, i, 0.0, buf,
                                                    bd.DTYPE_BF16, stream())]
        for c in calls:
            with pytest.raises(bd.BoostError) as e:
                c()
            assert e.value.code == bd.EINVAL
        bd.boost_kv_read(gpu_ctx, pool, 0, i, buf, buf, 0, stream())  # nothing to do
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_pages_are_the_pool(gpu_ctx):
    """The pages' addresses: consecutive in HBM, K then V, layer by layer; a
    block written through kv_write is found there (bf16)."""
    import torch
    H, D = 2, 128
    pool = new_pool(gpu_ctx, H, H, 512, layers=2, fmt=bd.KV_BF16)
    try:
        base = [bd.boost_kv_pages(pool, l, w) for l in (0, 1) for w in (0, 1)]
        flat = np.concatenate(base)
        assert len(flat) == 4 * H and np.all(np.diff(flat) == bd.PAGE_BYTES)

        class Memory:
            __cuda_array_interface__ = {"data": (int(flat[0]), False), "typestr": "<i2", "version": 2,
                                        "shape": (2, 2, H, 512, 16, D)}
        view = torch.as_tensor(Memory(), device="cuda")
        rng = np.random.default_rng(8)
        k, v = rand_kv(rng, (1, H, D)), rand_kv(rng, (1, H, D))
        bd.boost_kv_write(gpu_ctx, pool, 1, dev_i32([37 * 16 + 3]), to_dev_u16(k), to_dev_u16(v), 1,
                          stream())
        sync()
        assert np.array_equal(host_u16(view[1, 0, :, 37, 3].contiguous()), k[0])
        assert np.array_equal(host_u16(view[1, 1, :, 37, 3].contiguous()), v[0])
        assert int((view != 0).sum()) == np.count_nonzero(k) + np.count_nonzero(v)
    finally:
        bd.boost_kv_pool_destroy(pool)
