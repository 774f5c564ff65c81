"""GPU parity of block summaries, selection and attention over selected blocks."""
import numpy as np
import pytest

from oracle import gemv as og
from oracle import kv4
from oracle import select as osel
from paper_2609_13592_amd import binding as bd
from tests.gpu_util import dev_f32, dev_u16, host_u16, stream, sync, to_dev_u16

pytestmark = pytest.mark.gpu


def dev_i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def rand_u16(rng, shape):
    return og.f32_to_bf16(rng.standard_normal(shape).astype(np.float32))


class Cache:
    """A pool with requests of `lens` tokens at random blocks, and what its
    keys and values stand for."""

    def __init__(self, ctx, rng, fmt, lens, H, Hq, mode=bd.KV_ALL_HBM, M=0, extra=20, mb=None,
                 layers=1, layer=0):
        self.ctx, self.fmt, self.H, self.Hq, self.layer = ctx, fmt, H, Hq, layer
        self.lens = np.asarray(lens)
        need = [(int(L) + 15) // 16 for L in self.lens]
        self.mb = mb or max(1, max(need))
        nb = sum(need) + extra
        self.pool = bd.boost_kv_pool_create_format(
            ctx, fmt, layers, H, 128, nb, M, mode, q_heads=Hq, max_batch=len(need),
            max_blocks_per_seq=self.mb)
        self.nb = bd.boost_kv_pool_info(self.pool)["nb_pool"]
        ids = rng.permutation(self.nb)[:sum(need)]
        self.tables = np.full((len(need), self.mb), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.tables[b, :n] = ids[at:at + n]
            at += n
        self.k = [rand_u16(rng, (int(L), H, 128)) for L in self.lens]
        self.v = [rand_u16(rng, (int(L), H, 128)) for L in self.lens]
        self.q = rand_u16(rng, (len(need), Hq, 128))

    def write(self, b=None):
        slots, kk, vv = [], [], []
        for i, L in enumerate(self.lens):
            if L and (b is None or i == b):
                t = np.arange(int(L))
                slots.append(self.tables[i, t // 16] * 16 + t % 16)
                kk.append(self.k[i])
                vv.append(self.v[i])
        if slots:
            s = np.concatenate(slots)
            bd.boost_kv_write(self.ctx, self.pool, self.layer, dev_i32(s), to_dev_u16(np.concatenate(kk)),
                              to_dev_u16(np.concatenate(vv)), len(s), stream())
            sync()

    def meaning(self, x):
        return kv4.stored(x) if self.fmt == bd.KV_FP4 else og.bf16_to_f32(x).astype(np.float64)

    def index(self, starts=None, ends=None, hint=None):
        ends = self.lens if ends is None else ends
        starts = np.zeros_like(ends) if starts is None else starts
        bd.boost_kv_index_update(self.ctx, self.pool, self.layer, dev_i32(self.tables), self.mb,
                                 dev_i32(starts), dev_i32(ends), len(self.lens),
                                 hint or max(1, int((ends - starts).max())), stream())

    def select(self, top, first=0, last=0, tables=None, q=None):
        import torch
        B = len(self.lens)
        q = self.q if q is None else q
        sc = torch.full((B, self.H, self.mb), 77.0, dtype=torch.float32, device="cuda")
        sel = torch.full((B, self.H, top), 99, dtype=torch.int32, device="cuda")
        bd.boost_kv_select(self.ctx, self.pool, self.layer, to_dev_u16(q), B, q.shape[1],
                           dev_i32(self.tables if tables is None else tables), self.mb,
                           dev_i32(self.lens), top, first, last, sc, sel, stream())
        sync()
        return sc.cpu().numpy(), sel.cpu().numpy()

    def attend(self, sel, dtype=bd.DTYPE_F32, tables=None):
        B = len(self.lens)
        out = dev_f32(B, self.Hq, 128) if dtype == bd.DTYPE_F32 else dev_u16(B, self.Hq, 128)
        bd.boost_sparse_attn_decode(self.ctx, self.pool, self.layer, to_dev_u16(self.q), B, self.Hq,
                                    dev_i32(self.tables if tables is None else tables), self.mb,
                                    dev_i32(self.lens), dev_i32(sel), sel.shape[2], 0.0, out, dtype,
                                    stream())
        sync()
        return out.cpu().numpy() if dtype == bd.DTYPE_F32 else host_u16(out)

    def check_selection(self, top, first=0, last=0):
        sc, sel = self.select(top, first, last)
        for b, L in enumerate(self.lens):
            n = (int(L) + 15) // 16
            want = np.zeros((self.H, 0)) if n == 0 else osel.scores(
                og.bf16_to_f32(self.q[b]).astype(np.float64), self.meaning(self.k[b]))
            assert np.array_equal(sc[b, :, :n], want), b
            assert np.all(sc[b, :, n:] == 77.0)  # past the context: as it was
            assert np.array_equal(sel[b], osel.select(want, top, first, last)), b
        return sel

    def check_attention(self, o, sel, lens=None, skip=None):
        """Within the bound of the row's own sums: a score is an fp32 sum of
        128 exact products and a scaling (130 roundings of 2^-24 against
        sum |q k|), exp2 adds 2^-22, a normalised probability twice that; a
        4-bit pool's parts 2^-16; sums of N tokens and the merge
        (N + 200) * 2^-24."""
        G = self.Hq // self.H
        qf = og.bf16_to_f32(self.q).astype(np.float64)
        for b, L in enumerate(self.lens):
            k, v = self.meaning(self.k[b]), self.meaning(self.v[b])
            n = (int(L) + 15) // 16
            for h in range(self.Hq):
                t = []
                for i in sel[b, h // G][:n]:
                    if 0 <= i < n and not (skip is not None and (b, i) in skip):
                        t += list(range(16 * i, min(16 * i + 16, int(L))))
                if not t:
                    assert np.all(o[b, h] == 0)
                    continue
                kh, vh = k[t, h // G], v[t, h // G]
                want = kv4.attend(qf[b, h][None], kh, vh)[0]
                e = 130 * 2.0 ** -24 / np.sqrt(128) * (np.abs(qf[b, h]) @ np.abs(kh).T).max() + 2.0 ** -22
                tol = np.abs(vh).max() * (2 * e + 2.0 ** -16 + (len(t) + 200) * 2.0 ** -24)
                assert np.abs(o[b, h] - want).max() <= tol, (b, h)

    def close(self):
        bd.boost_kv_pool_destroy(self.pool)


FORMATS = [bd.KV_BF16, bd.KV_FP4]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hq", [(8, 32), (2, 16), (1, 1), (5, 10)])
def test_summaries_selection_and_attention(gpu_ctx, fmt, H, Hq):
    """From no context to long ones, blocks around every border, lists shorter
    and longer than the context."""
    rng = np.random.default_rng(Hq)
    c = Cache(gpu_ctx, rng, fmt, [1, 15, 16, 17, 0, 300, 1000, 4700], H, Hq)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        bd.boost_kv_index_enable(c.pool)  # again: no-op
        c.index()
        for top, first, last in ((1, 0, 0), (1, 1, 0), (1, 0, 1), (7, 1, 2), (64, 0, 0), (400, 2, 2)):
            sel = c.check_selection(top, first, last)
            o = c.attend(sel)
            c.check_attention(o, sel)
            assert np.array_equal(c.attend(sel, bd.DTYPE_BF16), og.f32_to_bf16(o))
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H,Hq", [(8, 32), (8, 8), (8, 64), (10, 20)])
def test_whole_lists_of_many_heads(gpu_ctx, fmt, H, Hq):
    """Enough heads to fill the card with a workgroup for each list: rows that
    select nothing, requests without tokens, partial blocks anywhere."""
    rng = np.random.default_rng(H + Hq)
    lens = rng.integers(1, 700, size=50, endpoint=True)
    lens[3] = lens[49] = 0
    c = Cache(gpu_ctx, rng, fmt, lens, H, Hq)
    try:
        c.write()
        n = (lens + 15) // 16
        sel = np.full((50, H, 40), -1, np.int32)
        for b in range(50):
            for h in range(H):
                m = min(40, int(n[b]))
                sel[b, h, :m] = np.sort(rng.permutation(int(n[b]))[:m])
        sel[7], sel[8, 1] = -1, -1
        sel[9, 0, 1:] = -1
        o = c.attend(sel)
        c.check_attention(o, sel)
        assert np.array_equal(c.attend(sel, bd.DTYPE_BF16), og.f32_to_bf16(o))
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B", [3, 70])
def test_lengths_past_the_table(gpu_ctx, fmt, B):
    """Contexts as long as an int32 goes end with the table, in every call."""
    rng = np.random.default_rng(B)
    c = Cache(gpu_ctx, rng, fmt, [480] * B, 2, 8)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        sel = c.check_selection(12, 1, 1)

        def dense():
            o = dev_f32(B, 8, 128)
            bd.boost_paged_attn_decode(gpu_ctx, c.pool, 0, to_dev_u16(c.q), B, 8, dev_i32(c.tables), c.mb,
                                       dev_i32(c.lens), 0.0, o, bd.DTYPE_F32, stream())
            sync()
            return o.cpu().numpy()
        want = (c.attend(sel), dense())
        c.lens = np.array([2 ** 31 - 1 - i % 20 for i in range(B)])
        c.index(hint=480)
        assert np.array_equal(c.select(12, 1, 1)[1], sel)
        for a, b in zip((c.attend(sel), dense()), want):
            assert np.array_equal(a, b)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_placement_does_not_change_a_bit(gpu_ctx, fmt):
    outs = []
    for mode, M in ((bd.KV_ALL_HBM, 0), (bd.KV_LPP, 2), (bd.KV_ALL_HOST, 0)):
        c = Cache(gpu_ctx, np.random.default_rng(3), fmt, [900, 33, 2000], 8, 32, mode, M)
        try:
            c.write()
            bd.boost_kv_index_enable(c.pool)
            c.index()
            sc, sel = c.select(20, 1, 1)
            outs.append((sc, sel, c.attend(sel)))
        finally:
            c.close()
    for o in outs[1:]:
        for a, b in zip(o, outs[0]):
            assert np.array_equal(a, b)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,hi", [(70, 400), (1, 70000), (300, 60)])
def test_sizes(gpu_ctx, fmt, B, hi):
    """Both item searches of attention; thousands of blocks in one selection."""
    rng = np.random.default_rng(B)
    lens = rng.integers(1, hi, size=B, endpoint=True)
    lens[0] = hi
    lens[2::7] = 0
    H, Hq = (2, 8) if hi > 1000 else (4, 16)
    c = Cache(gpu_ctx, rng, fmt, lens, H, Hq)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        sel = c.check_selection(33, 1, 1)
        c.check_attention(c.attend(sel), sel)
        c.check_selection(257, 0, 3)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [200, 256, 257, 512, 513, 2048, 5000, 8193, 32769, 70001])
def test_selection_over_tables_of_every_width(gpu_ctx, fmt, n):
    """Tables that name each of 300 blocks (and some that are none) many times:
    many equal scores, and every way a workgroup holds the keys."""
    import torch
    rng = np.random.default_rng(n)
    H, Hq = 2, 8
    c = Cache(gpu_ctx, rng, fmt, [4800], H, Hq)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        one = osel.scores(og.bf16_to_f32(c.q[0]).astype(np.float64), c.meaning(c.k[0]))  # [H, 300]
        at = rng.integers(0, 300, size=n)
        table = c.tables[0, at][None].copy()
        want = one[:, at]
        none = rng.random(n) < 0.01
        table[0, none], want[:, none] = -1, -np.inf
        for top, first, last in ((1, 0, 0), (5, 2, 3), (300, 1, 2), (n // 2, 0, 1), (n - 1, 1, 0)):
            sc = torch.full((1, H, n), 77.0, dtype=torch.float32, device="cuda")
            sel = torch.full((1, H, top), 99, dtype=torch.int32, device="cuda")
            bd.boost_kv_select(gpu_ctx, c.pool, 0, to_dev_u16(c.q), 1, Hq, dev_i32(table), n,
                               dev_i32([16 * n - 5]), top, first, last, sc, sel, stream())
            sync()
            assert np.array_equal(sc.cpu().numpy()[0], want)
            assert np.array_equal(sel.cpu().numpy()[0], osel.select(want, top, first, last)), top
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_updates_block_by_block(gpu_ctx, fmt):
    """A context that grows: updates of one token, of a few, of ranges that
    the hint is too small for, leave the same summaries as one over all; other
    requests' and layers' summaries stay as they are."""
    rng = np.random.default_rng(4)
    c = Cache(gpu_ctx, rng, fmt, [250, 100], 4, 8, layers=2, layer=1)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        full = c.lens
        for end in (1, 2, 16, 17, 40, 41, 250):
            ends = np.minimum(full, end)
            c.index(np.array([{1: 0, 2: 1, 16: 2, 17: 16, 40: 17, 41: 40, 250: 41}[end]] * 2), ends,
                    hint=1)
            c.lens = ends
            keep = c.k
            c.k = [x[:n] for x, n in zip(keep, ends)]
            c.check_selection(3, 1, 1)
            c.k, c.lens = keep, full
        # a new range of request 0 alone, its keys having changed below it too
        before, _ = c.select(4)
        c.k[0][:] = rand_u16(rng, c.k[0].shape)
        c.write(0)
        c.index(np.array([48, 50]), np.array([80, 50]))
        after, _ = c.select(4)
        changed = (before != after).any(1)
        assert np.all(changed[0, 3:5]) and not changed[0, :3].any() and not changed[0, 5:].any()
        assert not changed[1].any()
        c.layer = 0  # nothing was ever summarised there
        sc, _ = c.select(4)
        assert np.all(sc[0, :, :16] == 0)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_ties_take_the_lowest_index(gpu_ctx, fmt):
    """Equal blocks have equal scores; a zero query makes all of them equal."""
    rng = np.random.default_rng(5)
    c = Cache(gpu_ctx, rng, fmt, [1600, 1601, 4096], 2, 4)
    try:
        for b in range(3):
            one = rand_u16(rng, (16, 2, 128))
            n = len(c.k[b])
            c.k[b][:] = np.tile(one, (n // 16 + 1, 1, 1))[:n]
        c.q[1] = 0
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        for top, first, last in ((5, 0, 0), (50, 1, 3), (99, 0, 1), (255, 0, 0)):
            sel = c.check_selection(top, first, last)
        assert sel[2].tolist() == [list(range(255))] * 2
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_values_that_are_not_finite(gpu_ctx, fmt):
    """A key that is NaN or infinite: its block is selected (score +inf); a
    query head that is: it counts as 0.  Behind the context neither matters."""
    rng = np.random.default_rng(6)
    c = Cache(gpu_ctx, rng, fmt, [500, 500, 250], 2, 8)
    try:
        bad = np.full((c.nb * 16, 2, 128), 0x7fc0, np.uint16)
        bad[::3] = 0xff80
        bd.boost_kv_write(gpu_ctx, c.pool, 0, dev_i32(np.arange(c.nb * 16)), to_dev_u16(bad),
                          to_dev_u16(bad), c.nb * 16, stream())
        c.k[0][100, 1, 9] = 0x7fc0
        c.k[0][499, 0, 0] = 0x7f80
        c.k[1][20, :, 127] = 0xff80
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        c.q[1, 3, 50] = 0x7fc0
        c.q[2, 0:4, 1] = 0x7f80
        sel = c.check_selection(3)
        assert 6 in sel[0, 1] and 31 in sel[0, 0] and 1 in sel[1, 0]
        c.q[1:] = rand_u16(rng, c.q[1:].shape)
        sel = np.tile(np.arange(20, dtype=np.int32), (3, 2, 1))  # clean blocks of request 2
        o = c.attend(sel)
        assert np.all(np.isfinite(o[2]))
        dense = dev_f32(3, 8, 128)
        bd.boost_paged_attn_decode(gpu_ctx, c.pool, 0, to_dev_u16(c.q), 3, 8, dev_i32(c.tables), c.mb,
                                   dev_i32(c.lens), 0.0, dense, bd.DTYPE_F32, stream())
        sync()
        assert np.all(np.isfinite(dense[2].cpu().numpy()))
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_lists_as_they_may_come(gpu_ctx, fmt):
    """Entries in any order, twice, -1 between, past the context and the
    table, extreme; a partial block in the middle; a list of nothing."""
    rng = np.random.default_rng(7)
    c = Cache(gpu_ctx, rng, fmt, [330, 330, 330, 20, 330], 2, 8, mb=30)
    try:
        c.write()
        sel = np.full((5, 2, 25), -1, np.int32)
        sel[0, :, :21] = [rng.permutation(21) for _ in range(2)]          # all, shuffled
        sel[1, 0, :6] = [20, 3, 3, 7, 20, 3]                              # twice, the partial one too
        sel[1, 1, :9] = [-1, 5, 21, 29, 30, -2 ** 31, 2 ** 31 - 1, 20, 0]
        sel[2, 1, 0] = 20                                                 # the partial block alone
        sel[3, :, :4] = [0, 1, 0, 1]     # only two entries of a two-block context count
        sel[4, 0, 20], sel[4, 0, 21] = 4, 5  # entry 21 is past the 21 that count
        o = c.attend(sel)
        c.check_attention(o, sel)
        assert np.all(o[2, :4] == 0)
        assert np.array_equal(c.attend(sel, bd.DTYPE_BF16), og.f32_to_bf16(o))
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_outside_the_pool(gpu_ctx, fmt):
    """Table entries that name no block: score -inf, attention leaves them out."""
    rng = np.random.default_rng(8)
    c = Cache(gpu_ctx, rng, fmt, [640, 100], 2, 8)
    try:
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        t = c.tables.copy()
        t[0, [0, 5, 39]] = [-1, c.nb, 2 ** 31 - 1]
        t[1, 6] = -7
        clean, _ = c.select(4)
        c.tables, keep = t, c.tables
        c.index()  # skips them
        c.tables = keep
        sc, sel = c.select(37, tables=t)
        assert np.all(sc[0][:, [0, 5, 39]] == -np.inf) and np.all(sc[1][:, 6] == -np.inf)
        ok = np.ones((2, c.mb), bool)
        ok[0, [0, 5, 39]] = ok[1, 6] = False
        n = [40, 7]
        for b in range(2):
            assert np.array_equal(sc[b][:, :n[b]][:, ok[b, :n[b]]], clean[b][:, :n[b]][:, ok[b, :n[b]]])
        assert not np.isin([0, 5, 39], sel[0]).any()
        sel, _ = np.broadcast_arrays(np.arange(40, dtype=np.int32), np.zeros((2, 2, 40)))
        o = c.attend(sel, tables=t)
        c.check_attention(o, sel, skip={(0, 0), (0, 5), (0, 39), (1, 6)})
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_every_block_gives_the_dense_result(gpu_ctx, fmt):
    rng = np.random.default_rng(9)
    c = Cache(gpu_ctx, rng, fmt, [1000, 5, 333], 8, 32)
    try:
        c.write()
        sel = np.tile(np.arange(c.mb, dtype=np.int32), (3, 8, 1))
        o = c.attend(sel)
        dense = dev_f32(3, 32, 128)
        bd.boost_paged_attn_decode(gpu_ctx, c.pool, 0, to_dev_u16(c.q), 3, 32, dev_i32(c.tables), c.mb,
                                   dev_i32(c.lens), 0.0, dense, bd.DTYPE_F32, stream())
        sync()
        # both within their bound of the exact row (check_attention): twice that
        assert np.abs(o - dense.cpu().numpy()).max() < 1e-3
        c.check_attention(o, sel)
        c.check_attention(dense.cpu().numpy(), sel)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_offsets_past_32_bits(gpu_ctx, fmt):
    """Tensors of more than 4 GiB each (two layers, the second used): the last
    blocks of the pool written, read, summarised, copied and attended to."""
    rng = np.random.default_rng(11)
    big = 160000 if fmt == bd.KV_BF16 else 540000
    c = Cache(gpu_ctx, rng, fmt, [900, 33, 1], 8, 32, extra=big, layers=2, layer=1)
    try:
        pages = bd.boost_kv_pages(c.pool, 1, 0)
        assert int(pages[-1]) - int(pages[0]) > 2 ** 32
        need = [(int(L) + 15) // 16 for L in c.lens]
        ids = c.nb - 1 - rng.permutation(sum(need))
        for b in range(3):
            at = sum(need[:b])
            c.tables[b, :need[b]] = ids[at:at + need[b]]
        c.write()
        bd.boost_kv_index_enable(c.pool)
        c.index()
        sel = c.check_selection(20, 1, 1)
        whole = np.tile(np.arange(c.mb, dtype=np.int32), (3, 8, 1))
        o, dense = c.attend(sel), dev_f32(3, 32, 128)
        c.check_attention(o, sel)

        def attend_all():
            bd.boost_paged_attn_decode(gpu_ctx, c.pool, 1, to_dev_u16(c.q), 3, 32, dev_i32(c.tables), c.mb,
                                       dev_i32(c.lens), 0.0, dense, bd.DTYPE_F32, stream())
            sync()
            return dense.cpu().numpy()
        d = attend_all()
        c.check_attention(d, whole)
        for b, L in enumerate(c.lens):
            t = np.arange(int(L))
            k, v = dev_u16(int(L), 8, 128), dev_u16(int(L), 8, 128)
            bd.boost_kv_read(gpu_ctx, c.pool, 1, dev_i32(c.tables[b, t // 16] * 16 + t % 16), k, v, int(L),
                             stream())
            sync()
            assert np.array_equal(og.bf16_to_f32(host_u16(k)).astype(np.float64), c.meaning(c.k[b]))
            assert np.array_equal(og.bf16_to_f32(host_u16(v)).astype(np.float64), c.meaning(c.v[b]))
        # the same blocks elsewhere: every bit the same
        to = c.nb - 1000 - ids[::-1]
        to = to - to.min() + c.nb // 2
        bd.boost_kv_copy_blocks(gpu_ctx, c.pool, 0, 2, ids, to, len(ids), stream())
        new = dict(zip(ids.tolist(), to.tolist()))
        c.tables = np.where(c.tables >= 0, np.vectorize(lambda i: new.get(i, -1))(c.tables), -1).astype(np.int32)
        assert np.array_equal(c.check_selection(20, 1, 1), sel)
        assert np.array_equal(c.attend(sel), o)
        assert np.array_equal(attend_all(), d)
    finally:
        c.close()


def test_two_pools_on_two_streams(gpu_ctx):
    """A pool of each format, each on a stream of its own, their calls in turn
    and nothing waited for in between: the results of either one alone."""
    import torch
    cs, want, runs = [], [], []
    try:
        for fmt in FORMATS:
            c = Cache(gpu_ctx, np.random.default_rng(20 + fmt), fmt, [3000, 17, 640, 0], 8, 32)
            cs.append(c)
            c.write()
            bd.boost_kv_index_enable(c.pool)
            c.index()
            _, sel = c.select(24, 1, 1)
            want.append((sel, c.attend(sel)))
        for c in cs:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                t, ln, q = dev_i32(c.tables), dev_i32(c.lens), to_dev_u16(c.q)
                sc = torch.zeros((4, 8, c.mb), dtype=torch.float32, device="cuda")
                sel = torch.full((4, 8, 24), 99, dtype=torch.int32, device="cuda")
                out = torch.full((4, 32, 128), float("nan"), device="cuda")
                zero = dev_i32([0] * 4)
            runs.append((c, st, t, ln, q, sc, sel, out, zero))
        sync()
        for _ in range(20):
            for c, st, t, ln, q, sc, sel, out, zero in runs:
                s = st.cuda_stream
                bd.boost_kv_index_update(gpu_ctx, c.pool, 0, t, c.mb, zero, ln, 4, 3000, s)
                bd.boost_kv_select(gpu_ctx, c.pool, 0, q, 4, 32, t, c.mb, ln, 24, 1, 1, sc, sel, s)
                bd.boost_sparse_attn_decode(gpu_ctx, c.pool, 0, q, 4, 32, t, c.mb, ln, sel, 24, 0.0, out,
                                            bd.DTYPE_F32, s)
        sync()
        for r, (sel, o) in zip(runs, want):
            assert np.array_equal(r[6].cpu().numpy(), sel)
            assert np.array_equal(r[7].cpu().numpy(), o)
    finally:
        for c in cs:
            c.close()


def test_wide_groups_select(gpu_ctx):
    """Selection takes up to 16 query heads per KV head."""
    rng = np.random.default_rng(10)
    for H, Hq in ((2, 32), (1, 11)):
        c = Cache(gpu_ctx, rng, bd.KV_BF16, [700, 50], H, Hq)
        try:
            c.write()
            bd.boost_kv_index_enable(c.pool)
            c.index()
            c.check_selection(9, 1, 1)
        finally:
            c.close()


def test_refusals(gpu_ctx):
    import torch
    pool = bd.boost_kv_pool_create(gpu_ctx, 1, 2, 128, 100, 0, bd.KV_ALL_HBM, q_heads=8, max_batch=4,
                                   max_blocks_per_seq=8)
    small = bd.boost_kv_pool_create(gpu_ctx, 1, 2, 64, 100, 0, bd.KV_ALL_HBM, q_heads=8, max_batch=4,
                                    max_blocks_per_seq=8)
    try:
        z = torch.zeros(4 * 8 * 128 + 8, dtype=torch.int32, device="cuda")
        off = z.view(torch.int16)[1:]

        def sel(pool=pool, q=z, layer=0, B=4, Hq=8, mb=8, top=4, first=1, last=1, sc=z, out=z):
            bd.boost_kv_select(gpu_ctx, pool, layer, q, B, Hq, z, mb, z, top, first, last, sc, out, stream())

        def att(q=z, layer=0, B=4, Hq=8, mb=8, s=z, top=4, dt=bd.DTYPE_F32):
            bd.boost_sparse_attn_decode(gpu_ctx, pool, layer, q, B, Hq, z, mb, z, s, top, 0.0, z, dt,
                                        stream())

        def upd(layer=0, B=4, mb=8, tok=1, pool=pool):
            bd.boost_kv_index_update(gpu_ctx, pool, layer, z, mb, z, z, B, tok, stream())

        def refused(f, **kw):
            with pytest.raises(bd.BoostError) as e:
                f(**kw)
            assert e.value.code == bd.EINVAL, kw

        refused(sel), refused(upd)  # no summaries yet
        refused(lambda: bd.boost_kv_index_enable(small))
        bd.boost_kv_index_enable(pool)
        sel(), upd(), att()
        for kw in (dict(layer=1), dict(layer=-1), dict(B=0), dict(Hq=7), dict(Hq=0), dict(Hq=34), dict(mb=0),
                   dict(top=0), dict(first=-1), dict(last=-1), dict(first=3, last=2), dict(q=off),
                   dict(q=0), dict(sc=0), dict(out=0), dict(first=2 ** 31 - 1, last=2 ** 31 - 1)):
            refused(sel, **kw)
        for kw in (dict(layer=1), dict(B=0), dict(mb=0), dict(tok=0)):
            refused(upd, **kw)
        for kw in (dict(layer=1), dict(B=5), dict(Hq=4), dict(mb=9), dict(top=0), dict(s=0), dict(dt=7),
                   dict(q=off)):
            refused(att, **kw)
    finally:
        sync()
        bd.boost_kv_pool_destroy(pool)
        bd.boost_kv_pool_destroy(small)


def test_lists_and_batches_too_long(gpu_ctx):
    import torch
    pool = bd.boost_kv_pool_create(gpu_ctx, 1, 2, 128, 100, 0, bd.KV_ALL_HBM, q_heads=8, max_batch=1,
                                   max_blocks_per_seq=8)
    try:
        bd.boost_kv_index_enable(pool)
        z = torch.zeros(8 * 128, dtype=torch.int32, device="cuda")
        for f in (lambda: bd.boost_kv_select(gpu_ctx, pool, 0, z, 65536, 8, z, 8, z, 4, 0, 0, z, z, stream()),
                  lambda: bd.boost_kv_index_update(gpu_ctx, pool, 0, z, 8, z, z, 65536, 1, stream())):
            with pytest.raises(bd.BoostError) as e:
                f()
            assert e.value.code == bd.EINVAL
        for top in (2 ** 27 + 1, 2 ** 31 - 1):
            for f in (lambda: bd.boost_kv_select(gpu_ctx, pool, 0, z, 1, 8, z, 8, z, top, 0, 0, z, z, stream()),
                      lambda: bd.boost_sparse_attn_decode(gpu_ctx, pool, 0, z, 1, 8, z, 8, z, z, top, 0.0, z,
                                                          bd.DTYPE_F32, stream())):
                with pytest.raises(bd.BoostError) as e:
                    f()
                assert e.value.code == bd.EINVAL
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_decode_step_captured_and_replayed(gpu_ctx, fmt):
    """Append, summary, selection and attention in one graph, replayed while
    the inputs change, against the same calls made directly."""
    import torch
    rng = np.random.default_rng(11)
    lens = np.array([700, 31, 4000])
    H, Hq, top = 8, 32, 12
    caches = [Cache(gpu_ctx, np.random.default_rng(12), fmt, lens + 8, H, Hq) for _ in range(2)]
    try:
        state = []
        for c in caches:
            c.lens = lens.copy()
            c.k, c.v = [x[:n] for x, n in zip(c.k, lens)], [x[:n] for x, n in zip(c.v, lens)]
            c.write()
            bd.boost_kv_index_enable(c.pool)
            c.index()
            state.append(dict(k=dev_u16(3, H, 128), v=dev_u16(3, H, 128), q=dev_u16(3, Hq, 128),
                              t=dev_i32(c.tables), pos=dev_i32(lens), ends=dev_i32(lens + 1),
                              sc=dev_f32(3, H, c.mb), sel=dev_i32(np.zeros((3, H, top))),
                              o=dev_f32(3, Hq, 128)))
        sync()

        def step(c, s, st):
            bd.boost_kv_append(gpu_ctx, c.pool, 0, s["t"], c.mb, s["pos"], s["k"], s["v"], 3, st)
            bd.boost_kv_index_update(gpu_ctx, c.pool, 0, s["t"], c.mb, s["pos"], s["ends"], 3, 1, st)
            bd.boost_kv_select(gpu_ctx, c.pool, 0, s["q"], 3, Hq, s["t"], c.mb, s["ends"], top, 1, 2,
                               s["sc"], s["sel"], st)
            bd.boost_sparse_attn_decode(gpu_ctx, c.pool, 0, s["q"], 3, Hq, s["t"], c.mb, s["ends"],
                                        s["sel"], top, 0.0, s["o"], bd.DTYPE_F32, st)

        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            step(caches[0], state[0], torch.cuda.current_stream().cuda_stream)
        for turn in range(4):
            new = {n: to_dev_u16(rand_u16(rng, tuple(state[0][n].shape))) for n in ("k", "v", "q")}
            for s in state:
                for n, x in new.items():
                    s[n].copy_(x)
                s["pos"].copy_(dev_i32(lens + turn))
                s["ends"].copy_(dev_i32(lens + turn + 1))
            graph.replay()
            step(caches[1], state[1], stream())
            sync()
            assert torch.equal(state[0]["sel"], state[1]["sel"])
            assert torch.equal(state[0]["o"], state[1]["o"])
            assert bool(torch.isfinite(state[0]["o"]).all()) and float(state[0]["o"].abs().max()) > 0
    finally:
        for c in caches:
            c.close()
