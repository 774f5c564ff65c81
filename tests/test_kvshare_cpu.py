"""Shared, truncated and compacted blocks of the KV allocator (plan-only pools)
against a reference that keeps sets of holders."""
import numpy as np
import pytest
from hypothesis import given, settings, strategies as st

from oracle import kvpool as okv
from paper_2609_13592_amd import binding as bd


@pytest.fixture(scope="module")
def plan_ctx():
    ctx = bd.boost_init(-1)
    yield ctx
    bd.boost_shutdown(ctx)


class Sharing(okv.DSRAllocator):
    """The allocator's reference with blocks that several requests hold."""

    def holders(self, b):
        return sum(b in bl for bl in self.req_blocks.values())

    def _release(self, b):
        if self.holders(b) == 0:
            self._push(b)

    def free_request(self, rid):
        for b in self.req_blocks.pop(rid):
            self._release(b)
        del self.req_type[rid]

    def fork(self, parent, child, n):
        if parent not in self.req_type or child in self.req_type or \
                not 1 <= n <= len(self.req_blocks[parent]):
            return bd.EINVAL
        self.req_type[child] = self.req_type[parent]
        self.req_blocks[child] = self.req_blocks[parent][:n]
        return None

    def unshare(self, rid, i):
        if rid not in self.req_type or i >= len(self.req_blocks[rid]):
            return bd.EINVAL
        b = self.req_blocks[rid][i]
        if self.holders(b) == 1:
            return b, b
        if self.n_free() == 0:
            return bd.EAGAIN
        t = self.req_type[rid]
        if not self.free[t]:
            t = 1 - t
        self.req_type[rid] = t
        self.req_blocks[rid][i] = self._pop(t)
        return b, self.req_blocks[rid][i]

    def truncate(self, rid, n):
        if rid not in self.req_type or n > len(self.req_blocks[rid]):
            return bd.EINVAL
        while len(self.req_blocks[rid]) > n:
            self._release(self.req_blocks[rid].pop())
        return None

    def compact(self, limit):
        moves = []
        for t in (okv.LOCAL, okv.SHH):
            while len(moves) < limit:
                used = sorted({b for bl in self.req_blocks.values() for b in bl
                               if (b in self.shh_set) == (t == okv.SHH)})
                if not used or not self.free[t] or self.free[t][0] > used[-1]:
                    break
                s, d = used[-1], self._pop(t)
                for bl in self.req_blocks.values():
                    bl[:] = [d if b == s else b for b in bl]
                self._push(s)
                moves.append((s, d))
        return moves

    def used(self):
        return {b for bl in self.req_blocks.values() for b in bl}


def code(f, *args):
    try:
        return f(*args)
    except bd.BoostError as e:
        return e.code


def replay(plan_ctx, nb, H, M, events, fmt=bd.KV_BF16):
    pool = bd.boost_kv_pool_create_format(plan_ctx, fmt, 2, H, 128, nb, M, q_heads=H)
    try:
        n_pool = bd.boost_kv_pool_info(pool)["nb_pool"]
        hh = np.array([bd.boost_kv_block_host_heads(pool, b) for b in range(n_pool)])
        hi = hh.max()
        shh = np.flatnonzero(hh == hi) if hi != hh.min() else []
        a = Sharing(shh, sorted(set(range(n_pool)) - set(shh)))
        for kind, x, y, n in events:
            ids = sorted(a.req_type)
            x, y = (ids[v % len(ids)] if ids and v < 20 else v for v in (x, y))
            if kind == "alloc":
                assert bd.boost_kv_alloc(pool, x, n) == a.alloc(x, n)
            elif kind == "free":
                if x in a.req_type:
                    bd.boost_kv_free(pool, x)
                    a.free_request(x)
            elif kind == "fork":
                assert code(bd.boost_kv_fork, pool, x, y + 40, n) == a.fork(x, y + 40, n)
            elif kind == "unshare":
                held = max(1, len(a.req_blocks.get(x, [])))
                i = n % (held + 1)
                assert code(bd.boost_kv_unshare, pool, x, i) == a.unshare(x, i)
            elif kind == "truncate":
                held = len(a.req_blocks.get(x, []))
                keep = n % (held + 2)
                assert code(bd.boost_kv_truncate, pool, x, keep) == a.truncate(x, keep)
            else:
                src, dst = bd.boost_kv_compact(pool, n % 60)
                assert list(zip(src.tolist(), dst.tolist())) == a.compact(n % 60)
                assert not set(src.tolist()) & set(dst.tolist())
            s = bd.boost_kv_stats(pool)
            assert (s["free_shh"], s["free_local"]) == (a.n_free(okv.SHH), a.n_free(okv.LOCAL))
            assert s["used_blocks"] == len(a.used())
            assert s["used_host_head_blocks"] == int(sum(hh[b] for b in a.used()))
            assert s["requests"] == len(a.req_type)
            for r in a.req_type:
                assert bd.boost_kv_request_blocks(pool, r).tolist() == a.req_blocks[r]
                assert bd.boost_kv_request_type(pool, r) == a.req_type[r]
    finally:
        bd.boost_kv_pool_destroy(pool)


KINDS = ["alloc", "alloc", "alloc", "fork", "fork", "unshare", "unshare", "truncate", "free", "compact"]


@given(st.sampled_from([2, 8]), st.integers(2, 20),
       st.lists(st.tuples(st.sampled_from(KINDS), st.integers(0, 30), st.integers(0, 30),
                          st.integers(1, 200)), min_size=1, max_size=60))
@settings(max_examples=80, deadline=None)
def test_decisions_match_the_reference(plan_ctx, H, M, events):
    replay(plan_ctx, 500, H, M, events)


@pytest.mark.parametrize("fmt", [bd.KV_BF16, bd.KV_FP4])
def test_a_full_pool(plan_ctx, fmt):
    """Every block held: nothing to unshare into, nothing to move; after the
    first free block there is."""
    n = 512 if fmt == bd.KV_BF16 else 1920
    replay(plan_ctx, n, 8, 12, [("alloc", 31, 0, n - 3), ("alloc", 32, 0, 3), ("fork", 32, 0, 3),
                                ("unshare", 40, 0, 1), ("alloc", 33, 0, 1), ("compact", 0, 0, 59),
                                ("truncate", 31, 0, n - 4), ("unshare", 40, 0, 1),
                                ("unshare", 40, 0, 1), ("free", 32, 0, 1), ("compact", 0, 0, 59),
                                ("free", 40, 0, 1), ("compact", 0, 0, 59)], fmt)


def test_compaction_packs_both_lists(plan_ctx):
    rng = np.random.default_rng(0)
    pool = bd.boost_kv_pool_create(plan_ctx, 1, 8, 128, 4000, 12)
    try:
        nb = bd.boost_kv_pool_info(pool)["nb_pool"]
        hh = np.array([bd.boost_kv_block_host_heads(pool, b) for b in range(nb)])
        for r in range(40):
            bd.boost_kv_alloc(pool, r, int(rng.integers(1, 90)))
        for r in range(0, 40, 3):
            bd.boost_kv_free(pool, r)
        before = {r: bd.boost_kv_request_blocks(pool, r) for r in range(40) if r % 3}
        src, dst = bd.boost_kv_compact(pool, nb)
        to = dict(zip(src.tolist(), dst.tolist()))
        used = []
        for r, old in before.items():
            new = bd.boost_kv_request_blocks(pool, r)
            assert new.tolist() == [to.get(b, b) for b in old.tolist()]
            assert np.array_equal(hh[new], hh[old])  # no request changes tier
            used += new.tolist()
        for level in set(hh.tolist()):
            ids = np.flatnonzero(hh == level)
            held = [b for b in used if hh[b] == level]
            assert sorted(held) == ids[:len(held)].tolist()
        again = bd.boost_kv_compact(pool, nb)
        assert len(again[0]) == 0
    finally:
        bd.boost_kv_pool_destroy(pool)


def test_refusals(plan_ctx):
    pool = bd.boost_kv_pool_create(plan_ctx, 2, 8, 128, 512, 4)
    try:
        bd.boost_kv_alloc(pool, 1, 4)
        bd.boost_kv_fork(pool, 1, 2, 2)
        for f, *args in ((bd.boost_kv_fork, 9, 3, 1), (bd.boost_kv_fork, 1, 2, 1),
                         (bd.boost_kv_fork, 1, 1, 1), (bd.boost_kv_fork, 1, 3, 0),
                         (bd.boost_kv_fork, 1, 3, 5), (bd.boost_kv_unshare, 9, 0),
                         (bd.boost_kv_unshare, 1, 4), (bd.boost_kv_truncate, 9, 0),
                         (bd.boost_kv_truncate, 1, 5), (bd.boost_kv_request_blocks, 9)):
            with pytest.raises(bd.BoostError) as e:
                f(pool, *args)
            assert e.value.code == bd.EINVAL
        assert bd.boost_kv_stats(pool)["requests"] == 2
        lib = bd.load()
        import ctypes as C
        n = C.c_uint32()
        assert lib.boost_kv_compact(pool, 3, None, None, C.byref(n)) == bd.EINVAL
        assert lib.boost_kv_compact(pool, 0, None, None, C.byref(n)) == 0 and n.value == 0
        assert lib.boost_kv_compact(pool, 0, None, None, None) == bd.EINVAL
        assert lib.boost_kv_request_blocks(pool, 1, None, 4, C.byref(n)) == bd.EINVAL
        assert lib.boost_kv_unshare(pool, 1, 0, None, None) == bd.EINVAL
        for f in (lib.boost_kv_fork, lib.boost_kv_truncate):
            f_args = (None, 1, 2, 1)[:len(f.argtypes)]
            assert f(*f_args) == bd.EINVAL
        # device work needs a device
        one = np.zeros(1, np.int32)
        for call in (lambda: bd.boost_kv_copy_blocks(plan_ctx, pool, 0, 1, one, one + 1, 1),
                     lambda: bd.boost_kv_index_enable(pool), lambda: bd.boost_kv_pages(pool, 0, 0),
                     lambda: bd.boost_kv_read(plan_ctx, pool, 0, one, one, one, 1)):
            with pytest.raises(bd.BoostError) as e:
                call()
            assert e.value.code == bd.ENODEV
        with pytest.raises(ValueError):
            bd.boost_kv_copy_blocks(plan_ctx, pool, 0, 1, one, one, 2)
    finally:
        bd.boost_kv_pool_destroy(pool)


@pytest.mark.parametrize("mode,M,budget", [(bd.KV_LPP, 3, 0), (bd.KV_ALL_HBM, 0, 0), (bd.KV_ALL_HOST, 0, 0),
                                           (bd.KV_BUDGET, 0, 2 * 2 * 5 * bd.PAGE_BYTES)])
def test_geometry_of_a_4_bit_pool(plan_ctx, mode, M, budget):
    """1920 blocks of 1088 bytes a page; host pages and host heads by the rules
    of every pool."""
    H = 4
    pool = bd.boost_kv_pool_create_format(plan_ctx, bd.KV_FP4, 2, H, 128, 5000, M, mode, q_heads=H,
                                          hbm_budget_bytes=budget)
    try:
        i = bd.boost_kv_pool_info(pool)
        assert bd.boost_kv_pool_format(pool) == bd.KV_FP4
        assert (i["blocks_per_page"], i["nb_pool"], i["pages_per_tensor"]) == (1920, 5760, 12)
        host = {bd.KV_LPP: 4, bd.KV_ALL_HBM: 0, bd.KV_ALL_HOST: 12, bd.KV_BUDGET: 7}[mode]
        assert i["host_pages_per_tensor"] == host
        for b in (0, 1919, 1920, 5759):
            want = sum((h * 5760 + b) // 1920 >= 12 - host for h in range(H))
            assert bd.boost_kv_block_host_heads(pool, b) == want
    finally:
        bd.boost_kv_pool_destroy(pool)
    for fmt, D in ((bd.KV_FP4, 64), (2, 128), (-1, 128)):
        with pytest.raises(bd.BoostError) as e:
            bd.boost_kv_pool_create_format(plan_ctx, fmt, 1, H, D, 100, 3)
        assert e.value.code == bd.EINVAL
