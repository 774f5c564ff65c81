"""A decode step over a 4-bit pool, and with attention over selected blocks:
the append, the summaries, the selection and the attention as one program."""
import numpy as np
import pytest

import synth
from oracle import decode_step as ods
from oracle import gemv as og
from oracle import kv4
from oracle import select as osel
from paper_2609_13592_amd import binding as bd
from paper_2609_13592_amd.step import DecodeModel, Dims
from tests.gpu_util import dev_u16, fill_pool, host_u16, stream, sync, to_dev_u16
from tests.test_gpu_decode_step import check_ids, check_logits, model_weights

pytestmark = pytest.mark.gpu
FORMATS = [bd.KV_BF16, bd.KV_FP4]


def i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Run:
    """A model of `dims` whose requests hold all but the last of `lengths`."""

    def __init__(self, ctx, dims, fmt, lengths, top=0, mode=bd.KV_ALL_HBM, M=0, fold=True):
        self.ctx, self.dims, self.lengths, self.top = ctx, dims, np.asarray(lengths), top
        self.w = model_weights(dims, 5)
        self.mats = {n: bd.boost_place_weights_map(
            ctx, a, a.nbytes, np.zeros(-(-a.nbytes // bd.PAGE_BYTES), np.uint8))
            for n, a in self.w.items() if not n.startswith("norm")}
        norms = {n: to_dev_u16(a) for n, a in self.w.items() if n.startswith("norm")}
        B = len(lengths)
        need = (self.lengths + 15) // 16
        self.mb = int(need.max())
        self.pool = bd.boost_kv_pool_create_format(
            ctx, fmt, dims.layers, dims.hkv, dims.hd, int(need.sum()), M, mode, q_heads=dims.hq,
            max_batch=B, max_blocks_per_seq=self.mb)
        self.tables = np.full((B, self.mb), -1, np.int32)
        for b in range(B):
            self.tables[b, :need[b]] = bd.boost_kv_alloc(self.pool, b, int(need[b]))
        rng = np.random.default_rng(6)
        self.old = []
        for l in range(dims.layers):
            kv = [[synth.normal_bf16(rng, (int(L) - 1, dims.hkv, dims.hd), 1.0) for L in lengths]
                  for _ in range(2)]
            self.old.append(kv)
            fill_pool(bd, ctx, self.pool, l, self.lengths - 1, *kv, tables=self.tables)
        self.model = DecodeModel(ctx, dims, B, self.mb, self.pool, self.mats, norms,
                                 fold_slices=fold, top_blocks=top)
        self.tokens = rng.integers(0, dims.vocab, size=B)
        self.dev = [i32(a) for a in (self.tokens, self.lengths - 1, self.lengths, self.tables)]
        if top:
            for l in range(dims.layers):
                bd.boost_kv_index_update(ctx, self.pool, l, self.dev[3], self.mb,
                                         i32(np.zeros(B)), self.dev[1], B,
                                         max(1, int(self.lengths.max()) - 1), stream())

    def step(self):
        ids, logits = self.model.step(*self.dev, stream())
        sync()
        return ids.cpu().numpy(), logits.cpu().numpy()

    def held(self, l):
        """K and V of every request as the pool now holds them (fp64)."""
        out = []
        for b, L in enumerate(self.lengths):
            t = np.arange(int(L))
            k, v = (dev_u16(int(L), self.dims.hkv, self.dims.hd) for _ in range(2))
            bd.boost_kv_read(self.ctx, self.pool, l, i32(self.tables[b, t // 16] * 16 + t % 16), k, v,
                             int(L), stream())
            sync()
            out.append([og.bf16_to_f32(host_u16(x)).astype(np.float64) for x in (k, v)])
        return out

    def close(self):
        for t in self.mats.values():
            bd.boost_tensor_free(t)
        bd.boost_kv_pool_destroy(self.pool)


def attended(held, q, lists):
    """decode_attention over what the pool holds, of the listed blocks."""
    o = np.zeros(q.shape)
    for b, (k, v) in enumerate(held):
        G = q.shape[1] // k.shape[1]
        for h in range(q.shape[1]):
            t = np.arange(k.shape[0])
            if lists is not None:
                t = t[np.isin(t // 16, lists[b][h // G])]
            o[b, h] = kv4.attend(q[b, h][None], k[t, h // G], v[t, h // G])[0]
    return o


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("top", [0, 100, 9])
@pytest.mark.parametrize("mode,M,fold", [(bd.KV_ALL_HBM, 0, True), (bd.KV_LPP, 2, False)])
def test_step_matches_the_oracle(gpu_ctx, monkeypatch, fmt, top, mode, M, fold):
    """One layer, its attention over the cache as the step left it: the earlier
    tokens are what was written, the new one is within a step of its group's
    grid (bf16: a unit in the last place) of the oracle's, and the logits meet
    the composed step's bars given the blocks that the step selected, which
    are those of the oracle's own ranking of the step's queries."""
    dims = Dims(layers=1, d=512, hq=8, hkv=2, hd=128, ffn=384, vocab=500)
    r = Run(gpu_ctx, dims, fmt, [1, 17, 300, 16, 1025], top, mode, M, fold)
    try:
        ids, logits = r.step()
        held = r.held(0)
        lists = None
        if top:
            q = r.model.q.cpu().double().numpy()
            lists = r.model.sel.cpu().numpy()
            for b, (k, _) in enumerate(held):
                assert np.array_equal(lists[b], osel.select(osel.scores(q[b], k), top, 1, 2)), b
        seen = {}

        def attention(q16, ks, vs):
            seen["kv"] = [(og.bf16_to_f32(k[-1]), og.bf16_to_f32(v[-1])) for k, v in zip(ks, vs)]
            return attended(held, og.bf16_to_f32(q16).astype(np.float64), lists)
        monkeypatch.setattr(ods, "decode_attention", attention)
        ref, _, _ = ods.decode_step(r.w, r.tokens, [r.old[0][0]], [r.old[0][1]],
                                    r.lengths, dims.__dict__)
        check_logits(logits, ref)
        check_ids(ids, ref)
        for b, L in enumerate(r.lengths):
            for i in range(2):
                old = r.old[0][i][b]
                want = kv4.stored(old) if fmt == bd.KV_FP4 else og.bf16_to_f32(old)
                assert np.array_equal(held[b][i][:-1], want), (b, i)
                new = seen["kv"][b][i].astype(np.float64).reshape(dims.hkv, 4, 32)
                top_of = np.abs(new).max(-1, keepdims=True)
                # bf16: an fp32 sum on the other side of a rounding; 4 bits: the grid's widest
                # step is 2 of 6, its scale is at most twice what 7 would need
                tol = top_of * 2.0 ** -7 if fmt == bd.KV_BF16 else top_of * (2 / 3.5) * 1.01
                got = held[b][i][-1].reshape(dims.hkv, 4, 32)
                assert np.all(np.abs(got - new) <= tol), (b, i)
    finally:
        r.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("top", [0, 5])
def test_placement_folding_and_replays_keep_every_bit(gpu_ctx, fmt, top):
    """Two layers: host pages or none, slices folded or not, and replays of a
    captured step (which appends and summarises the same token again)."""
    import torch
    dims = Dims(layers=2, d=2048, hq=16, hkv=4, hd=128, ffn=512, vocab=500)
    lengths = [33, 1, 700, 16, 17, 250]
    outs = []
    for mode, M, fold in ((bd.KV_ALL_HBM, 0, True), (bd.KV_LPP, 3, True), (bd.KV_ALL_HOST, 0, False)):
        r = Run(gpu_ctx, dims, fmt, lengths, top, mode, M, fold)
        try:
            outs.append(r.step())
            if mode == bd.KV_LPP:
                continue
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                s = torch.cuda.current_stream().cuda_stream
                ids, logits = r.model.step(*r.dev, s)
            for _ in range(3):
                logits.fill_(float("nan"))
                ids.fill_(-1)
                sync()
                g.replay()
                sync()
                outs.append((ids.cpu().numpy(), logits.cpu().numpy()))
                r.step()
            del g
        finally:
            r.close()
    for ids, logits in outs[1:]:
        assert np.array_equal(ids, outs[0][0])
        assert np.array_equal(logits.view(np.uint32), outs[0][1].view(np.uint32))


@pytest.mark.parametrize("fmt", FORMATS)
def test_bytes_of_a_step(gpu_ctx, fmt):
    dims = Dims(layers=2, d=256, hq=4, hkv=2, hd=128, ffn=384, vocab=1000)
    row = 512 if fmt == bd.KV_BF16 else 136  # K and V of a token and head
    r = Run(gpu_ctx, dims, fmt, [1, 40, 100], 0)
    try:
        dense = r.model.bytes_per_step(r.lengths)
        sparse = DecodeModel(gpu_ctx, dims, 3, r.mb, r.pool, r.mats, r.model.norms, top_blocks=2)
        assert dense - sparse.bytes_per_step(r.lengths) == 2 * 2 * (
            (8 + 68) * row - (1 + 3 + 7) * 257)
    finally:
        r.close()
