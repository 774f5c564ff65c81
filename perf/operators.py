"""The long-context operators of the KV pool, as cases that can be timed and checked.

* ``write4``  tokens into a pool held in 4 bits, and back: a prompt's keys and values are quantised into their slots,
              then read as bf16 (what a swap-out or a dense pass over a cached prefix does);
* ``attn4``   decode attention over a pool held in 4 bits;
* ``index``   the block summaries of whole prompts, and the blocks that a query selects by them;
* ``sparse``  one layer's decode over a long context: the summary of the block with the new token, the selection of
              blocks for every KV head, and attention over those alone;
* ``copy``    blocks copied in every layer, as forked requests do before they write.

``modulus`` is the pool's linear placement (the last 1/M of its pages on host; 0 keeps everything in HBM).  Where
``own`` is false the operators are computed from elementary torch operations on a plain paged cache.
"""
import math

import numpy as np
import torch

own = False

HD = 128  # head dimension
T = 16  # tokens per block


def listed():
    return [
        # the new tokens of an odd batch: 37 requests, five KV heads; latency
        {"name": "37 tokens into 4 bits", "kind": "write4", "tokens": 37, "kv_heads": 5, "modulus": 0},
        # a long prompt's keys and values of one layer, in and out
        {"name": "prompt of 20011 into 4 bits", "kind": "write4", "tokens": 20011, "kv_heads": 8, "modulus": 0},
        # a chat of one user: the call with the fewest work items
        {"name": "4-bit attention, one short", "kind": "attn4", "q_heads": 32, "kv_heads": 8, "batch": 1,
         "ctx_lo": 301, "ctx_hi": 301, "empty": False, "modulus": 0},
        # the 64-request configuration of the bf16 pool (1/130 of a 4-bit tensor's 40 pages is less than one: all in HBM)
        {"name": "4-bit attention, batch 64", "kind": "attn4", "q_heads": 32, "kv_heads": 8, "batch": 64,
         "ctx_lo": 512, "ctx_hi": 4096, "empty": False, "modulus": 130},
        # eight query heads per KV head, ragged contexts down to one token, an empty one among them
        {"name": "4-bit attention, ragged", "kind": "attn4", "q_heads": 64, "kv_heads": 8, "batch": 19,
         "ctx_lo": 1, "ctx_hi": 9000, "empty": True, "modulus": 0},
        # two long documents
        {"name": "4-bit attention, two long", "kind": "attn4", "q_heads": 32, "kv_heads": 8, "batch": 2,
         "ctx_lo": 90001, "ctx_hi": 110003, "empty": False, "modulus": 0},
        # prompts that have just been written: every block summarised, then the first selection
        {"name": "index of 4 prompts", "kind": "index", "q_heads": 32, "kv_heads": 8, "batch": 4, "ctx_lo": 9001,
         "ctx_hi": 16384, "empty": False, "modulus": 0, "format": "bf16", "top": 64, "first": 1, "last": 2},
        # one request over a very long context: 1 block of 64 is read
        {"name": "sparse, one of 131072", "kind": "sparse", "q_heads": 32, "kv_heads": 8, "batch": 1, "ctx_lo": 131072,
         "ctx_hi": 131072, "empty": False, "modulus": 0, "format": "bf16", "top": 128, "first": 1, "last": 2},
        # a batch over long contexts, a part of the cache on host
        {"name": "sparse, 16 of 2000..30000", "kind": "sparse", "q_heads": 32, "kv_heads": 8, "batch": 16,
         "ctx_lo": 2000, "ctx_hi": 30000, "empty": False, "modulus": 130, "format": "bf16", "top": 64, "first": 1,
         "last": 4},
        # both together: blocks selected from a 4-bit cache, contexts shorter than the selection among them
        {"name": "sparse in 4 bits, ragged", "kind": "sparse", "q_heads": 64, "kv_heads": 8, "batch": 23, "ctx_lo": 1,
         "ctx_hi": 20000, "empty": True, "modulus": 0, "format": "fp4", "top": 96, "first": 2, "last": 3},
        # one forked request's last block in a two-layer model: the smallest copy
        {"name": "copy of 1 block", "kind": "copy", "pairs": 1, "layers": 2, "kv_heads": 8},
        # many forked requests' last blocks in an 8B model's cache
        {"name": "copy of 61 blocks, 32 layers", "kind": "copy", "pairs": 61, "layers": 32, "kv_heads": 8},
    ]


LARGEST = 5e8  # bytes of one pass of a drawn case, at most


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["write4"] * 2 + ["attn4"] * 5 + ["index"] * 2 + ["sparse"] * 5 + ["copy"] * 2)
    kv_heads = rng.choice([1, 2, 4, 5, 8, 8])
    if kind == "copy":
        return {"kind": kind, "pairs": _log(rng, 1, 240), "layers": _log(rng, 1, 32), "kv_heads": rng.choice([2, 4, 8])}
    if kind == "write4":
        return {"kind": kind, "tokens": _log(rng, 1, 40000), "kv_heads": kv_heads, "modulus": rng.choice([0, 130])}
    group = rng.choice([1, 2, 4, 4, 8])
    hi = _log(rng, 1, 110000)
    lo = rng.choice([1, max(1, hi // 8), hi])
    batch = max(1, min(_log(rng, 1, 160), 260000 // hi))
    c = {"kind": kind, "q_heads": group * kv_heads, "kv_heads": kv_heads, "batch": batch, "ctx_lo": lo, "ctx_hi": hi,
         "empty": batch > 2 and rng.random() < 0.3, "modulus": rng.choice([0, 0, 130])}
    if kind != "attn4":
        c["format"] = rng.choice(["bf16", "fp4"])
        c["top"] = _log(rng, 4, 300)
        c["first"] = rng.choice([0, 1, 2])
        c["last"] = rng.choice([0, 1, 2])
    return c


def draw(rng):
    while True:
        c = _draw(rng)
        if work(c)["bytes"] <= LARGEST:
            return c


def _lens(case, seed):
    """Context lengths uniform over [ctx_lo, ctx_hi]: one draw from each of `batch` equal parts of the range, in random
    order, so that every seed has other lengths and nearly the same total; the second is 0 where one is empty."""
    rng = np.random.default_rng(seed)
    n, lo, hi = case["batch"], case["ctx_lo"], case["ctx_hi"]
    u = (rng.permutation(n) + rng.random(n)) / n
    lens = np.minimum(hi, lo + np.floor(u * (hi - lo + 1))).astype(np.int64)
    if case["empty"]:
        lens[1] = 0
    return lens


def work(case):
    """What a pass reads and writes once each, and its arithmetic (expected context lengths)."""
    H, row = case["kv_heads"], HD * 2
    row4 = HD // 2 + HD // 32  # a token's K (or V) row of one head in 4 bits
    kind = case["kind"]
    if kind == "copy":
        return {"bytes": case["pairs"] * case["layers"] * H * 2 * T * row * 2, "flops": 0}
    if kind == "write4":
        return {"bytes": case["tokens"] * H * 2 * (2 * row + 2 * row4), "flops": 0}
    Hq, B = case["q_heads"], case["batch"]
    live = B - (1 if case["empty"] else 0)
    mean = (case["ctx_lo"] + case["ctx_hi"]) / 2
    io = B * Hq * row
    if kind == "attn4":
        return {"bytes": live * mean * H * 2 * row4 + 2 * io, "flops": live * mean * Hq * HD * 4}
    k_row, blocks = (row if case["format"] == "bf16" else row4), live * math.ceil(mean / T)
    summary = blocks * H * (2 * HD + 1)
    score = blocks * Hq * 2 * HD * 2
    if kind == "index":
        return {"bytes": live * mean * H * k_row + 2 * summary + io + blocks * H * 4 + B * H * case["top"] * 4,
                "flops": score}
    picked = live * min(mean, case["top"] * T)
    return {"bytes": live * H * (T * k_row + 2 * HD + 1) + summary + picked * H * 2 * k_row + 2 * io
            + B * H * case["top"] * 4, "flops": score + picked * Hq * HD * 4}


# --------------------------------------------------------------------------------------------- inputs
def _normal(seed, what, shape, dtype=torch.bfloat16):
    """~N(0, 1) on the GPU, a stream of its own for every (seed, what)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + what)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _kv(case, seed, tokens):
    """Keys and values bf16 [tokens, H, HD]; a few channels of a head are larger than the others, as keys' are."""
    got = []
    for what in (500, 501):
        gain = torch.exp2(_normal(seed, what + 10, (1, case["kv_heads"], HD), torch.float32))
        got.append((_normal(seed, what, (tokens, case["kv_heads"], HD), torch.float32) * gain).to(torch.bfloat16))
    return got


def _query(case, seed):
    return _normal(seed, 200, (case["batch"], case["q_heads"], HD))


def _pairs(case, seed):
    """Blocks that are copied, and others that take the copies; a source may serve several."""
    rng = np.random.default_rng(seed)
    order = rng.permutation(512)
    src = order[rng.integers(0, 200, size=case["pairs"])]
    return src.astype(np.int32), order[200:200 + case["pairs"]].astype(np.int32)


class State:
    pass


class _Pool:
    """The library's pool, given back when neither a state nor a view of its memory needs it any more."""

    def __init__(self, bd, handle):
        self.bd, self.handle = bd, handle

    def __del__(self):
        try:
            torch.cuda.synchronize()
            self.bd.boost_kv_pool_destroy(self.handle)
        except Exception:  # the interpreter is going down
            pass


_CTX = None


def _library():
    global _CTX
    from paper_2609_13592_amd import binding as bd
    if _CTX is None:
        _CTX = bd.boost_init(torch.cuda.current_device())
    return bd, _CTX


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _fill(s, case, lens):
    """A pool (or, in the plain form, a paged cache) for requests of `lens` tokens, and every token's slot.  Each request
    gets the blocks of the first half of its context at once, as a prompt does, the rest in turn, as decoding does."""
    need = [-(-int(n) // T) for n in lens]
    s.mb = -(-case.get("ctx_hi", int(lens.max())) // T)  # a table as wide as the longest request may get
    s.fp4 = case["kind"] in ("write4", "attn4") or case["format"] == "fp4"
    if own:
        s.bd, s.ctx = _library()
        s.pool = s.bd.boost_kv_pool_create_format(
            s.ctx, s.bd.KV_FP4 if s.fp4 else s.bd.KV_BF16, 1, case["kv_heads"], HD, max(1, sum(need)),
            case["modulus"] or 2, s.bd.KV_LPP if case["modulus"] else s.bd.KV_ALL_HBM,
            q_heads=case.get("q_heads", case["kv_heads"]), max_batch=len(need), max_blocks_per_seq=s.mb)
        s.owner = _Pool(s.bd, s.pool)
        take = lambda b, n: s.bd.boost_kv_alloc(s.pool, b, n)  # noqa: E731
    else:
        ids = iter(range(max(1, sum(need))))
        take = lambda b, n: [next(ids) for _ in range(n)]  # noqa: E731
    rows = [take(b, (n + 1) // 2) if n else [] for b, n in enumerate(need)]
    for i in range(0, s.mb, 4):
        for b, n in enumerate(need):
            if len(rows[b]) < n:
                rows[b] += take(b, min(4, n - len(rows[b])))
    tables = np.full((len(need), s.mb), -1, np.int32)
    slots = [np.zeros(0, np.int64)]
    for b, r in enumerate(rows):
        tables[b, :len(r)] = r
        t = np.arange(int(lens[b]))
        slots.append(tables[b, t // T].astype(np.int64) * T + t % T)
    slots = np.concatenate(slots)
    s.tables = torch.from_numpy(tables).cuda()
    s.lens = torch.from_numpy(lens.astype(np.int32)).cuda()
    if not own:
        s.nb = max(1, sum(need))
        s.tables = s.tables.clamp(min=0).long()
        s.lens = s.lens.long()
    return torch.from_numpy(slots.astype(np.int32) if own else slots).cuda()


def _rows(s, case):
    """The plain paged cache: rows by slot, bf16 or (codes, scale bytes)."""
    n, H = s.nb * T, case["kv_heads"]
    if s.fp4:
        return [(torch.zeros((n, H, HD // 2), dtype=torch.uint8, device="cuda"),
                 torch.zeros((n, H, HD // 32), dtype=torch.uint8, device="cuda")) for _ in (0, 1)]
    return [torch.zeros((n, H, HD), dtype=torch.bfloat16, device="cuda") for _ in (0, 1)]


def prepare(case, seed):
    s = State()
    s.case, H = case, case["kv_heads"]
    kind = case["kind"]
    if kind == "copy":
        s.src, s.dst = _pairs(case, seed)
        shape = (case["layers"], 2, H, 512, T, HD)
        if own:  # the pool's pages in HBM follow each other: one view of them all
            s.bd, s.ctx = _library()
            s.pool = s.bd.boost_kv_pool_create_format(s.ctx, s.bd.KV_BF16, case["layers"], H, HD, 512, 2,
                                                      s.bd.KV_ALL_HBM, max_batch=1, max_blocks_per_seq=1)
            s.owner = _Pool(s.bd, s.pool)
            s.cache = _view(int(s.bd.boost_kv_pages(s.pool, 0, 0)[0]), shape, s.owner)
        else:
            s.cache = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
            s.src, s.dst = (torch.from_numpy(v.astype(np.int64)).cuda() for v in (s.src, s.dst))
        for layer in range(case["layers"]):
            s.cache[layer] = _normal(seed, 600 + layer, shape[1:])
        return s
    lens = np.array([case["tokens"]]) if kind == "write4" else _lens(case, seed)
    slots = _fill(s, case, lens)
    k, v = _kv(case, seed, int(slots.numel()))
    n = int(slots.numel())
    if not own:
        s.rows = _rows(s, case)
    if kind == "write4":
        s.slots, s.k, s.v, s.n = slots, k, v, n
        s.k_out, s.v_out = torch.empty_like(k), torch.empty_like(v)
        return s
    if own:
        if n:
            s.bd.boost_kv_write(s.ctx, s.pool, 0, slots, k, v, n, _stream())
    else:
        _store(s.rows, s.fp4, slots, k, v)
    B = case["batch"]
    s.q = _query(case, seed)
    s.o = torch.empty_like(s.q)
    if kind == "attn4":
        return s
    s.starts = (s.lens - 1).clamp(min=0) if kind == "sparse" else torch.zeros_like(s.lens)
    s.scores = torch.zeros((B, H, s.mb), dtype=torch.float32, device="cuda")
    s.sel = torch.empty((B, H, case["top"]), dtype=torch.int32, device="cuda")
    if own:
        s.bd.boost_kv_index_enable(s.pool)
    else:
        s.index = [torch.zeros((s.nb, H, HD), dtype=torch.int8, device="cuda") for _ in (0, 1)]
        s.index.append(torch.zeros((s.nb, H), dtype=torch.int8, device="cuda"))
    if kind == "sparse":  # the summaries that the prompt and earlier steps have left
        if own:
            s.bd.boost_kv_index_update(s.ctx, s.pool, 0, s.tables, s.mb, torch.zeros_like(s.lens), s.lens, B,
                                       int(lens.max()), _stream())
        else:
            _update(s, torch.arange(s.mb, device="cuda").expand(B, s.mb))
    return s


class _Memory:
    def __init__(self, address, shape, owner):
        self.owner = owner  # torch keeps this object as long as a tensor of its memory lives
        self.__cuda_array_interface__ = {"data": (address, False), "shape": shape, "typestr": "<i2", "version": 2}


def _view(address, shape, owner):
    return torch.as_tensor(_Memory(address, shape, owner), device="cuda").view(torch.bfloat16)


# ---------------------------------------------------------------------------------------- plain forms
def _pow2(e):
    """2^e for whole e, in 64 bits and exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _codes(x):
    """bf16 [..., HD] in 4 bits: two codes a byte (even dim low), and a scale byte for each 32 dims."""
    g = x.float().reshape(*x.shape[:-1], HD // 32, 32)
    m, ex = torch.frexp(g.abs().amax(-1))
    e = (ex - 3 + (m > 0.875).int()).clamp(-127, 125)  # the largest value is at most 7 steps
    e = torch.where(m == 0, torch.full_like(e, -127), e)
    y = (g.double() * _pow2(-e)[..., None]).float()
    a = y.abs()
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte()
            + (a >= 3.5).byte() + (a > 5).byte() + 8 * (y < 0).byte()).reshape(*x.shape[:-1], HD // 2, 2)
    return code[..., 0] + 16 * code[..., 1], (e + 127).byte()


def _values(codes, scales):
    """What the codes stand for, in 32 bits."""
    steps = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).int().reshape(*scales.shape, 32)
    return (steps[c] * _pow2(scales.int() - 127).float()[..., None]).reshape(*codes.shape[:-1], HD)


def _store(rows, fp4, slots, k, v):
    for r, x in zip(rows, (k, v)):
        if fp4:
            r[0][slots], r[1][slots] = _codes(x)
        else:
            r[slots] = x


def _blocks(s, which, ids, head=None):
    """Blocks `ids` in 32 bits: [..., T, H, HD], or of KV heads `head` alone [..., T, HD]."""
    def take(x):
        x = x.view(s.nb, T, *x.shape[1:])
        return x[ids] if head is None else x[ids, :, head]
    r = s.rows[which]
    return _values(take(r[0]), take(r[1])) if s.fp4 else take(r).float()


def _attend(q, k, v, live):
    """q [B, H, G, HD], k and v [B, H, N, HD], live [B, H or 1, N]: softmax over what is live, zero rows where nothing is."""
    score = (q @ k.transpose(-1, -2).contiguous()) * HD ** -0.5
    score = score.masked_fill(~live[:, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    return (p @ v) / total.masked_fill(total == 0, 1.0)


def _update(s, blk):
    """Summaries of the logical blocks blk [B, n]: for every dim the largest and smallest key of the block's live tokens,
    outwards in whole steps of 2^e, the smallest at which none is over 127."""
    k = _blocks(s, 0, torch.gather(s.tables, 1, blk))  # [B, n, T, H, HD]
    at = blk[..., None] * T + torch.arange(T, device="cuda")
    live = (at < s.lens[:, None, None])[..., None, None]
    m, ex = torch.frexp((k.abs() * live).amax((2, 4)))
    e = torch.where(m == 0, torch.full_like(ex, -126), (ex - 7 + (m > 127 / 128).int()).clamp(min=-126))
    step = _pow2(-e).float()[..., None]
    hi = torch.ceil(k.masked_fill(~live, -math.inf).amax(2) * step)
    lo = torch.floor(k.masked_fill(~live, math.inf).amin(2) * step)
    here = live[:, :, 0, 0, 0]
    ids = torch.gather(s.tables, 1, blk)[here]
    for to, x in zip(s.index, (hi, lo, e)):
        to[ids] = x[here].to(torch.int8)


def _select(s, case):
    """Scores [B, H, blocks] and the selected blocks, ascending, -1 behind the last."""
    B, H = case["batch"], case["kv_heads"]
    q = s.q.float().view(B, H, -1, HD)
    m, ex = torch.frexp(q.abs().amax(-1))
    e = torch.where(m == 0, torch.full_like(ex, -126), (ex - 7 + (m > 127 / 128).int()).clamp(min=-126))
    q8 = torch.round(q * _pow2(-e).float()[..., None]).clamp(-127, 127)
    hi, lo = (x[s.tables].permute(0, 2, 3, 1).float().contiguous() for x in s.index[:2])  # [B, H, HD, blocks]
    bound = q8.clamp(min=0) @ hi + q8.clamp(max=0) @ lo  # whole numbers below 2^24: exact
    both = e[..., None] + s.index[2][s.tables].permute(0, 2, 1)[:, :, None].int()
    score = (bound.double() * _pow2(both)).float().amax(2)
    at = torch.arange(s.mb, device="cuda")
    n = ((s.lens + T - 1) // T)[:, None, None]
    s.scores = torch.where(at < n, score, s.scores)
    always = (at < case["first"]) | (at >= n - case["last"])
    key = score.masked_fill(always, math.inf).masked_fill(at >= n, -math.inf)
    top = min(case["top"], s.mb)
    sel = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :top]
    sel = torch.where(torch.arange(top, device="cuda") < n, sel, torch.full_like(sel, s.mb))
    sel = torch.sort(sel, -1).values
    sel = torch.where(sel == s.mb, torch.full_like(sel, -1), sel)
    return torch.nn.functional.pad(sel, (0, case["top"] - top), value=-1)


def _plain(s):
    case, kind = s.case, s.case["kind"]
    if kind == "copy":
        s.cache[:, :, :, s.dst] = s.cache[:, :, :, s.src]
        return s.cache
    if kind == "write4":
        _store(s.rows, True, s.slots, s.k, s.v)
        return [_values(r[0][s.slots], r[1][s.slots]).to(torch.bfloat16) for r in s.rows]
    B, H = case["batch"], case["kv_heads"]
    q = s.q.float().view(B, H, -1, HD)
    if kind == "attn4":
        k, v = (_blocks(s, w, s.tables).reshape(B, s.mb * T, H, HD).transpose(1, 2).contiguous() for w in (0, 1))
        live = torch.arange(s.mb * T, device="cuda") < s.lens[:, None, None]
        return _attend(q, k, v, live).to(torch.bfloat16).view(B, -1, HD)
    if kind == "index":
        _update(s, torch.arange(s.mb, device="cuda").expand(B, s.mb))
        sel = _select(s, case)
        return [s.scores, sel.int()]
    _update(s, (s.starts // T)[:, None])
    sel = _select(s, case)
    ids = torch.gather(s.tables[:, None].expand(B, H, s.mb), 2, sel.clamp(min=0))
    head = torch.arange(H, device="cuda")[None, :, None]
    k, v = (_blocks(s, w, ids, head).reshape(B, H, -1, HD) for w in (0, 1))
    at = sel[..., None] * T + torch.arange(T, device="cuda")
    live = ((sel[..., None] >= 0) & (at < s.lens[:, None, None, None])).view(B, H, -1)
    return [sel.int(), _attend(q, k, v, live).to(torch.bfloat16).view(B, -1, HD)]


# ------------------------------------------------------------------------------------------------ run
def run(s):
    if not own:
        return _plain(s)
    bd, c, st, case = s.bd, s.ctx, _stream(), s.case
    kind = case["kind"]
    if kind == "copy":
        bd.boost_kv_copy_blocks(c, s.pool, 0, case["layers"], s.src, s.dst, case["pairs"], st)
        return s.cache
    if kind == "write4":
        bd.boost_kv_write(c, s.pool, 0, s.slots, s.k, s.v, s.n, st)
        bd.boost_kv_read(c, s.pool, 0, s.slots, s.k_out, s.v_out, s.n, st)
        return [s.k_out, s.v_out]
    B, Hq = case["batch"], case["q_heads"]
    if kind == "attn4":
        bd.boost_paged_attn_decode(c, s.pool, 0, s.q, B, Hq, s.tables, s.mb, s.lens, 0.0, s.o, bd.DTYPE_BF16, st)
        return s.o
    new = 1 if kind == "sparse" else s.mb * T
    bd.boost_kv_index_update(c, s.pool, 0, s.tables, s.mb, s.starts, s.lens, B, new, st)
    bd.boost_kv_select(c, s.pool, 0, s.q, B, Hq, s.tables, s.mb, s.lens, case["top"], case["first"], case["last"],
                       s.scores, s.sel, st)
    if kind == "index":
        return [s.scores, s.sel]
    bd.boost_sparse_attn_decode(c, s.pool, 0, s.q, B, Hq, s.tables, s.mb, s.lens, s.sel, case["top"], 0.0, s.o,
                                bd.DTYPE_BF16, st)
    return [s.sel, s.o]


# ---------------------------------------------------------------------------------------------- exact
def _exact4(x):
    """The value in 4 bits that is nearest to each of x (64 bits), from the definition: multiples of the group's step
    out of 0, 1/2, 1, 3/2, 2, 3, 4, 6, the even one of two that are as near."""
    x = x.double()
    g = x.reshape(-1, 32)
    top = g.abs().amax(1, keepdim=True)
    step = torch.full_like(top, 2.0 ** -127)
    live = top > 0
    power = torch.ceil(torch.log2(torch.where(live, top, torch.ones_like(top)) / 7))
    for p in (power - 1, power, power + 1):  # log2 may be a rounding off at a border: the smallest that holds
        fits = live & (top <= 7 * _pow2(p)) & (top > 3.5 * _pow2(p))
        step = torch.where(fits, _pow2(p.clamp(-127, 125)), step)
    a = g.abs() / step
    out = torch.zeros_like(a)
    grid = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
    for i in range(1, 8):
        middle = (grid[i - 1] + grid[i]) / 2
        up = (a > middle) | ((a == middle) & (i % 2 == 0))
        out = torch.where(up, torch.full_like(a, grid[i]), out)
    return (out * step * g.sign()).reshape(x.shape)


def _exact_sel(case, q, k):
    """Scores and selected blocks of one request: q [H, G, HD], k [L, H, HD], both in 64 bits."""
    L, H = k.shape[0], k.shape[1]
    n = -(-L // T)

    def grid(top):  # the smallest power of two of which top is at most 127
        p = torch.floor(torch.log2(top.clamp(min=2.0 ** -140) / 127))
        for _ in range(2):
            p = torch.where(top > 127 * _pow2(p), p + 1, p)
        return _pow2(p.clamp(min=-126))

    last = k[-1:].expand(n * T - L, H, HD)  # a token twice changes no extreme
    b = torch.cat([k, last]).view(n, T, H, HD)
    step = grid(b.abs().amax((1, 3)))  # [n, H]
    hi, lo = torch.ceil(b.amax(1) / step[..., None]), torch.floor(b.amin(1) / step[..., None])
    qs = grid(q.abs().amax(2))
    q8 = torch.round(q / qs[..., None]).clamp(-127, 127)
    score = torch.empty((H, n), dtype=torch.float64, device=k.device)
    for h in range(H):
        each = torch.maximum(q8[h][:, None] * hi[None, :, h], q8[h][:, None] * lo[None, :, h]).sum(-1)
        score[h] = (each * qs[h][:, None] * step[None, :, h]).amax(0)
    sel = np.full((H, case["top"]), -1, np.int32)
    for h, row in enumerate(score.cpu().numpy()):
        keep = set(range(min(case["first"], n))) | set(range(max(0, n - case["last"]), n))
        for i in np.argsort(-row, kind="stable"):
            if len(keep) >= min(n, case["top"]):
                break
            keep.add(int(i))
        sel[h, :len(keep)] = sorted(keep)
    return score, sel


def exact(case, seed):
    kind, H = case["kind"], case["kv_heads"]
    if kind == "copy":
        src, dst = _pairs(case, seed)
        cache = torch.stack([_normal(seed, 600 + i, (2, H, 512, T, HD)) for i in range(case["layers"])])
        for a, b in zip(src.tolist(), dst.tolist()):
            cache[:, :, :, b] = cache[:, :, :, a]
        return cache
    if kind == "write4":
        return [_exact4(x) for x in _kv(case, seed, case["tokens"])]
    lens = _lens(case, seed)
    k, v = _kv(case, seed, int(lens.sum()))
    q = _query(case, seed).double().view(case["batch"], H, -1, HD)
    mb = -(-case["ctx_hi"] // T)
    out = torch.zeros_like(q)
    scores = torch.zeros((case["batch"], H, mb), dtype=torch.float64, device="cuda")
    chosen = np.full((case["batch"], H, case["top"]), -1, np.int32) if kind != "attn4" else None
    at = 0
    for b, n in enumerate(int(n) for n in lens):
        kb, vb = k[at:at + n], v[at:at + n]
        at += n
        if n == 0:
            continue
        four = kind == "attn4" or case["format"] == "fp4"
        kb, vb = (_exact4(x) if four else x.double() for x in (kb, vb))
        if kind != "attn4":
            s, chosen[b] = _exact_sel(case, q[b], kb)
            scores[b, :, :s.shape[1]] = s
        if kind == "index":
            continue
        for h in range(H):
            kh, vh = kb[:, h], vb[:, h]
            if kind == "sparse":
                t = (torch.from_numpy(chosen[b, h][chosen[b, h] >= 0]).cuda().long()[:, None] * T
                     + torch.arange(T, device="cuda")).view(-1)
                t = t[t < n]
                kh, vh = kh[t], vh[t]
            out[b, h] = torch.softmax(q[b, h] @ kh.t() / math.sqrt(HD), -1) @ vh
    out = out.view(case["batch"], -1, HD)
    if kind == "attn4":
        return out
    chosen = torch.from_numpy(chosen)
    return [scores, chosen] if kind == "index" else [chosen, out]
