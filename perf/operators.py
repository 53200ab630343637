"""The operators a server puts around the decode step, as cases that can be timed: block tables of a paged cache, the
8-bit cache with one scale per block and head (append and attention), and the draw of the next token.

`run` computes each of them in plain torch operations, or, with `own` set, through the library's entry points.  Shapes:
20 query / 5 KV heads of 128 and a vocabulary of 128,256 are this library's 2B configuration; the others are generic.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
Q_MAX = {"int8": 127.0, "e4m3": 448.0}
A_MIN = 1e-30  # below this a block counts as all zero: its scale is that of A_MIN


def listed():
    return [
        # one decode step's bookkeeping for a small batch: every request gets one token, one has just finished
        {"name": "tables_decode", "op": "tables", "requests": 16, "block": 64, "max_blocks": 64, "new": "decode", "tokens": 16},
        # a server's step with everything in it: prompts of up to 2000 tokens beside decoding, idle and finished requests
        {"name": "tables_mixed", "op": "tables", "requests": 300, "block": 32, "max_blocks": 256, "new": "mixed", "tokens": 131072},
        # prompts of up to 500 tokens for thousands of requests at once (offline scoring): a million slots
        {"name": "tables_prefill", "op": "tables", "requests": 4096, "block": 16, "max_blocks": 96, "new": "prompts", "tokens": 1048576},
        # one new token for each of 16 sequences
        {"name": "append_decode", "op": "append", "kind": "int8", "heads": 20, "kv_heads": 5, "dim": 128, "block": 64, "requests": 16, "most_new": 1},
        # speculative decoding: up to 7 tokens for each of 75 sequences, small heads, small blocks
        {"name": "append_ragged", "op": "append", "kind": "e4m3", "heads": 16, "kv_heads": 4, "dim": 64, "block": 16, "requests": 75, "most_new": 7},
        # chunks of prompts: some ten thousand tokens
        {"name": "append_prefill", "op": "append", "kind": "int8", "heads": 20, "kv_heads": 5, "dim": 128, "block": 32, "requests": 11, "most_new": 2000},
        # one sequence with 4096 cached tokens: the latency of a single user's token
        {"name": "attend_one", "op": "attend", "kind": "int8", "heads": 20, "kv_heads": 5, "dim": 128, "block": 64, "requests": 1, "shortest": 4096, "longest": 4096},
        # 16 sequences of about 4096 tokens
        {"name": "attend_batch", "op": "attend", "kind": "e4m3", "heads": 20, "kv_heads": 5, "dim": 128, "block": 64, "requests": 16, "shortest": 3500, "longest": 4096},
        # a busy server: lengths from one token to 16 thousand in one batch, small blocks
        {"name": "attend_ragged", "op": "attend", "kind": "int8", "heads": 20, "kv_heads": 5, "dim": 128, "block": 16, "requests": 97, "shortest": 1, "longest": 16384},
        # one token, every filter on
        {"name": "sample_one", "op": "sample", "rows": 1, "vocab": 128256, "spread": 2.5, "filters": "all"},
        # 16 users with settings of their own, greedy ones among them
        {"name": "sample_batch", "op": "sample", "rows": 16, "vocab": 128256, "spread": 2.5, "filters": "mixed"},
        # many samples at temperature one without a filter, flat distributions (rollouts for training)
        {"name": "sample_flat", "op": "sample", "rows": 192, "vocab": 128256, "spread": 1.0, "filters": "none"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "sample"])
    if op == "tables":
        new = rng.choice(["decode", "mixed", "prompts"])
        requests = _log(rng, 1, 4000)
        most = {"decode": 1, "mixed": 700, "prompts": 256}[new]
        return {"op": op, "requests": requests, "block": rng.choice([16, 32, 64, 128]), "max_blocks": rng.randint(32, 96) if requests > 500 else rng.randint(64, 512),
                "new": new, "tokens": min(1000000, max(requests, _log(rng, requests, requests * most)))}
    heads, kv_heads = rng.choice([(20, 5), (16, 4), (32, 4), (8, 8), (28, 4), (6, 2)])
    shape = {"kind": rng.choice(["int8", "e4m3"]), "heads": heads, "kv_heads": kv_heads, "dim": rng.choice([64, 128]), "block": rng.choice([16, 32, 64, 128])}
    if op == "append":
        most_new = _log(rng, 1, 1000)
        return {"op": op, **shape, "requests": _log(rng, 1, max(1, min(300, 5000 // most_new))), "most_new": most_new}
    if op == "attend":
        longest = _log(rng, 1, 30000)
        most = 120000000 // (longest * kv_heads * shape["dim"])
        return {"op": op, **shape, "requests": _log(rng, 1, max(1, min(128, most))), "shortest": rng.randint(0, longest), "longest": longest}
    vocab = _log(rng, 100, 160000)
    return {"op": op, "rows": _log(rng, 1, max(1, min(256, 12000000 // vocab))), "vocab": vocab, "spread": rng.choice([0.5, 1.0, 2.5, 6.0]),
            "filters": rng.choice(["none", "all", "mixed", "top_k", "top_p"])}


# ------------------------------------------------------------------------------------------------------ inputs

def _to(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _prepare_tables(c, seed):
    rng = np.random.default_rng([seed, 1])
    R, B, most = c["requests"], c["block"], c["max_blocks"]
    cap = most * B
    share = max(1, 2 * c["tokens"] // R)  # tokens are for all requests together
    lengths = rng.integers(0, cap // 2, R)
    if c["new"] == "decode":
        new = np.ones(R, np.int64)
        if R > 1:
            new[rng.integers(0, R)] = -1
    elif c["new"] == "mixed":
        kind = rng.integers(0, 10, R)
        new = np.where(kind < 5, 1, np.where(kind < 7, rng.integers(1, 2 + min(2000, share), R), np.where(kind < 8, 0, -1)))
    else:
        lengths[:] = rng.integers(0, 2 * B, R)
        new = rng.integers(1, 2 + min(500, share), R)
    used = -(-lengths // B)
    need = np.where(new > 0, -(-(lengths + np.maximum(new, 0)) // B) - used, 0)
    # blocks enough for the step, now and then a few too little
    spare = int(need.sum()) + int(rng.integers(-2, 50))
    n_blocks = R * most
    n_free = min(max(0, spare - int(used[new < 0].sum())), n_blocks - int(used.sum()))
    ids = rng.permutation(n_blocks).astype(np.int32)
    tables = np.full((R, most), -1, np.int32)
    tables[np.arange(most) < used[:, None]] = ids[: int(used.sum())]
    free = np.full(n_blocks, -1, np.int32)
    free[:n_free] = ids[int(used.sum()): int(used.sum()) + n_free]
    return {"lengths": _to(lengths.astype(np.int32)), "new": _to(new.astype(np.int32)), "tables": _to(tables), "free": _to(free),
            "n_free": _to(np.array([n_free], np.int32))}


def _pages(rng, lengths, block):
    """Tables of shuffled blocks for sequences of these lengths, and the number of blocks of the pool."""
    used = -(-lengths // block)
    n_blocks = int(used.sum()) + 3
    ids = rng.permutation(n_blocks).astype(np.int32)
    tables = np.full((len(lengths), max(1, int(used.max()))), -1, np.int32)
    tables[np.arange(tables.shape[1]) < used[:, None]] = ids[: int(used.sum())]
    return tables, n_blocks


def _codes(shape, kind, gen):
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
    if kind == "int8":
        return (x * 38.0).round_().clamp_(-127, 127).to(torch.int8)
    return (x * 110.0).clamp_(-448, 448).to(torch.float8_e4m3fn)


def _scales(shape, kind, size, gen):
    """What blocks whose largest value is about `size` have."""
    s = torch.rand(shape, generator=gen, device=DEV, dtype=torch.float32) * 0.8 + 0.4
    s = s * (size / Q_MAX[kind])
    return s if kind == "int8" else torch.exp2(torch.ceil(torch.log2(s)))


def _prepare_append(c, seed):
    rng, gen = np.random.default_rng([seed, 2]), _generator(seed)
    R, B, H, D = c["requests"], c["block"], c["kv_heads"], c["dim"]
    sizes = np.random.default_rng([R, B, c["most_new"]])  # how many tokens and blocks there are goes by the case alone
    new = sizes.integers(max(1, c["most_new"] // 2), c["most_new"] + 1, R)
    start = sizes.integers(0, 3 * B, R)
    tables, n_blocks = _pages(rng, start + new, B)
    # the pool of the measurement: the blocks that hold a row of the step, in their shuffled order
    seq = np.repeat(np.arange(R), new)
    pos = np.concatenate([np.arange(s, s + n) for s, n in zip(start, new)])
    block = tables[seq, pos // B]
    touched, block = np.unique(block, return_inverse=True)
    n_blocks, T = len(touched) + 2, len(seq)
    pair = (n_blocks, H, B, D)
    t_max = int(pos.max()) + 1
    angle = np.arange(t_max, dtype=np.float64)[:, None] * 500000.0 ** (-2.0 * np.arange(D // 2) / D)
    table = np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)
    rand = lambda n: torch.randn((T, n * D), generator=gen, device=DEV, dtype=torch.float32) * 2.0  # noqa: E731
    return {"q": rand(c["heads"]), "k": rand(H), "v": rand(H), "positions": _to(pos.astype(np.int32)), "slots": _to((block * B + pos % B).astype(np.int32)),
            "rope": _to(table), "k_cache": _codes(pair, c["kind"], gen), "v_cache": _codes(pair, c["kind"], gen),
            "k_scale": _scales(pair[:2], c["kind"], 8.0, gen), "v_scale": _scales(pair[:2], c["kind"], 8.0, gen)}


def _prepare_attend(c, seed):
    rng, gen = np.random.default_rng([seed, 3]), _generator(seed)
    R, B, H, D = c["requests"], c["block"], c["kv_heads"], c["dim"]
    lo, hi = c["shortest"], c["longest"]
    # ragged batches have many short requests and few long ones
    lengths = np.rint(np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1), R)) - 1).astype(np.int64).clip(lo, hi)
    lengths[rng.integers(0, R)] = hi
    tables, n_blocks = _pages(rng, lengths, B)
    pair = (n_blocks, H, B, D)
    s = {"q": (torch.randn((R, c["heads"] * D), generator=gen, device=DEV) * 2.0).to(torch.bfloat16), "lengths": _to(lengths.astype(np.int32)), "tables": _to(tables),
         "k_cache": _codes(pair, c["kind"], gen), "v_cache": _codes(pair, c["kind"], gen),
         "k_scale": _scales(pair[:2], c["kind"], 2.5, gen), "v_scale": _scales(pair[:2], c["kind"], 2.5, gen)}
    if c["kind"] == "e4m3":  # rows past a sequence's end hold what an earlier request left there, NaN codes at worst
        last = [(tables[r, n // B], n % B) for r, n in enumerate(lengths) if n % B]
        if last:
            b, first = _to(np.array([x[0] for x in last], np.int64)), _to(np.array([x[1] for x in last], np.int64))
            stale = torch.arange(B, device=DEV) >= first[:, None]
            for cache in (s["k_cache"], s["v_cache"]):
                codes = cache.view(torch.uint8)
                codes[b] = torch.where(stale[:, None, :, None], torch.full((), 0x7F, dtype=torch.uint8, device=DEV), codes[b])
    return s


def _prepare_sample(c, seed):
    gen, M = _generator(seed), c["rows"]
    logits = torch.randn((M, c["vocab"]), generator=gen, device=DEV, dtype=torch.float32) * c["spread"]
    s = {"logits": logits, "u": torch.rand(M, generator=gen, device=DEV), "temperature": None, "top_k": None, "top_p": None, "min_p": None}
    rand = lambda lo, hi: torch.rand(M, generator=gen, device=DEV) * (hi - lo) + lo  # noqa: E731
    pick = lambda x, off: torch.where(torch.rand(M, generator=gen, device=DEV) < 0.5, x, torch.full_like(x, off))  # noqa: E731
    if c["filters"] in ("all", "mixed"):
        s["temperature"], s["top_k"] = rand(0.6, 1.2), rand(20.0, 80.0).int()
        s["top_p"], s["min_p"] = rand(0.85, 0.99), rand(0.005, 0.05)
    if c["filters"] == "mixed":
        s["temperature"] = torch.where(torch.rand(M, generator=gen, device=DEV) < 0.2, torch.zeros_like(s["temperature"]), s["temperature"])
        s["top_k"], s["top_p"], s["min_p"] = pick(s["top_k"], 0), pick(s["top_p"], 1.0), pick(s["min_p"], 0.0)
    if c["filters"] == "top_k":
        s["top_k"] = rand(1.0, 1000.0).int()
    if c["filters"] == "top_p":
        s["temperature"], s["top_p"] = rand(0.7, 1.5), rand(0.5, 0.97)
    return s


def prepare(case, seed):
    state = {"tables": _prepare_tables, "append": _prepare_append, "attend": _prepare_attend, "sample": _prepare_sample}[case["op"]](case, seed)
    return {"case": case, **state}


# ------------------------------------------------------------------------------------------------------ plain forms

def _plain_tables(s):
    c, cap, T = s["case"], s["case"]["max_blocks"] * s["case"]["block"], s["case"]["tokens"]
    B, most, n_blocks = c["block"], c["max_blocks"], s["free"].numel()
    lengths, new, n_free = s["lengths"].long(), s["new"].long(), s["n_free"].long()
    R = lengths.numel()
    used = (lengths + B - 1) // B
    gone, adds = new < 0, (new > 0) & (lengths + new <= cap)
    n = torch.where(adds, new, 0)
    need = torch.where(adds, (lengths + n + B - 1) // B - used, 0)
    back = torch.where(gone, used, 0)
    have = n_free + back.sum()
    # the finished requests' blocks go on top of the stack of free ones, in the order of the requests
    column = torch.arange(most, device=DEV)
    back_at = (n_free + torch.cumsum(back, 0) - back)[:, None] + column
    stack = s["free"].clone()
    at = (column < back[:, None]).nonzero(as_tuple=True)
    stack[back_at[at]] = s["tables"][at]
    # requests are served in order while blocks and places for tokens last
    cum_need, cum_n = torch.cumsum(need, 0), torch.cumsum(n, 0)
    ok = adds & (cum_need <= have) & (cum_n <= T)
    served = ok | (new == 0) | gone
    n_ok, need_ok = torch.where(ok, n, 0), torch.where(ok, need, 0)
    fresh = (column >= used[:, None]) & (column < (used + need_ok)[:, None])
    place = have - 1 - ((cum_need - need)[:, None] + column - used[:, None])
    tables = torch.where(fresh, stack[place.clamp(0, n_blocks - 1)], s["tables"])
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(n_ok, 0)])
    t = torch.arange(T, device=DEV)
    live = t < cu[-1]
    r = torch.searchsorted(cu[1:], t, right=True).clamp(max=R - 1)
    pos = lengths[r] + t - cu[r]
    block = tables[r, (pos // B).clamp(0, most - 1)].long()
    minus = torch.full_like(t, -1)
    after = torch.where(gone, 0, lengths + n_ok)
    whole = lambda x: x.to(torch.int32)  # noqa: E731
    return {"tables": tables, "free": stack, "n_free": whole(have - need_ok.sum()), "lengths": whole(after), "served": whole(served), "cu_tokens": whole(cu),
            "seq_ids": whole(torch.where(live, r, minus)), "positions": whole(torch.where(live, pos, minus)),
            "row_lengths": whole(torch.where(live, pos + 1, 0)), "slots": whole(torch.where(live, block * B + pos % B, minus))}


def _rotate(x, cos_sin):
    lo, hi = x.chunk(2, -1)
    c, s = cos_sin[:, None, :, 0], cos_sin[:, None, :, 1]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def _scale_of(amax, kind):
    a = amax.clamp(min=A_MIN)
    if kind == "int8":
        return (a / torch.full_like(a, 127.0)).float()
    m, e = torch.frexp(a)  # the smallest power of two whose 448-fold is no less: 448 = 0.875 * 2^9
    k = torch.where(m <= 0.875, e - 9, e - 8).int()
    return ((k + 127) << 23).view(torch.float32)


def _encode(x, kind):
    """The codes nearest to x (64 bits: a value next to the middle between two codes has to fall to the right one), even ones in the middle."""
    if kind == "int8":
        return x.round().clamp(-127, 127).to(torch.int8)
    step = torch.exp2(torch.frexp(x)[1].clamp(min=-5) - 4.0)
    return ((x / step).round() * step).clamp(-448, 448).to(torch.float8_e4m3fn)


def _store(cache, scale, x, block, where, off, first, kind):
    """Rows x go to `off` of their blocks (`block`: the distinct ones, `where`: each row's).  A block that has earlier rows keeps its scale
    unless a new row needs a larger one; the earlier rows' codes are then brought to it."""
    B = cache.shape[2]
    amax = torch.zeros((len(block), x.shape[1]), device=DEV, dtype=torch.float64).scatter_reduce_(0, where[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
    need, before = _scale_of(amax, kind), scale[block]
    after = torch.where(first[:, None] > 0, torch.maximum(before, need), need)
    tile = cache.view(torch.uint8)[block]
    moved = _encode(tile.view(cache.dtype).double() * before.double()[..., None, None] / after.double()[..., None, None], kind).view(torch.uint8)
    earlier = (torch.arange(B, device=DEV) < first[:, None])[:, None, :, None] & (after > before)[..., None, None]
    tile = torch.where(earlier, moved, tile)
    tile[where, :, off] = _encode(x / after.double()[where][..., None], kind).view(torch.uint8)
    cache.view(torch.uint8)[block] = tile
    scale[block] = after


def _plain_append(s):
    c = s["case"]
    B, D, T = c["block"], c["dim"], s["slots"].numel()
    cos_sin = s["rope"][s["positions"].long()]
    q = _rotate(s["q"].view(T, -1, D), cos_sin)
    k = _rotate(s["k"].view(T, -1, D).double(), cos_sin.double())
    slots = s["slots"].long()
    block, where = torch.unique(slots // B, return_inverse=True)
    first = torch.full_like(block, B).scatter_reduce_(0, where, slots % B, "amin")
    _store(s["k_cache"], s["k_scale"], k, block, where, slots % B, first, c["kind"])
    _store(s["v_cache"], s["v_scale"], s["v"].view(T, -1, D).double(), block, where, slots % B, first, c["kind"])
    return q.reshape(T, -1).to(torch.bfloat16)


def _values(cache, scale):
    if cache.dtype == torch.int8:
        return cache * scale[..., None, None]
    return cache.float() * scale[..., None, None]


def _plain_attend(s):
    c = s["case"]
    R, H, D = c["requests"], c["kv_heads"], c["dim"]
    tables = s["tables"].long().clamp(min=0)
    pick = lambda cache, scale: _values(cache.view(torch.uint8)[tables].view(cache.dtype), scale[tables]).transpose(1, 2).reshape(R, H, -1, D)  # noqa: E731
    k, v = pick(s["k_cache"], s["k_scale"]), pick(s["v_cache"], s["v_scale"])
    live = (torch.arange(k.shape[2], device=DEV) < s["lengths"][:, None])[:, None, None]
    q = s["q"].float().view(R, H, -1, D) / math.sqrt(D)
    score = torch.where(live, q @ k.transpose(2, 3), -math.inf)
    p = torch.where(live, torch.exp(score - score.amax(-1, keepdim=True)), 0.0)
    v = torch.where(live[:, :, 0, :, None], v, 0.0)
    out = (p @ v) / p.sum(-1, keepdim=True)
    out = torch.where((s["lengths"] > 0)[:, None, None, None], out, 0.0)
    return out.reshape(R, -1).to(torch.bfloat16)


def _plain_sample(s):
    logits = s["logits"].double()
    M, V = logits.shape
    full = lambda x, off: torch.full((M, 1), off, device=DEV, dtype=torch.float64) if x is None else x.double()[:, None]  # noqa: E731
    T, top_k, top_p, min_p = full(s["temperature"], 1.0), full(s["top_k"], 0.0), full(s["top_p"], 1.0), full(s["min_p"], 0.0)
    top, order = torch.sort(logits, dim=-1, descending=True, stable=True)  # equal ones: the lowest index first
    greedy = ~(T > 0)
    w = torch.exp((top - top[:, :1]) / torch.where(greedy, 1.0, T))
    rank = torch.arange(V, device=DEV)
    w = torch.where((top_k <= 0) | (rank < top_k), w, 0.0)
    before = torch.cumsum(w, -1) - w
    keep = (rank == 0) | (top_p >= 1) | (before < top_p * w.sum(-1, keepdim=True))
    keep = torch.where(greedy, rank == 0, keep & (w >= min_p))
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))  # the draw goes over the tokens in the order of their ids
    total = torch.cumsum(w, -1)
    target = s["u"].double()[:, None] * total[:, -1:]
    first = ((total <= target).sum(-1, keepdim=True)).clamp(max=V - 1)
    return first[:, 0].to(torch.int32), torch.log(w.gather(1, first) / total[:, -1:])[:, 0].float()


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2504_12285_b200 import binding as bl
    if op == "tables":
        if not own:
            return _plain_tables(s)
        c = s["case"]
        lengths, n_free, served, cu, seq_ids, positions, row_lengths, slots = bl.bitlinear_block_tables(
            s["lengths"], s["new"], s["tables"], s["free"], s["n_free"], c["block"], c["tokens"])
        return {"tables": s["tables"], "free": s["free"], "n_free": n_free, "lengths": lengths, "served": served, "cu_tokens": cu, "seq_ids": seq_ids,
                "positions": positions, "row_lengths": row_lengths, "slots": slots}
    if op == "append":
        c = s["case"]
        if own:
            q = bl.bitlinear_rope_kv8(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["rope"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                                      c["heads"], c["kv_heads"], c["dim"])
        else:
            q = _plain_append(s)
        return {"q": q, "k": _values(s["k_cache"], s["k_scale"]), "v": _values(s["v_cache"], s["v_scale"]), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if op == "attend":
        c = s["case"]
        if not own:
            return _plain_attend(s)
        return bl.bitlinear_attention_decode_kv8(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["tables"], s["lengths"], c["heads"], c["kv_heads"],
                                                 c["dim"])
    if not own:
        return _plain_sample(s)
    return bl.bitlinear_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])


# ------------------------------------------------------------------------------------------------------ what a pass needs

def work(case):
    c = case
    if c["op"] == "tables":
        # lengths in and out, new tokens, flags, offsets; an id per 16 .. 128 tokens read and written; four numbers per token
        return {"bytes": 20.0 * c["requests"] + 16.0 * c["tokens"] + 8.0 * c["tokens"] / c["block"], "flops": 10.0 * c["tokens"]}
    if c["op"] == "append":
        T = c["requests"] * (max(1, c["most_new"] // 2) + c["most_new"]) / 2
        kv, q, D = c["kv_heads"] * c["dim"], c["heads"] * c["dim"], c["dim"]
        # projections in, rotated queries and codes out, one row of the angle table and two indexes for each token
        return {"bytes": T * (4.0 * (q + 2 * kv) + 2.0 * q + 2.0 * kv + 4.0 * D + 8.0), "flops": T * (3.0 * (q + kv) + 4.0 * kv)}
    if c["op"] == "attend":
        lo, hi, R = c["shortest"], c["longest"], c["requests"]
        mean = hi if hi == lo else (hi - lo) / math.log((hi + 1) / (lo + 1))
        rows = (R - 1) * mean + hi  # of all sequences
        return {"bytes": rows * c["kv_heads"] * (2.0 * c["dim"] + 8.0 / c["block"]) + 4.0 * R * c["heads"] * c["dim"], "flops": 4.0 * rows * c["heads"] * c["dim"]}
    return {"bytes": 4.0 * c["rows"] * c["vocab"] + 28.0 * c["rows"], "flops": 10.0 * c["rows"] * c["vocab"]}


# ------------------------------------------------------------------------------------------------------ from the definitions, in 64 bits

def _host(s):
    return {k: v.view(torch.uint8).cpu().numpy() if isinstance(v, torch.Tensor) and v.dtype == torch.float8_e4m3fn else v.cpu().numpy() if isinstance(v, torch.Tensor) else v
            for k, v in s.items()}


def _e4m3_grid():
    """The 127 values of 8 bits with 4 of exponent and 3 of fraction that are no less than zero, by their codes."""
    code = np.arange(127)
    e, f = code >> 3, code & 7
    return np.where(e > 0, (8 + f) * 2.0 ** (e - 10.0), f * 2.0 ** -9)


def _nearest(x, kind):
    """Codes' values nearest to x, the even code where two are as near."""
    if kind == "int8":
        return np.clip(np.rint(x), -127, 127)
    grid, a = _e4m3_grid(), np.minimum(np.abs(x), 448.0)
    up = np.searchsorted(grid, a).clip(1, 126)
    low, high = grid[up - 1], grid[up]
    higher = (a - low > high - a) | ((a - low == high - a) & (up % 2 == 0))
    return np.copysign(np.where(higher, high, low), x)


def _decoded(codes, kind):
    if kind == "int8":
        return codes.astype(np.float64)
    grid = np.append(_e4m3_grid(), np.nan)
    return np.where(codes < 128, 1.0, -1.0) * grid[codes & 127]


def _exact_tables(s):
    c = s["case"]
    B, cap, T = c["block"], c["max_blocks"] * c["block"], c["tokens"]
    h = _host(s)
    tables, free, lengths, R = h["tables"].copy(), h["free"].copy(), h["lengths"].astype(np.int64), c["requests"]
    top = int(h["n_free"][0])
    served, cu, after = np.ones(R, np.int32), np.zeros(R + 1, np.int64), lengths.copy()
    columns = [np.full(T, -1, np.int64), np.full(T, -1, np.int64), np.zeros(T, np.int64), np.full(T, -1, np.int64)]
    for r in np.nonzero(h["new"] < 0)[0]:
        n = -(-int(lengths[r]) // B)
        free[top: top + n] = tables[r, :n]
        top, after[r] = top + n, 0
    t, shut = 0, False
    for r in range(R):
        n, old = int(h["new"][r]), int(lengths[r])
        if n > 0:
            first, last = -(-old // B), -(-(old + n) // B)
            long = old + n > cap
            shut = shut or (not long and (last - first > top or t + n > T))
            served[r] = not (long or shut)
            if served[r]:
                for b in range(first, last):
                    top -= 1
                    tables[r, b] = free[top]
                pos = np.arange(old, old + n)
                for to, what in zip(columns, (r, pos, pos + 1, tables[r, pos // B].astype(np.int64) * B + pos % B)):
                    to[t: t + n] = what
                t, after[r] = t + n, old + n
        cu[r + 1] = t
    i32 = lambda x: np.asarray(x).astype(np.int32)  # noqa: E731
    return {"tables": tables, "free": free, "n_free": i32([top]), "lengths": i32(after), "served": i32(served), "cu_tokens": i32(cu), "seq_ids": i32(columns[0]),
            "positions": i32(columns[1]), "row_lengths": i32(columns[2]), "slots": i32(columns[3])}


def _exact_append(s):
    c, h = s["case"], _host(s)
    B, D, kind = c["block"], c["dim"], c["kind"]
    T = len(h["slots"])
    theta = h["rope"].astype(np.float64)[h["positions"]]
    turn = theta[..., 0] + 1j * theta[..., 1]

    def rotated(x):
        x = x.astype(np.float64).reshape(T, -1, D)
        z = (x[..., : D // 2] + 1j * x[..., D // 2:]) * turn[:, None]
        return np.concatenate([z.real, z.imag], -1)

    out = {"q": rotated(h["q"]).reshape(T, -1)}
    for name, x in (("k", rotated(h["k"])), ("v", h["v"].astype(np.float64).reshape(T, -1, D))):
        codes, scale = _decoded(h[name + "_cache"], kind), h[name + "_scale"].astype(np.float64)
        for b in np.unique(h["slots"] // B):
            rows = np.nonzero(h["slots"] // B == b)[0]
            off = h["slots"][rows] % B
            a = np.maximum(np.abs(x[rows]).max((0, 2)), A_MIN)
            need = (a / 127.0).astype(np.float32).astype(np.float64) if kind == "int8" else 2.0 ** np.ceil(np.log2(a / 448.0))  # codes are multiples of the scale as it is stored
            if off.min() > 0:
                new = np.maximum(scale[b], need)
                codes[b, :, : off.min()] = _nearest(codes[b, :, : off.min()] * (scale[b] / new)[:, None, None], kind)
            else:
                new = need
            codes[b][:, off] = _nearest(x[rows].transpose(1, 0, 2) / new[:, None, None], kind)
            scale[b] = new
        out[name], out[name + "_scale"] = codes * scale[..., None, None], scale
    return {k: out[k] for k in ("q", "k", "v", "k_scale", "v_scale")}


def _exact_attend(s):
    c = s["case"]
    R, G, H, D = c["requests"], c["heads"] // c["kv_heads"], c["kv_heads"], c["dim"]
    out = torch.zeros((R, H, G, D), dtype=torch.float64, device=DEV)
    k_codes, v_codes = (s[n].view(torch.uint8) for n in ("k_cache", "v_cache"))
    value = torch.from_numpy(_decoded(np.arange(256), "e4m3") if c["kind"] == "e4m3" else np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)).to(DEV)
    for r, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        at = torch.arange(n, device=DEV)
        block, off = s["tables"][r].long()[at // c["block"]], at % c["block"]
        k = value[k_codes[block, :, off].long()] * s["k_scale"].double()[block][..., None]
        v = value[v_codes[block, :, off].long()] * s["v_scale"].double()[block][..., None]
        q = s["q"][r].double().view(H, G, D)
        p = torch.softmax(torch.einsum("hgd,nhd->hgn", q, k) / D ** 0.5, -1)
        out[r] = torch.einsum("hgn,nhd->hgd", p, v)
    return out.view(R, -1).cpu().numpy()


def _exact_sample(s):
    h = _host(s)
    M, V = h["logits"].shape
    ids, logp = np.zeros(M, np.int32), np.zeros(M)
    for m in range(M):
        row = h["logits"][m].astype(np.float64)
        get = lambda name, off: off if h[name] is None else float(h[name][m])  # noqa: E731
        T, k, p, low = get("temperature", 1.0), int(get("top_k", 0)), get("top_p", 1.0), get("min_p", 0.0)
        if not T > 0:
            ids[m] = int(np.argmax(row))
            continue
        w = np.exp((row - row.max()) / T)
        kept = np.ones(V, bool)
        if 0 < k < V or p < 1:
            order = np.argsort(-row, kind="stable")
            order = order[:k] if 0 < k < V else order
            if p < 1:
                reached = np.cumsum(w[order])
                order = order[: int(np.searchsorted(reached, p * reached[-1])) + 1]
            kept[:] = False
            kept[order] = True
        w = np.where(kept & (w >= low), w, 0.0)
        total = np.cumsum(w)
        ids[m] = int(np.searchsorted(total, float(h["u"][m]) * total[-1], side="right"))
        logp[m] = math.log(w[ids[m]] / total[-1])
    return ids, logp


def exact(case, seed):
    return {"tables": _exact_tables, "append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](prepare(case, seed))
