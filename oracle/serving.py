"""CPU oracle of the serving operators around a decode step: the bookkeeping of a paged cache, the 8-bit cache with one
scale per block and KV head (append, attention) and the draw of the next token.  TEST INFRASTRUCTURE ONLY (see
oracle/__init__.py).  Everything is the definition of include/bitlinear.h, one request, block or row at a time, in fp64 or
in whole numbers."""
from __future__ import annotations

import math

import numpy as np

INT8, E4M3 = 0, 1


def block_tables(lengths, new_tokens, tables, free_blocks, n_free, block_rows, t_cap):
    """One step of the bookkeeping; returns a dict of the state after it and of what the step lays out."""
    R, max_blocks = tables.shape
    cap = max_blocks * block_rows
    tables, stack = tables.copy(), list(free_blocks[:n_free])
    lengths = [min(max(int(x), 0), cap) for x in lengths]
    used = [-(-n // block_rows) for n in lengths]
    for r in range(R):
        if new_tokens[r] < 0:
            stack += list(tables[r, :used[r]])
    out = {"served": np.ones(R, np.int32), "cu_tokens": np.zeros(R + 1, np.int32)}
    rows, pushed = [], list(stack)
    full = False
    for r in range(R):
        n = int(new_tokens[r])
        if n > 0:
            need = -(-(lengths[r] + n) // block_rows) - used[r]
            fits = lengths[r] + n <= cap
            if fits and (need > len(stack) or len(rows) + n > t_cap):
                full = True
            if not fits or full:
                out["served"][r] = 0
            else:
                for b in range(used[r], used[r] + need):
                    tables[r, b] = stack.pop()
                for p in range(lengths[r], lengths[r] + n):
                    block = int(tables[r, p // block_rows])
                    inside = 0 <= block < len(free_blocks)
                    rows.append((r, p, p + 1, block * block_rows + p % block_rows if inside else -1))
                lengths[r] += n
        elif n < 0:
            lengths[r] = 0
        out["cu_tokens"][r + 1] = len(rows)
    cols = np.tile(np.array([[-1], [-1], [0], [-1]], np.int32), (1, t_cap))
    if rows:
        cols[:, :len(rows)] = np.array(rows, np.int64).T
    free = free_blocks.copy()
    free[n_free:len(pushed)] = pushed[n_free:len(free)]  # a stack never grows past its array
    return {**out, "tables": tables, "free_blocks": free, "n_free": min(len(stack), len(free)), "lengths": np.array(lengths, np.int32), "seq_ids": cols[0],
            "positions": cols[1], "row_lengths": cols[2], "slots": cols[3]}


_E4M3 = np.array([(f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)) for e in range(16) for f in range(8)])
_E4M3[127] = np.nan


def decode(codes: np.ndarray, kind: int) -> np.ndarray:
    """The numbers that codes (uint8 bit patterns) stand for, without their scale."""
    if kind == INT8:
        return codes.view(np.int8).astype(np.float64)
    return np.where(codes & 0x80, -1.0, 1.0) * _E4M3[codes & 0x7f]


def encode(x: np.ndarray, kind: int) -> np.ndarray:
    """The nearest codes, ties to even, beyond the range the range's end (uint8 bit patterns)."""
    if kind == INT8:
        return np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
    a = np.abs(x)
    order = np.searchsorted(_E4M3[:127], a)  # the first code whose value is no less
    hi = np.minimum(order, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _E4M3[lo], _E4M3[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    code = np.where(a >= 448.0, 126, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_for(amax: float, kind: int) -> np.float32:
    if not math.isfinite(amax):
        return np.float32(np.nan)
    a = max(float(amax), 1e-30)
    if kind == INT8:
        return np.float32(a / 127.0)
    s = 2.0 ** math.floor(math.log2(a / 448.0))
    while 448.0 * s < a:
        s *= 2.0
    while 448.0 * (s / 2.0) >= a:
        s /= 2.0
    return np.float32(s)


def rotate(x: np.ndarray, positions: np.ndarray, table: np.ndarray) -> np.ndarray:
    """x [T, heads, D] (fp32 values, taken exactly) turned by the fp32 (cos, sin) pairs of the table, in fp64."""
    half = x.shape[-1] // 2
    lo, hi = x[..., :half].astype(np.float64), x[..., half:].astype(np.float64)
    c, s = table[positions, :, 0].astype(np.float64)[:, None], table[positions, :, 1].astype(np.float64)[:, None]
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)


def append8(values, slots, codes, scale, kind):
    """Rows `values` (fp64 [T, n_kv, D]) into a pool (codes uint8 [n_blocks, n_kv, rows, D], scale fp32 [n_blocks, n_kv]), in place.
    Tokens with a negative slot are not stored."""
    rows = codes.shape[2]
    for b in sorted({int(s) // rows for s in slots if s >= 0}):
        mine = [t for t, s in enumerate(slots) if s >= 0 and s // rows == b]
        off = [int(slots[t]) % rows for t in mine]
        first = min(off)
        for h in range(codes.shape[1]):
            need = scale_for(np.abs(values[mine, h]).max(), kind)
            old = scale[b, h]
            new = need if first == 0 else np.maximum(old, need)  # NaN if either is
            if first > 0 and new > old:
                codes[b, h, :first] = encode(decode(codes[b, h, :first], kind) * float(old) / float(new), kind)
            codes[b, h, off] = 0 if np.isnan(new) else encode(values[mine, h] / float(new), kind)
            scale[b, h] = new


def attention8(q, k_codes, v_codes, k_scale, v_scale, table, length, n_q, n_kv, D, kind):
    """One query row (fp64 [n_q, D]) against the first `length` rows that the table names; rows of ids outside the pool are left
    out.  Returns (result [n_q, D], the largest value magnitude, a bound on the scores' error in fp32)."""
    n_blocks, rows = k_codes.shape[0], k_codes.shape[2]
    at = [(int(table[t // rows]), t % rows) for t in range(length)]
    at = [x for x in at if 0 <= x[0] < n_blocks]
    out = np.zeros((n_q, D))
    if not at:
        return out, 0.0, 0.0
    b, r = np.array(at).T
    k = decode(k_codes[b, :, r], kind) * k_scale[b].astype(np.float64)[..., None]
    v = decode(v_codes[b, :, r], kind) * v_scale[b].astype(np.float64)[..., None]
    worst = 0.0
    for h in range(n_q):
        g = h // (n_q // n_kv)
        s = k[:, g] @ q[h] / math.sqrt(D)
        p = np.exp(s - s.max())
        out[h] = (p / p.sum()) @ v[:, g]
        if kind == INT8:
            # queries in units of 1 / (16256 * 256) of the head's largest: half a unit by rounding, half by the two fp32 roundings (2^-24 each)
            # of a quotient of at most 2^22 units.  Sums are whole numbers; ten fp32 roundings of the score and of what scales it
            err = float(np.abs(k[:, g]).sum(-1).max() * np.abs(q[h]).max()) / (16256 * 256) / math.sqrt(D) + 10 * 2.0 ** -24 * float(np.abs(s).max())
        else:
            # D products in fp32, each addition off by 2^-23 at most (the tensor cores may cut instead of round), and three roundings
            # of the scaled score
            err = (D + 4) * 2.0 ** -23 * float((np.abs(k[:, g]) @ np.abs(q[h])).max()) / math.sqrt(D)
        worst = max(worst, err)
    return out, float(np.abs(v).max()), worst


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(id, log probability) of one row."""
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    V, top = len(l), l.max()
    if top == -np.inf:
        return -1, -np.inf
    if not temperature > 0:
        return int(np.argmax(l)), 0.0
    if top == np.inf:
        w = (l == np.inf).astype(np.float64)
    else:
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(l == -np.inf, 0.0, np.exp((l - top) / float(temperature)))
    ranked = sorted(range(V), key=lambda i: (-l[i], i)) if V <= 5000 else list(np.lexsort((np.arange(V), -l)))
    if 0 < top_k < V:
        ranked = ranked[:top_k]
    if top_p < 1:
        goal, run, n = float(top_p) * math.fsum(w[ranked]), 0.0, 0
        sums = np.cumsum(w[ranked])
        n = int(np.searchsorted(sums, goal, side="left")) + 1 if goal > 0 else 1
        ranked = ranked[:max(1, n)]
    least = min(float(min_p), 1.0) if min_p > 0 else 0.0
    kept = np.zeros(V)
    idx = np.array(ranked)
    kept[idx] = np.where(w[idx] >= least, w[idx], 0.0)
    sums = np.cumsum(kept)
    goal = min(max(float(u), 0.0), 1.0) * sums[-1]
    i = int(np.searchsorted(sums, goal, side="right"))
    if i >= V or goal >= sums[-1]:
        i = int(np.nonzero(kept)[0][-1])
    return i, math.log(kept[i] / sums[-1])
