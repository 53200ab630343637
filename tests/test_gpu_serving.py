"""The serving operators (block tables, 8-bit cache append and attention, sampling) against their 64-bit oracle.

Whole numbers, codes, scales and chosen tokens have to be equal: the kernels form what decides them in 64 bits, as the oracle
does.  Tolerances of the floating-point results are derived where they are used."""
import math

import numpy as np
import pytest
import torch

from oracle import decode_step as ds
from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from paper_2504_12285_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = [sv.INT8, sv.E4M3]
DTYPE = {sv.INT8: torch.int8, sv.E4M3: torch.float8_e4m3fn}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def host(t):
    return (t.view(torch.uint8) if t.dtype in (torch.int8, torch.float8_e4m3fn) else t).cpu().numpy()


# ------------------------------------------------------------------------------------------------- block tables

def tables_case(R, max_blocks, rows, seed, shortage=0, decode=False, longest=None):
    """A consistent state: every block is in one table or on the stack of free ones."""
    rng = np.random.default_rng(seed)
    cap = max_blocks * rows
    lengths = rng.integers(0, cap + 1, R)
    new = np.ones(R, np.int64) if decode else rng.integers(-1, 3 * rows if longest is None else longest, R)
    new[rng.random(R) < 0.1] = 0
    new[rng.random(R) < 0.1] = -1
    used = -(-lengths // rows)
    need = np.where((new > 0) & (lengths + new <= cap), -(-(lengths + np.maximum(new, 0)) // rows) - used, 0)
    n_free = max(0, int(need.sum()) - int(used[new < 0].sum()) - shortage)
    n_blocks = int(used.sum()) + n_free + 1
    ids = rng.permutation(n_blocks).astype(np.int32)
    tables = np.full((R, max_blocks), -7, np.int32)
    tables[np.arange(max_blocks) < used[:, None]] = ids[:used.sum()]
    free = np.full(n_blocks, -5, np.int32)
    free[:n_free] = ids[used.sum():used.sum() + n_free]
    return lengths.astype(np.int32), new.astype(np.int32), tables, free, n_free


def check_tables(lengths, new, tables, free, n_free, rows, t_cap, in_place=False):
    want = sv.block_tables(lengths, new, tables, free, n_free, rows, t_cap)
    ld, td, fd, nd = dev(lengths), dev(tables), dev(free), dev(np.array([n_free], np.int32))
    kw = dict(lengths_out=ld, n_free_out=nd) if in_place else {}
    got = bl.bitlinear_block_tables(ld, dev(new), td, fd, nd, rows, t_cap, **kw)
    got = dict(zip(("lengths", "n_free", "served", "cu_tokens", "seq_ids", "positions", "row_lengths", "slots"), got))
    assert int(got.pop("n_free")[0]) == want["n_free"]
    for name, t in {**got, "tables": td, "free_blocks": fd}.items():
        assert np.array_equal(host(t), want[name]), name
    if not in_place:
        assert np.array_equal(host(ld), lengths) and int(nd[0]) == n_free
    return want


@pytest.mark.parametrize("R,max_blocks,rows", [(1, 1, 1), (1, 5, 16), (3, 4, 64), (16, 64, 64), (37, 9, 7), (128, 3, 32), (129, 12, 16), (700, 5, 128), (2500, 3, 16)])
@pytest.mark.parametrize("in_place", [False, True])
def test_block_tables(R, max_blocks, rows, in_place):
    for seed, kw in enumerate((dict(), dict(decode=True), dict(shortage=2), dict(shortage=10 ** 6), dict(longest=max_blocks * rows + 3))):
        case = tables_case(R, max_blocks, rows, 100 * R + seed, **kw)
        tokens = int(np.maximum(case[1], 0).sum())
        for t_cap in sorted({0, R, tokens, max(0, tokens - 1), tokens // 2 + 3, tokens + 5}):
            check_tables(*case, rows, t_cap, in_place)


def test_block_tables_no_requests_and_bad_state():
    check_tables(np.zeros(0, np.int32), np.zeros(0, np.int32), np.zeros((0, 4), np.int32), np.arange(3, dtype=np.int32), 2, 16, 9)
    # lengths outside the table, a huge new_tokens, ids outside the pool, a stack height outside its array: counted as the nearest
    # valid, refused, or marked -1; nothing is written out of place
    tables = np.array([[3, 99, -1, -1], [0, 1, 2, -4], [4, -1, -1, -1]], np.int32)
    check_tables(np.array([17, 64, -9], np.int32), np.array([1, 2 ** 31 - 1, 3], np.int32), tables, np.array([5, 6, 7, 8, 9, 0, 0, 0, 0, 0], np.int32), 5, 16, 8)
    check_tables(np.array([20, 70, 3], np.int32), np.array([-1, -1, 5], np.int32), tables, np.array([5, 6, 7, 8, 9, 0, 0, 0, 0, 0], np.int32), 5, 16, 8)
    ld, td, fd = dev(np.array([0], np.int32)), dev(np.full((1, 4), -1, np.int32)), dev(np.arange(3, dtype=np.int32))
    out = bl.bitlinear_block_tables(ld, dev(np.array([40], np.int32)), td, fd, dev(np.array([99], np.int32)), 16, 40)
    assert host(td).tolist() == [[2, 1, 0, -1]] and int(out[1][0]) == 0


def test_block_tables_many_requests():
    for in_place in (False, True):
        case = tables_case(20000, 6, 16, 6, shortage=5)
        check_tables(*case, 16, int(np.maximum(case[1], 0).sum()) - 1000, in_place)


def test_block_tables_large_step_is_the_same_every_time():
    case = tables_case(3000, 40, 16, 5, longest=200)
    tokens = int(np.maximum(case[1], 0).sum())
    want = check_tables(*case, 16, tokens)
    assert want["cu_tokens"][-1] > 100000
    for _ in range(3):
        check_tables(*case, 16, tokens, in_place=True)


# ------------------------------------------------------------------------------------------------- append

def make_pool(n_blocks, n_kv, rows, D, kind, seed, size=6.0):
    rng = np.random.default_rng(seed)
    shape = (n_blocks, n_kv, rows, D)
    codes = [sv.encode(rng.standard_normal(shape) * (40.0 if kind == sv.INT8 else 100.0), kind) for _ in range(2)]
    scales = [np.array([[sv.scale_for(a, kind) for a in row] for row in rng.uniform(0.3, 1.2, shape[:2]) * size], np.float32) for _ in range(2)]
    return codes, scales


def pool_to_dev(codes, scales, kind):
    return [dev(c).view(DTYPE[kind]) for c in codes] + [dev(s) for s in scales]


def check_append(kind, n_q, n_kv, D, rows, slots, positions, seed, size=2.0, n_blocks=None, t_max=512):
    slots, positions = np.asarray(slots, np.int32), np.asarray(positions, np.int32)
    T = len(slots)
    n_blocks = n_blocks or int(max(slots.max(initial=0), 0)) // rows + 2
    rng = np.random.default_rng(seed)
    q, k, v = ((rng.standard_normal((T, h * D)) * size).astype(np.float32) for h in (n_q, n_kv, n_kv))
    if T > 2:
        k[1], v[1] = 0.0, 0.0
        v[2] *= 30.0  # a row that makes its block's scale grow
    codes, scales = make_pool(n_blocks, n_kv, rows, D, kind, seed + 1)
    pool = pool_to_dev(codes, scales, kind)
    table = bl.bitlinear_rope_table(D, t_max, device=DEV)
    out = bl.bitlinear_rope_kv8(dev(q), dev(k), dev(v), dev(positions), dev(slots), table, *pool, n_q, n_kv, D)
    torch.cuda.synchronize()
    tab = host(table)
    placed = (positions >= 0) & (positions < t_max)
    stored = np.where(placed & (slots >= 0) & (slots < n_blocks * rows), slots, -1)
    at = np.where(placed, positions, 0)
    sv.append8(sv.rotate(k.reshape(T, n_kv, D), at, tab), stored, codes[0], scales[0], kind)
    sv.append8(v.reshape(T, n_kv, D).astype(np.float64), stored, codes[1], scales[1], kind)
    for got, want, name in zip(pool, codes + scales, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(host(got), want), name  # codes and scales bit for bit; rows of others untouched
    # q: the fp32 operations of the other append calls, one rounding to bf16: half a bf16 step and three fp32 roundings of the pair;
    # below 2^-126 bf16 values are 2^-133 apart whatever their size, so half a step is 2^-134 there (and fp32's 2^-150)
    ref = sv.rotate(q.reshape(T, n_q, D), at, tab).reshape(T, -1) * placed[:, None]
    qn = out.float().cpu().numpy().astype(np.float64)
    assert np.all(np.abs(qn - ref) <= 2.0 ** -8 * np.abs(ref) + 3 * 2.0 ** -24 * 2 * float(np.abs(q).max()) + 1.01 * 2.0 ** -134)
    return out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_kv,D,rows", [(20, 5, 128, 64), (4, 2, 64, 16), (8, 1, 128, 32), (3, 3, 64, 128)])
def test_append_one_token_per_sequence(kind, n_q, n_kv, D, rows):
    rng = np.random.default_rng(rows)
    T = 9
    blocks = rng.permutation(T + 3)[:T]
    off = rng.integers(0, rows, T)
    off[:3] = [0, rows - 1, 5]
    check_append(kind, n_q, n_kv, D, rows, blocks * rows + off, off + rows * rng.integers(0, 3, T), 11)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,rows,runs", [
    (128, 64, [(0, 64)]),                               # one whole block
    (128, 16, [(3, 40), (0, 1), (15, 2), (7, 9)]),      # runs that start and end inside blocks
    (64, 128, [(100, 300), (1, 127)]),
    (128, 32, [(0, 700), (31, 33), (16, 16)]),          # more tokens than a launch gives a CTA each
    (64, 16, [(i % 16, 1 + i % 5) for i in range(90)]),
])
def test_append_runs_of_tokens(kind, D, rows, runs):
    rng = np.random.default_rng(len(runs))
    used = [-(-(s + n) // rows) for s, n in runs]
    ids = rng.permutation(sum(used) + 2)
    slots, pos, b = [], [], 0
    for (s, n), u in zip(runs, used):
        p = np.arange(s, s + n)
        slots += list(ids[b + p // rows] * rows + p % rows)
        pos += list(p)
        b += u
    check_append(kind, 4, 2, D, rows, slots, pos, 21, n_blocks=sum(used) + 2, t_max=1024)


@pytest.mark.parametrize("kind", KINDS)
def test_append_leaves_out_what_has_no_place(kind):
    rows = 16
    # padding, slots past the pool, positions past the table of angles, a run interrupted by padding at its end
    slots = [16 * 3 + 4, 16 * 3 + 5, -1, 16 * 1, 10 ** 6, 16 * 2 + 7, 16 * 2 + 8, -1, -1, 16 * 5 + 1]
    pos = [4, 5, -1, 32, 3, 100, 99, 7, -1, -1]
    out = check_append(kind, 4, 2, 64, rows, slots, pos, 31, n_blocks=7, t_max=100)
    assert not out[2].any() and not out[5].any() and not out[8].any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("size", [0.0, 1e-38, 1e-20, 1e4, 1e30])
def test_append_extreme_magnitudes(kind, size):
    check_append(kind, 4, 2, 64, 16, [16, 17, 40, 41, 3], [0, 1, 8, 9, 3], 41, size=size, n_blocks=4)


@pytest.mark.parametrize("kind", KINDS)
def test_append_keeps_any_scale_and_survives_fp32_overflow(kind):
    """A block whose scale something else wrote (no power of two, far larger than needed), and keys whose rotation leaves fp32."""
    n_kv, D, rows, T = 2, 64, 16, 24
    rng = np.random.default_rng(5)
    k, v = ((rng.standard_normal((T, n_kv * D)) * 3).astype(np.float32) for _ in range(2))
    k[16:] = np.sign(k[16:]) * np.float32(3.3e38)
    slots = np.array([16 * (t // 4) + 3 + t % 4 for t in range(T)], np.int32)
    pos = rng.integers(0, 200, T).astype(np.int32)
    codes, scales = make_pool(7, n_kv, rows, D, kind, 6)
    for s in scales:
        s[:3] = rng.uniform(0.01, 0.7, (3, n_kv)).astype(np.float32)
    pool = pool_to_dev(codes, scales, kind)
    table = bl.bitlinear_rope_table(D, 200, device=DEV)
    bl.bitlinear_rope_kv8(torch.zeros(T, 4 * D, device=DEV), dev(k), dev(v), dev(pos), dev(slots), table, *pool, 4, n_kv, D)
    with np.errstate(over="ignore"):
        sv.append8(sv.rotate(k.reshape(T, n_kv, D), pos, host(table)), slots, codes[0], scales[0], kind)
        sv.append8(v.reshape(T, n_kv, D).astype(np.float64), slots, codes[1], scales[1], kind)
    for got, want in zip(pool, codes + scales):
        assert np.array_equal(host(got), want)


@pytest.mark.parametrize("kind", KINDS)
def test_append_rounds_the_middle_to_even(kind):
    # values exactly in the middle between two codes: position 0 turns nothing, so they arrive as given
    D, rows = 64, 16
    base = np.arange(D, dtype=np.float64)
    if kind == sv.INT8:
        v = (base - 32 + 0.5).astype(np.float32) * 0.25
        v[0] = 127 * 0.25  # the scale is 0.25
    else:
        grid = sv.decode(np.arange(0, 127, dtype=np.uint8), kind)
        mid = (grid[:-1] + grid[1:]) / 2
        v = mid[np.linspace(0, len(mid) - 1, D).astype(int)].astype(np.float32)
        v[0] = 448.0
    kv = np.stack([v, -v])
    codes, scales = make_pool(2, 1, rows, D, kind, 1)
    pool = pool_to_dev(codes, scales, kind)
    table = bl.bitlinear_rope_table(D, 4, device=DEV)
    pos = dev(np.array([0, 0], np.int32))
    bl.bitlinear_rope_kv8(dev(kv), dev(kv), dev(kv), pos, dev(np.array([0, 1], np.int32)), table, *pool, 1, 1, D)
    want = sv.encode(kv.astype(np.float64) / (0.25 if kind == sv.INT8 else 1.0), kind)
    assert np.array_equal(host(pool[0])[0, 0, :2], want) and np.array_equal(host(pool[1])[0, 0, :2], want)


# ------------------------------------------------------------------------------------------------- attention

def attend_case(kind, n_q, n_kv, D, rows, lengths, seed, seq_ids=None, n_seq=None, slack_blocks=2):
    rng = np.random.default_rng(seed)
    n_seq = n_seq or len(lengths)
    seq = np.arange(len(lengths)) if seq_ids is None else np.asarray(seq_ids)
    longest = max(1, max(lengths))
    per = -(-longest // rows) + slack_blocks
    n_blocks = n_seq * per + 2
    tables = rng.permutation(n_blocks)[:n_seq * per].reshape(n_seq, per).astype(np.int32)
    codes, scales = make_pool(n_blocks, n_kv, rows, D, kind, seed + 1, size=2.5)
    # rows that no length covers hold the worst bits there are
    live = np.zeros((n_blocks, rows), bool)
    for m, n in enumerate(lengths):
        if 0 <= seq[m] < n_seq:
            t = np.arange(max(n, 0))
            live[tables[seq[m]][t // rows], t % rows] = True
    for c in codes:
        c[np.broadcast_to(~live[:, None, :, None], c.shape)] = 0x7f if kind == sv.E4M3 else 0x80
    dead = ~live.any(1)
    for s in scales:
        s[dead] = np.nan
    q = torch.randn(len(lengths), n_q * D, generator=torch.Generator().manual_seed(seed)) * 2.0
    return q.to(torch.bfloat16), codes, scales, tables


def check_attention(got, q, codes, scales, tables, lengths, n_q, n_kv, D, kind, seq_ids=None):
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    qn = q.float().numpy().astype(np.float64)
    rows = codes[0].shape[2]
    for m, n in enumerate(lengths):
        s = m if seq_ids is None else seq_ids[m]
        n = min(max(n, 0), tables.shape[1] * rows) if 0 <= s < len(tables) else 0
        ref, vmax, err = sv.attention8(qn[m].reshape(n_q, D), *codes, *scales, tables[s if n else 0], n, n_q, n_kv, D, kind)
        # the result's rounding to bf16 (2^-8 of it), the weights' to f16 (2^-11 of each, so of the largest value) and the fp32
        # scores' error, which moves weights by as much twice over; 1e-6 for the fp32 sums behind it
        tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2 * err + 1e-6) * vmax
        assert np.all(np.abs(got[m].reshape(n_q, D) - ref) <= tol), (m, n, np.abs(got[m].reshape(n_q, D) - ref).max(), vmax)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_kv,D,rows,lengths", [
    (20, 5, 128, 64, [4096]),
    (20, 5, 128, 64, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 300, 1000]),
    (20, 5, 128, 16, [1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 500, 0, 7]),
    (4, 2, 64, 16, [5, 64, 65, 513]),
    (16, 2, 64, 128, [1, 127, 128, 129, 700]),
    (8, 1, 128, 32, [33, 1, 2000]),
    (3, 3, 64, 32, [90, 0, 1]),
    (7, 1, 128, 128, [257]),
    (6, 2, 128, 16, [0]),
])
def test_attention(kind, n_q, n_kv, D, rows, lengths):
    q, codes, scales, tables = attend_case(kind, n_q, n_kv, D, rows, lengths, 51)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)), n_q, n_kv, D)
    torch.cuda.synchronize()
    assert bl.bitlinear_poll_status() == 0
    check_attention(out, q, codes, scales, tables, lengths, n_q, n_kv, D, kind)


@pytest.mark.parametrize("kind", KINDS)
def test_attention_many_rows_of_all_lengths(kind):
    # more rows than a warp scans at once, short and long mixed, so that runs begin and end everywhere
    rng = np.random.default_rng(3)
    lengths = [int(x) for x in np.exp(rng.uniform(0, np.log(3000), 150))]
    lengths[7] = lengths[40] = 0
    q, codes, scales, tables = attend_case(kind, 4, 2, 64, 32, lengths, 61)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)), 4, 2, 64)
    check_attention(out, q, codes, scales, tables, lengths, 4, 2, 64, kind)
    assert bl.bitlinear_poll_status() == 0


@pytest.mark.parametrize("kind", KINDS)
def test_attention_more_rows_than_a_batch_of_lengths(kind):
    rng = np.random.default_rng(4)
    lengths = [int(x) for x in rng.integers(0, 40, 700)]
    lengths[300] = 900
    q, codes, scales, tables = attend_case(kind, 2, 1, 64, 16, lengths, 63, slack_blocks=0)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)), 2, 1, 64)
    check_attention(out, q, codes, scales, tables, lengths, 2, 1, 64, kind)


@pytest.mark.parametrize("kind,D", [(sv.INT8, 64), (sv.E4M3, 128)])
def test_attention_long_sequence(kind, D):
    lengths = [150001, 3]
    q, codes, scales, tables = attend_case(kind, 6, 2, D, 128, lengths, 64)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)), 6, 2, D)
    check_attention(out, q, codes, scales, tables, lengths, 6, 2, D, kind)
    assert bl.bitlinear_poll_status() == 0


@pytest.mark.parametrize("kind", KINDS)
def test_attention_rows_of_one_sequence_and_missing_ones(kind):
    lengths = [10, 11, 12, 400, 5, -3, 10 ** 6, 77]
    seq = [0, 0, 0, 1, 9, 1, 1, -1]
    n = 2
    plain = [10, 11, 12, 400, 0, 0, 420, 0]  # row 6's length is taken as its table's end
    q, codes, scales, tables = attend_case(kind, 4, 1, 128, 16, plain, 71, seq_ids=[0, 0, 0, 1, -1, 1, 1, -1], n_seq=n, slack_blocks=0)
    lengths[6] = 10 ** 6
    last = tables.shape[1] * 16
    plain[6] = last
    for c in codes:  # make every row of sequence 1 a live one
        c[tables[1]] = sv.encode(np.random.default_rng(5).standard_normal(c[tables[1]].shape) * 30, kind)
    for s in scales:
        s[tables[1]] = sv.scale_for(3.0, kind)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)), 4, 1, 128,
                                            seq_ids=dev(np.array(seq, np.int32)))
    check_attention(out, q, codes, scales, tables, lengths, 4, 1, 128, kind, seq_ids=seq)
    assert not out[4].any() and not out[5].any() and not out[7].any()


@pytest.mark.parametrize("rows", [16, 64])
def test_attention_leaves_out_blocks_that_are_not_in_the_pool(rows):
    lengths = [100, 200, 64]
    q, codes, scales, tables = attend_case(sv.INT8, 4, 2, 64, rows, lengths, 81)
    tables[0, 1] = -1
    tables[1, 0] = len(codes[0])
    tables[1, 2] = 2 ** 31 - 1
    tables[2, :] = -1
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, sv.INT8), dev(tables), dev(np.array(lengths, np.int32)), 4, 2, 64)
    check_attention(out, q, codes, scales, tables, lengths, 4, 2, 64, sv.INT8)
    assert not out[2].any()


@pytest.mark.parametrize("kind", KINDS)
def test_attention_block_scales_far_apart(kind):
    """Scales that differ by many powers of two between blocks, all-zero blocks among them, and queries of tiny and large size."""
    lengths = [300, 300, 300]
    q, codes, scales, tables = attend_case(kind, 4, 1, 64, 16, lengths, 91)
    rng = np.random.default_rng(9)
    scales[0][tables] = (2.0 ** rng.integers(-12, -5, tables.shape + (1,))).astype(np.float32)
    scales[1][tables] = (2.0 ** rng.integers(-20, 4, tables.shape + (1,))).astype(np.float32)
    for c, s in zip(codes, scales):
        c[tables[:, 0]] = 0
        s[tables[:, 0]] = sv.scale_for(0.0, kind)
    q = q.float()
    q[1] *= 1e-30
    q[2] *= 4.0
    q = q.to(torch.bfloat16)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)), 4, 1, 64)
    check_attention(out, q, codes, scales, tables, lengths, 4, 1, 64, kind)


def test_attention_hand_cases():
    n_q, n_kv, D, rows = 4, 2, 64, 16
    lengths = [1, 25, 0]
    q, codes, scales, tables = attend_case(sv.INT8, n_q, n_kv, D, rows, lengths, 95)
    q[1] = 0
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, sv.INT8), dev(tables), dev(np.array(lengths, np.int32)), n_q, n_kv, D)
    out = out.float().cpu().numpy().astype(np.float64).reshape(3, n_q, D)
    v = sv.decode(codes[1], sv.INT8) * scales[1].astype(np.float64)[..., None, None]
    first = v[tables[0, 0], 1, 0]
    assert np.all(np.abs(out[0, 3] - first) <= 2.0 ** -8 * np.abs(first))  # one row: its value
    mean = np.concatenate([v[tables[1, 0], 0], v[tables[1, 1], 0, :9]]).mean(0)  # a zero query: the mean
    assert np.all(np.abs(out[1, 0] - mean) <= 2.0 ** -8 * np.abs(mean) + 2.0 ** -11 * np.abs(v[tables[1, :2], 0]).max())
    assert not out[2].any()


def test_attention_far_offsets():
    """A pool of more than 2^32 bytes: its last blocks are read where they lie."""
    n_kv, D, rows, n_blocks = 5, 128, 128, 53000  # 4.3 GB each for keys and values
    pool = [torch.zeros(n_blocks, n_kv, rows, D, dtype=torch.int8, device=DEV) for _ in range(2)]
    scale = [torch.full((n_blocks, n_kv), 0.02, device=DEV) for _ in range(2)]
    gen = torch.Generator(DEV).manual_seed(3)
    tables = np.array([[n_blocks - 1, 0, n_blocks - 7]], np.int32)
    for c in pool:
        for b in tables[0]:
            c[b] = torch.randint(-127, 128, c[b].shape, generator=gen, device=DEV).to(torch.int8)
    q = torch.randn(1, 20 * D, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool, *scale, dev(tables), dev(np.array([300], np.int32)), 20, n_kv, D)
    small = [host(c[torch.from_numpy(tables[0].astype(np.int64)).to(DEV)]) for c in pool]
    check_attention(out, q, small, [host(s[:3]) for s in scale], np.array([[0, 1, 2]], np.int32), [300], 20, n_kv, D, sv.INT8)
    # and the append finds them too
    k = torch.randn(1, n_kv * D, generator=torch.Generator().manual_seed(5)).to(DEV)
    table = bl.bitlinear_rope_table(D, 512, device=DEV)
    bl.bitlinear_rope_kv8(torch.zeros(1, 20 * D, device=DEV), k, k, dev(np.array([300], np.int32)), dev(np.array([(n_blocks - 7) * rows + 44], np.int32)), table,
                          *pool, *scale, 20, n_kv, D)
    got = host(pool[1][n_blocks - 7, :, 44])
    want_codes, want_scale = small[1][2:3].copy(), np.full((1, n_kv), 0.02, np.float32)
    sv.append8(k.cpu().numpy().reshape(1, n_kv, D).astype(np.float64), [44], want_codes, want_scale, sv.INT8)
    assert np.array_equal(got, want_codes[0, :, 44])


# ------------------------------------------------------------------------------------------------- sampling

def check_sample(logits, u, dtype=torch.float32, strided=False, **filters):
    logits = np.asarray(logits, np.float32)
    M, V = logits.shape
    t = torch.from_numpy(logits).to(dtype)
    seen = t.float().numpy()
    if strided:
        wide = torch.full((M, V + 13), 77.0, dtype=dtype)
        wide[:, 5:5 + V] = t
        t = wide.to(DEV)[:, 5:5 + V]
    else:
        t = t.to(DEV)
    u = np.asarray(u, np.float32)
    kinds = {"temperature": np.float32, "top_k": np.int32, "top_p": np.float32, "min_p": np.float32}
    given = {n: np.broadcast_to(np.asarray(x, kinds[n]), M).copy() for n, x in filters.items()}
    ids, logp = bl.bitlinear_sample(t, dev(u), **{n: dev(x) for n, x in given.items()})
    ids, logp = host(ids), host(logp).astype(np.float64)
    for m in range(M):
        want, lp = sv.sample(seen[m], u[m], **{n: x[m] for n, x in given.items()})
        assert ids[m] == want, (m, ids[m], want, {n: x[m] for n, x in given.items()}, u[m])
        # one fp32 rounding of the logarithm; weights and sums are exact to 2^-44 of the largest weight
        assert logp[m] == lp or abs(logp[m] - lp) <= 2.0 ** -23 * abs(lp) + V * 2.0 ** -43, (m, logp[m], lp)


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=1.3, top_k=50, top_p=0.95, min_p=0.02),
           dict(top_k=1), dict(top_p=0.0), dict(min_p=1.0), dict(temperature=0.0), dict(temperature=0.05, top_p=0.999), dict(temperature=30.0, top_k=400, top_p=0.3)]


@pytest.mark.parametrize("V", [1, 2, 31, 513, 2048, 2049, 4999])
@pytest.mark.parametrize("filters", FILTERS)
def test_sample(V, filters):
    rng = np.random.default_rng(V)
    check_sample(rng.standard_normal((6, V)) * 2.5, rng.random(6), **filters)


@pytest.mark.parametrize("V", [128256, 50001, bl.SAMPLE_MAX_VOCAB])
@pytest.mark.parametrize("filters", [dict(), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.02), dict(top_p=0.9), dict(top_k=3000, temperature=1.7)])
def test_sample_large_vocabulary(V, filters):
    rng = np.random.default_rng(V)
    check_sample(rng.standard_normal((3, V)) * np.array([[0.5], [1.0], [4.0]]), rng.random(3), **filters)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("strided", [False, True])
def test_sample_types_strides_and_settings_per_row(dtype, strided):
    rng = np.random.default_rng(8)
    M, V = 33, 3001
    check_sample(rng.standard_normal((M, V)) * 3, rng.random(M), dtype, strided, temperature=rng.choice([0.0, 0.5, 1.0, 2.0], M), top_k=rng.choice([0, -3, 1, 40, V, V + 9], M),
                 top_p=rng.choice([1.0, 0.9, 0.5, 1.5], M), min_p=rng.choice([0.0, 0.05, 0.3], M))


@pytest.mark.parametrize("filters", FILTERS + [dict(top_k=300), dict(top_k=700, top_p=0.8), dict(top_p=0.97, min_p=0.001)])
@pytest.mark.parametrize("spread", [0.6, 3.0])
def test_sample_many_rows(filters, spread):
    """More rows than the GPU takes at a time with a CTA per SM: smaller CTAs that share one."""
    rng = np.random.default_rng(31)
    l = rng.standard_normal((41, 17001)) * spread
    l[3] = np.round(l[3])  # ties
    l[4, 100:] = -np.inf
    l[5] = -np.inf
    check_sample(l, rng.random(41), **filters)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [3, 7, 130, 4097, 50001])
def test_sample_without_filters_types_and_strides(dtype, V):
    rng = np.random.default_rng(V)
    l = rng.standard_normal((9, V)) * 2
    u = rng.random(9)
    t = rng.choice([0.0, 0.3, 1.0, 4.0], 9)
    check_sample(l, u, dtype, True)
    check_sample(l, u, dtype, True, temperature=t)
    check_sample(l, u, dtype, False, temperature=t)
    l[:, : V // 2] -= 200.0  # the parts of most warps weigh nothing
    check_sample(l, u, dtype, True)
    check_sample(l, np.full(9, 1 - 2.0 ** -24), dtype, True)


@pytest.mark.parametrize("filters", FILTERS)
def test_sample_ties(filters):
    # a handful of different logits, so that every threshold falls among equal ones: those with the lowest ids stay
    rng = np.random.default_rng(12)
    check_sample(rng.integers(0, 4, (8, 6000)) * 0.5, rng.random(8), **filters)
    check_sample(np.zeros((4, 4100)), [0.0, 0.3, 0.5, 0.99], **filters)


@pytest.mark.parametrize("filters", FILTERS)
def test_sample_masked_rows(filters):
    rng = np.random.default_rng(13)
    V = 2500
    l = (rng.standard_normal((9, V)) * 2).astype(np.float32)
    l[0, 1:] = -np.inf                      # one token is left
    l[1] = -np.inf                          # none
    l[2, rng.random(V) < 0.9] = -np.inf
    l[3, rng.random(V) < 0.9] = np.finfo(np.float32).min
    l[4, 7] = np.nan
    l[5] = np.nan
    l[6, [5, 2000]] = np.inf
    l[7] = np.finfo(np.float32).min
    l[8, rng.random(V) < 0.5] = -0.0
    with np.errstate(over="ignore"):
        check_sample(l, rng.random(9), **filters)


@pytest.mark.parametrize("filters", [dict(), dict(top_p=0.7), dict(top_k=4), dict(min_p=0.5), dict(temperature=1e35), dict(temperature=1e-12), dict(temperature=1e-12, top_p=0.6),
                                     dict(temperature=1e-40, top_k=3)])
def test_sample_rows_at_the_ends_of_the_type(filters):
    """Rows whose largest logit is the type's lowest (what a mask left of a row) beside -infinity, or the type's largest, or whose parts
    are all masked but one."""
    low, high, V = np.finfo(np.float32).min, np.finfo(np.float32).max, 9000
    rng = np.random.default_rng(21)
    l = np.full((6, V), -np.inf, np.float32)
    l[0, rng.random(V) < 0.3] = low
    l[1, 4444] = low
    l[2] = low
    l[2, 5000:5003] = [1.0, 2.0, 1.5]
    l[3, rng.random(V) < 0.01] = high
    l[4, 7000:] = rng.standard_normal(2000) - 60.0
    l[4, 3] = 0.5
    l[5, ::2] = 0.0
    with np.errstate(over="ignore"):
        check_sample(l, rng.random(6), **filters)
        check_sample(l, np.full(6, 1 - 2.0 ** -24), **filters)


def test_sample_random_numbers_at_their_ends():
    rng = np.random.default_rng(14)
    l = np.tile(rng.standard_normal((1, 700)), (6, 1))
    u = np.array([0.0, 1 - 2.0 ** -24, 1.0, 5.0, -1.0, 2.0 ** -30], np.float32)
    check_sample(l, u)
    check_sample(l, u, top_k=3)
    t = torch.from_numpy(l[:1].astype(np.float32)).to(DEV)
    assert int(bl.bitlinear_sample(t, torch.tensor([float("nan")], device=DEV))[0][0]) == 0  # taken as 0: the first token of any weight


def test_sample_frequencies():
    """20,000 draws of one row: every count within five standard deviations of its expectation."""
    n, V = 20000, 60
    l = np.random.default_rng(15).standard_normal(V).astype(np.float32) * 1.5
    u = (np.arange(n, dtype=np.float64) + np.random.default_rng(16).random(n)) / n  # one in each of n equal parts
    ids, logp = bl.bitlinear_sample(torch.from_numpy(l).to(DEV).expand(n, V).contiguous(), dev(u.astype(np.float32)))
    p = np.exp(l.astype(np.float64) - l.max())
    p /= p.sum()
    counts = np.bincount(host(ids), minlength=V)
    assert np.all(np.abs(counts - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 2)
    assert np.allclose(host(logp), np.log(p)[host(ids)], atol=1e-6)


# ------------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("kind", KINDS)
def test_requests_come_and_go(kind):
    """Steps of a server with four places: prompts, single tokens, requests that finish and others that take their blocks, all
    through the operators, each step checked against the oracle on the same state."""
    n_q, n_kv, D, rows, R, max_blocks, n_blocks, t_cap, t_max, V = 4, 2, 64, 16, 4, 6, 15, 48, 96, 300
    steps = [[20, 0, 5, 0], [1, 30, 1, 0], [1, 1, 1, 3], [1, -1, 1, 1], [-1, 0, 14, 20], [0, 40, 1, 1], [30, 60, -1, 1], [10, 1, 2, 1]]
    rng = np.random.default_rng(17)
    lengths, tables = np.zeros(R, np.int32), np.full((R, max_blocks), -1, np.int32)
    free, n_free = rng.permutation(n_blocks).astype(np.int32), n_blocks
    codes, scales = make_pool(n_blocks, n_kv, rows, D, kind, 18)
    pool = pool_to_dev(codes, scales, kind)
    ld, td, fd, nd = dev(lengths), dev(tables), dev(free), dev(np.array([n_free], np.int32))
    table = bl.bitlinear_rope_table(D, t_max, device=DEV)
    tab = host(table)
    for new in steps:
        want = sv.block_tables(lengths, new, tables, free, n_free, rows, t_cap)
        _, _, served, cu, seq, pos, rl, slots = bl.bitlinear_block_tables(ld, dev(np.array(new, np.int32)), td, fd, nd, rows, t_cap, lengths_out=ld, n_free_out=nd)
        q, k, v = (rng.standard_normal((t_cap, h * D)).astype(np.float32) * rng.uniform(0.5, 3) for h in (n_q, n_kv, n_kv))
        qr = bl.bitlinear_rope_kv8(dev(q), dev(k), dev(v), pos, slots, table, *pool, n_q, n_kv, D)
        out = bl.bitlinear_attention_decode_kv8(qr, *pool, td, rl, n_q, n_kv, D, seq_ids=seq)
        for name, t in zip(("served", "cu_tokens", "seq_ids", "positions", "row_lengths", "slots", "tables", "free_blocks", "lengths"), (served, cu, seq, pos, rl, slots, td, fd, ld)):
            assert np.array_equal(host(t), want[name]), name
        lengths, tables, free, n_free = want["lengths"], want["tables"], want["free_blocks"], want["n_free"]
        at = np.maximum(want["positions"], 0)
        sv.append8(sv.rotate(k.reshape(t_cap, n_kv, D), at, tab), want["slots"], codes[0], scales[0], kind)
        sv.append8(v.reshape(t_cap, n_kv, D).astype(np.float64), want["slots"], codes[1], scales[1], kind)
        for got, w in zip(pool, codes + scales):
            assert np.array_equal(host(got), w)
        check_attention(out, qr.cpu(), codes, scales, tables, want["row_lengths"], n_q, n_kv, D, kind, seq_ids=want["seq_ids"])
        logits = rng.standard_normal((R, V)) * 2
        check_sample(logits, rng.random(R), temperature=0.8, top_k=40, top_p=0.9)
    assert bl.bitlinear_poll_status() == 0


def test_operators_in_a_recorded_graph_and_on_another_stream():
    """A recorded step replays on new contents of its buffers, on a stream that is not the default one, with a workspace full of
    NaN patterns, and gives the bits of the eager calls."""
    kind, n_q, n_kv, D, rows, M = sv.E4M3, 20, 5, 128, 16, 6
    lengths = [40, 1, 333, 16, 1200, 700]
    q, codes, scales, tables = attend_case(kind, n_q, n_kv, D, rows, lengths, 111)
    pool, qd, td, ld = pool_to_dev(codes, scales, kind), q.to(DEV), dev(tables), dev(np.array(lengths, np.int32))
    logits, u = torch.randn(M, 5000, device=DEV) * 2, torch.rand(M, device=DEV)
    p = torch.full((M,), 0.9, device=DEV)
    ws = torch.full((bl.bitlinear_attention_kv8_workspace_bytes(n_q, n_kv, D),), 0xff, dtype=torch.uint8, device=DEV)
    out, ids, logp = torch.empty_like(qd), torch.empty(M, dtype=torch.int32, device=DEV), torch.empty(M, device=DEV)

    def calls():
        bl.bitlinear_attention_decode_kv8(qd, *pool, td, ld, n_q, n_kv, D, out=out, ws=ws)
        bl.bitlinear_sample(logits, u, top_p=p, ids=ids, logprobs=logp)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            calls()
    torch.cuda.synchronize()
    for i in range(3):
        ld.copy_(dev(np.array([max(1, n - 7 * i) for n in lengths], np.int32)))
        logits.normal_()
        out.fill_(7.0), ids.fill_(-3)
        ws.fill_(0xff)
        graph.replay()
        got = out.clone(), ids.clone(), logp.clone()
        out.fill_(7.0), ids.fill_(-3)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            calls()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], ids) and torch.equal(got[2], logp)
    check_attention(out, q, codes, scales, tables, [max(1, n - 14) for n in lengths], n_q, n_kv, D, kind)


def small_layers(n_layers, H, F, kv, seed):
    layers = []
    for li in range(n_layers):
        layer = {}
        for i, (name, n, k) in enumerate((("q", H, H), ("k", kv, H), ("v", kv, H), ("o", H, H), ("gate", F, H), ("up", F, H), ("down", H, F))):
            packed, s_w = bl.bitlinear_pack_weights(wl.latent_weights(n, k, seed + 10 * li + i).to(DEV), wl.WEIGHT_EPS)
            layer[name] = (packed, s_w, wl.gain_random(k, seed + 100 + 10 * li + i).to(DEV))
        layers.append(layer)
    return layers


def paged_step(kv_dtype, rows=6, places=4, n_blocks=14, layers=2):
    from paper_2504_12285_b200 import chain as gpu_chain

    H, F, n_q, n_kv, hd, V = 256, 512, 4, 2, 64, 500
    table = (torch.randn(V, H, generator=torch.Generator().manual_seed(50)) * 0.3).to(torch.bfloat16).to(DEV)
    return gpu_chain.PagedDecodeStep(small_layers(layers, H, F, n_kv * hd, 8700), table, rows, places, n_blocks, 16, 5, H, F, n_q, n_kv, hd, kv_dtype, wl.RMS_EPS,
                                     device=DEV), table


@pytest.mark.parametrize("kind", KINDS)
def test_paged_decode_step_stage_by_stage(kind):
    """Requests of different lengths through PagedDecodeStep; the serving stages of a step against the oracle applied to the
    values the GPU fed into them."""
    st, table = paged_step(DTYPE[kind], layers=1)
    n_q, n_kv, hd = st.dims
    gen = torch.Generator().manual_seed(60)
    st.temperature.copy_(torch.tensor([0.0, 0.7, 1.0, 1.5]))
    st.top_k.copy_(torch.tensor([0, 20, 0, 5], dtype=torch.int32))
    st.top_p.copy_(torch.tensor([1.0, 1.0, 0.8, 0.95]))
    state = [host(t).copy() for t in (st.lengths, st.tables, st.free_blocks)] + [int(st.n_free[0])]
    pool = [host(t).copy() for t in st.cache[0]]
    tab = host(st.rope_table)
    for new in ([5, 1, 0, 0], [1, 1, 4, 0], [1, 1, 1, 1], [-1, 2, 1, 1], [6, 0, 0, 0], [3, 1, 1, 2]):
        st.new_tokens.copy_(torch.tensor(new, dtype=torch.int32))
        ids = torch.randint(0, 500, (6,), generator=gen, dtype=torch.int32)
        u = torch.rand(6, generator=gen)
        got_ids, logp = st.step(ids.to(DEV), u.to(DEV))
        torch.cuda.synchronize()
        assert bl.bitlinear_poll_status() == 0
        want = sv.block_tables(state[0], new, state[1], state[2], state[3], 16, 6)
        state = [want["lengths"], want["tables"], want["free_blocks"], want["n_free"]]
        for name, t in (("lengths", st.lengths), ("tables", st.tables), ("free_blocks", st.free_blocks), ("served", st.served), ("cu_tokens", st.cu_tokens),
                        ("slots", st.slots), ("positions", st.positions)):
            assert np.array_equal(host(t), want[name]), name
        at = np.maximum(want["positions"], 0)
        sv.append8(sv.rotate(host(st.k).reshape(6, n_kv, hd), at, tab), want["slots"], pool[0], pool[2], kind)
        sv.append8(host(st.v).reshape(6, n_kv, hd).astype(np.float64), want["slots"], pool[1], pool[3], kind)
        for got, w in zip(st.cache[0], pool):
            assert np.array_equal(host(got), w)
        check_attention(st.attn, st.q_rot.cpu(), pool[:2], pool[2:], want["tables"], want["row_lengths"], n_q, n_kv, hd, kind, seq_ids=want["seq_ids"])
        logits = host(st.logits)
        for r in range(want["cu_tokens"][-1]):
            p = want["seq_ids"][r]
            token, lp = sv.sample(logits[r], float(u[r]), float(st.temperature[p]), int(st.top_k[p]), float(st.top_p[p]))
            assert int(got_ids[r]) == token and abs(float(logp[r]) - lp) <= 1e-5 + 2.0 ** -23 * abs(lp)


def test_paged_decode_step_recorded():
    """The recorded step replays a changing batch - prompts, single tokens, a finished request whose blocks go to another - with the bits of
    the eager calls."""
    plan = ([5, 1, 0, 0], [1, 1, 4, 0], [1, 1, 1, 1], [-1, 2, 1, 1], [3, 1, 1, 1], [1, 1, 1, 1])

    def run(recorded):
        st, _ = paged_step(torch.int8)
        st.temperature.fill_(0.9), st.top_p.fill_(0.9)
        if recorded:
            st.capture()
        gen, outs = torch.Generator().manual_seed(61), []
        for new in plan:
            st.new_tokens.copy_(torch.tensor(new, dtype=torch.int32))
            ids, u = torch.randint(0, 500, (6,), generator=gen, dtype=torch.int32).to(DEV), torch.rand(6, generator=gen).to(DEV)
            if recorded:
                st.token_buf.copy_(ids), st.u_buf.copy_(u)
                got = st.step_graph()
            else:
                got = st.step(ids, u)
            n = int(st.cu_tokens[-1])
            outs += [got[0][:n].clone(), got[1][:n].clone(), st.logits[:n].clone()]
        torch.cuda.synchronize()
        return outs + [t.clone() for c in st.cache for t in (c[0].view(torch.uint8), c[1].view(torch.uint8), c[2], c[3])]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)
    assert bl.bitlinear_poll_status() == 0


def test_calls_on_two_streams_at_once():
    """Independent calls, each with a workspace of its own, in flight together: the bits of the calls alone."""
    kind, n_q, n_kv, D = sv.INT8, 20, 5, 128
    sets = []
    for i in range(2):
        lengths = [900 + 50 * i, 17, 2000, 5]
        q, codes, scales, tables = attend_case(kind, n_q, n_kv, D, 64, lengths, 120 + i)
        g = torch.Generator(DEV).manual_seed(i)
        sets.append((q.to(DEV), pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(lengths, np.int32)),
                     torch.randn(5, 30000, generator=g, device=DEV) * 2, torch.rand(5, generator=g, device=DEV), torch.full((5,), 0.9, device=DEV)))
    for s in sets:
        torch.cuda.synchronize()

    def calls(s):
        return (bl.bitlinear_attention_decode_kv8(s[0], *s[1], s[2], s[3], n_q, n_kv, D), *bl.bitlinear_sample(s[4], s[5], top_p=s[6]), *bl.bitlinear_sample(s[4], s[5]))

    alone = [calls(s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                outs.append(calls(s))
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        for a, b in zip(out, alone[i % 2]):
            assert torch.equal(a, b)


def test_binding_checks_shapes_types_and_devices():
    pool = pool_to_dev(*make_pool(4, 2, 16, 64, sv.INT8, 1), sv.INT8)
    q, t, n = torch.zeros(2, 256, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 4, dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    good = [q, *pool, t, n, 4, 2, 64]
    bl.bitlinear_attention_decode_kv8(*good)
    for i, bad in ((0, q.float()), (0, q[:, :128]), (1, pool[0].float()), (2, pool[1].view(torch.float8_e4m3fn)), (2, pool[1][:3]), (3, pool[2][:, :1]), (5, t.long()), (5, t[0]),
                   (6, n[:1]), (6, n.cpu()), (8, 1), (9, 128)):
        with pytest.raises((TypeError, ValueError)):
            bl.bitlinear_attention_decode_kv8(*good[:i], bad, *good[i + 1:])
    with pytest.raises(bl.BitLinearError):
        bl.bitlinear_attention_decode_kv8(*good, ws=torch.empty(64, dtype=torch.uint8, device=DEV))
    with pytest.raises(bl.BitLinearError):  # three rows, two sequences, no ids
        bl.bitlinear_attention_decode_kv8(torch.zeros(3, 256, dtype=torch.bfloat16, device=DEV), *pool, t, torch.ones(3, dtype=torch.int32, device=DEV), 4, 2, 64)
    logits, u = torch.zeros(3, 50, device=DEV), torch.zeros(3, device=DEV)
    for kw in (dict(u=u[:2]), dict(u=u.double()), dict(u=u, top_k=u), dict(u=u, temperature=u[:1]), dict(logits=logits.half()), dict(logits=logits.t()), dict(logits=logits[:, ::2]),
               dict(logits=logits[:1].expand(3, 50)), dict(ids=torch.zeros(3, device=DEV))):
        with pytest.raises((TypeError, ValueError)):
            bl.bitlinear_sample(**{"logits": logits, "u": u, **kw})
    f = torch.zeros(2, 256, device=DEV)
    kv = torch.zeros(2, 128, device=DEV)
    table = bl.bitlinear_rope_table(64, 32, device=DEV)
    good = [f, kv, kv, n, n, table, *pool, 4, 2, 64]
    bl.bitlinear_rope_kv8(*good)
    for i, bad in ((0, kv), (1, f), (2, kv.double()), (3, n.long()), (4, n[:1]), (5, table[:, :16]), (6, pool[0][:, :, :, :32]), (8, pool[2].half())):
        with pytest.raises((TypeError, ValueError)):
            bl.bitlinear_rope_kv8(*good[:i], bad, *good[i + 1:])
