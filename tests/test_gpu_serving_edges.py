"""The serving operators at their edges: settings that are no number, values that are not finite, queries with one large channel, prompts that fill
the append's tiles, recorded and eager steps in turn, calls that are refused before anything is written."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from test_gpu_serving import (DEV, DTYPE, KINDS, attend_case, check_append, check_attention, check_sample, check_tables, dev, host, make_pool, paged_step,
                              pool_to_dev)
from test_serving_edges import outlier_case

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------- sampling

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,V", [(4, 3000), (41, 17001)])
@pytest.mark.parametrize("filters", [dict(), dict(top_k=40, top_p=0.9, min_p=0.01), dict(top_p=0.95)])
def test_sample_takes_the_largest_where_the_temperature_is_no_number(dtype, M, V, filters):
    rng = np.random.default_rng(M)
    t = rng.uniform(0.5, 2.0, M)
    t[::2] = np.nan
    t[1] = -np.inf
    t[3] = np.inf
    check_sample(rng.standard_normal((M, V)) * 2, rng.random(M), dtype, temperature=t, **filters)


# ------------------------------------------------------------------------------------------------- attention

LENGTHS = [1, 40, 20000, 7, 300, 0]  # one CTA's own, several warps', and one that many CTAs share


def check_attention_but_nan(out, bad, q, codes, scales, tables, lengths, n_q, n_kv, D, kind):
    """Rows and heads marked in bad [M, n_q] are NaN in every dim, the others as check_attention wants them."""
    got = out.float().cpu().numpy().reshape(len(lengths), n_q, D)
    assert np.isnan(got[bad]).all()
    ref = out.clone().view(len(lengths), n_q, D)
    for m, n in enumerate(lengths):
        for h in np.nonzero(bad[m])[0]:
            want = sv.attention8(np.nan_to_num(q[m].double().numpy().reshape(n_q, D), nan=0.0, posinf=0.0, neginf=0.0), *codes, *scales, tables[m], n, n_q, n_kv, D, kind)[0][h]
            ref[m, int(h)] = torch.from_numpy(want).to(ref)
    clean = torch.where(torch.isfinite(q.float()), q.float(), 0.0).to(torch.bfloat16)
    check_attention(ref.view(len(lengths), -1), clean, codes, scales, tables, lengths, n_q, n_kv, D, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("n_q,n_kv,D", [(4, 1, 128), (8, 1, 64), (4, 2, 64)])
def test_attention_of_a_query_that_is_not_finite_is_nan(kind, value, n_q, n_kv, D):
    q, codes, scales, tables = attend_case(kind, n_q, n_kv, D, 64, LENGTHS, 131)
    bad = np.zeros((len(LENGTHS), n_q), bool)
    for m in range(len(LENGTHS)):
        h = (m + 1) % n_q
        q[m, h * D + 5] = value
        bad[m, h] = LENGTHS[m] > 0  # a row without a length gives zeros whatever its query
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, kind), dev(tables), dev(np.array(LENGTHS, np.int32)), n_q, n_kv, D)
    assert not out[-1].any()
    check_attention_but_nan(out, bad, q, codes, scales, tables, LENGTHS, n_q, n_kv, D, kind)
    assert bl.bitlinear_poll_status() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("pool", ["keys", "values"])
@pytest.mark.parametrize("at", [0, 100, 312])  # the first block, one in the middle, the last of 20,000 rows
def test_attention_over_a_block_whose_scale_is_no_number_is_nan(kind, pool, at):
    n_q, n_kv, D = 4, 2, 64
    q, codes, scales, tables = attend_case(kind, n_q, n_kv, D, 64, LENGTHS, 132)
    broken = [s.copy() for s in scales]
    broken[0 if pool == "keys" else 1][tables[2, at], 1] = np.nan
    bad = np.zeros((len(LENGTHS), n_q), bool)
    bad[2, 2:] = True
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, broken, kind), dev(tables), dev(np.array(LENGTHS, np.int32)), n_q, n_kv, D)
    check_attention_but_nan(out, bad, q, codes, scales, tables, LENGTHS, n_q, n_kv, D, kind)


@pytest.mark.parametrize("size", [4000.0, 200.0])
@pytest.mark.parametrize("n_q,n_kv,D", [(4, 2, 64), (20, 5, 128), (8, 1, 128), (7, 1, 64)])
def test_attention_of_queries_with_one_large_channel(size, n_q, n_kv, D):
    lengths = [300, 40, 17, 5000, 1]
    q, codes, scales, tables = outlier_case(n_q, n_kv, D, 16, lengths, 8, size)
    out = bl.bitlinear_attention_decode_kv8(q.to(DEV), *pool_to_dev(codes, scales, sv.INT8), dev(tables), dev(np.array(lengths, np.int32)), n_q, n_kv, D)
    check_attention(out, q, codes, scales, tables, lengths, n_q, n_kv, D, sv.INT8)


# ------------------------------------------------------------------------------------------------- append

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_append_of_values_that_are_not_finite(kind, D, value):
    """The scale of the block and head that gets one is NaN until the block's first row is written again; nothing else is touched."""
    n_kv, rows, T = 2, 16, 40
    rng = np.random.default_rng(6)
    k, v = ((rng.standard_normal((T, n_kv * D)) * 2).astype(np.float32) for _ in range(2))
    slots = np.arange(5, 5 + T, dtype=np.int32)
    k[13, 3] = value      # block 1, head 0
    v[30, D + 9] = value  # block 2, head 1
    codes, scales = make_pool(5, n_kv, rows, D, kind, 7)
    scales[1][0, 0] = np.nan  # block 0 goes on behind rows whose scale is no number
    pool = pool_to_dev(codes, scales, kind)
    table = bl.bitlinear_rope_table(D, 64, device=DEV)
    tab = host(table)

    def append(k, v, slots):
        T = len(slots)
        pos = slots.astype(np.int32)
        bl.bitlinear_rope_kv8(torch.zeros(T, 4 * D, device=DEV), dev(k), dev(v), dev(pos), dev(slots), table, *pool, 4, n_kv, D)
        with np.errstate(invalid="ignore"):
            sv.append8(sv.rotate(k.reshape(T, n_kv, D), pos, tab), slots, codes[0], scales[0], kind)
            sv.append8(v.reshape(T, n_kv, D).astype(np.float64), slots, codes[1], scales[1], kind)
        for got, want in zip(pool[2:], scales):
            assert np.array_equal(host(got), want, equal_nan=True)
        for got, want, s in zip(pool[:2], codes, scales):
            fine = ~np.isnan(s)
            assert np.array_equal(host(got)[fine], want[fine])
            assert np.array_equal(host(got)[~fine], want[~fine])

    append(k, v, slots)
    nan = [np.argwhere(np.isnan(s)).tolist() for s in scales]
    assert nan == [[[1, 0]], [[0, 0], [2, 1]]]
    append(np.ones((1, n_kv * D), np.float32), np.ones((1, n_kv * D), np.float32), np.array([45], np.int32))  # block 2 again: still no number
    assert np.isnan(host(pool[3])[2, 1])
    append(np.ones((3, n_kv * D), np.float32), np.ones((3, n_kv * D), np.float32), np.array([0, 16, 32], np.int32))
    assert not np.isnan(host(pool[2])).any() and not np.isnan(host(pool[3])).any()


def runs_in_blocks(runs, rows, rng):
    """Slots and positions of runs (first row, number of rows) of sequences over shuffled blocks, and the number of blocks."""
    used = [-(-(s + n) // rows) for s, n in runs]
    ids = rng.permutation(sum(used) + 2)
    slots, pos, b = [], [], 0
    for (s, n), u in zip(runs, used):
        p = np.arange(s, s + n)
        slots += list(ids[b + p // rows] * rows + p % rows)
        pos += list(p)
        b += u
    return np.array(slots, np.int64), np.array(pos, np.int64), sum(used) + 2


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,rows,shape", [(64, 16, "short"), (128, 16, "short"), (64, 128, "long"), (128, 32, "long"), (128, 64, "mixed"), (64, 32, "mixed")])
def test_append_of_prompts(kind, D, rows, shape):
    """More tokens than a CTA each would take (T * 2 * n_kv > 64 SMs' worth) and than one pass of the queries' CTAs: tiles with
    several runs, runs that cross tiles, a last tile in part, tokens without a place inside a tile."""
    rng = np.random.default_rng([D, rows])
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n_kv = 2
    least = max(16 * sms, 64 * sms // (2 * n_kv)) + 100
    runs = []
    while sum(n for _, n in runs) <= least:
        runs.append((int(rng.integers(0, 2 * rows)), int({"short": rng.integers(1, 6), "long": rng.integers(200, 700), "mixed": rng.choice([1, 2, 3, 17, 90])}[shape])))
    slots, pos, n_blocks = runs_in_blocks(runs, rows, rng)
    T = len(slots)
    if T % 16 == 0:
        slots, pos, T = slots[:-1], pos[:-1], T - 1
    assert T > 16 * sms and T * 2 * n_kv > 64 * sms and T % 16
    # a run's last tokens have no place: padding, a slot past the pool, a position past the table
    ends = np.cumsum([n for _, n in runs])[:-1] - 1
    for i, e in enumerate(ends[3::7]):
        slots[e] = (-1, n_blocks * rows + 5, slots[e])[i % 3]
        pos[e] = (-1, pos[e], 5000)[i % 3]
    check_append(kind, 4, n_kv, D, rows, slots, pos, 23, n_blocks=n_blocks, t_max=1024)


# ------------------------------------------------------------------------------------------------- block tables

def test_block_tables_of_blocks_as_long_as_the_type():
    """One block of 2^31 - 1 rows: lengths and blocks are counted without passing 32 bits."""
    rows = 2 ** 31 - 1
    for lengths, new in (([5, 0], [3, 0]), ([0, 7], [2, -1]), ([0, 0], [4, 9])):
        tables = np.full((2, 1), -1, np.int32)
        used = [i for i, n in enumerate(lengths) if n > 0]
        for i in used:
            tables[i] = 0
        check_tables(np.array(lengths, np.int32), np.array(new, np.int32), tables, np.zeros(1, np.int32), 0 if used else 1, rows, 20)


# ------------------------------------------------------------------------------------------------- the paged step

def test_paged_decode_step_eager_and_recorded_in_turn():
    """What the step says of its rows belongs to the step that ran last, recorded or not."""
    st, _ = paged_step(torch.int8)
    st.temperature.fill_(0.9)
    st.capture()
    state = [host(t).copy() for t in (st.lengths, st.tables, st.free_blocks)] + [int(st.n_free[0])]
    gen = torch.Generator().manual_seed(62)
    for i, new in enumerate(([5, 1, 0, 0], [1, 1, 4, 0], [1, 0, 1, 1], [-1, 2, 1, 1], [6, 0, 0, 0], [3, 1, 1, 2], [1, 1, 1, 1])):
        st.new_tokens.copy_(torch.tensor(new, dtype=torch.int32))
        ids, u = torch.randint(0, 500, (6,), generator=gen, dtype=torch.int32).to(DEV), torch.rand(6, generator=gen).to(DEV)
        if i in (0, 2, 3, 5):
            st.step(ids, u)
        else:
            st.token_buf.copy_(ids), st.u_buf.copy_(u)
            st.step_graph()
        want = sv.block_tables(state[0], new, state[1], state[2], state[3], 16, 6)
        state = [want["lengths"], want["tables"], want["free_blocks"], want["n_free"]]
        for name in ("lengths", "served", "cu_tokens", "seq_ids", "positions", "row_lengths", "slots"):
            assert np.array_equal(host(getattr(st, name)), want[name]), (i, name)
    assert bl.bitlinear_poll_status() == 0


def state_of(st):
    return [t.clone() for t in (st.lengths, st.tables, st.free_blocks, st.n_free)] + [x.view(torch.uint8).clone() for c in st.cache for x in c]


def test_paged_decode_step_refuses_before_it_changes_anything():
    st, _ = paged_step(torch.int8)
    ids, u = torch.zeros(6, dtype=torch.int32, device=DEV), torch.rand(6, device=DEV)
    st.new_tokens.copy_(torch.tensor([3, 1, 1, 0], dtype=torch.int32))
    before = state_of(st)
    wide = torch.zeros(20, dtype=torch.int32, device=DEV)
    for bad in ((wide, u), (ids[:4], u), (ids.long(), u), (ids.cpu(), u), (ids, u[:4]), (ids, u.double()), (ids, torch.rand(12, device=DEV)[::2])):
        with pytest.raises((TypeError, ValueError)):
            st.step(*bad)
    for name, bad in (("temperature", torch.ones(3, device=DEV)), ("top_k", torch.zeros(4, device=DEV)), ("top_p", torch.ones(4).double().to(DEV)), ("min_p", torch.zeros(4))):
        good = getattr(st, name)
        setattr(st, name, bad)
        with pytest.raises((TypeError, ValueError)):
            st.step(ids, u)
        setattr(st, name, good)
    for a, b in zip(before, state_of(st)):
        assert torch.equal(a, b)
    st.step(ids, u)
    assert st.lengths.tolist() == [3, 1, 1, 0]


def test_paged_decode_step_is_not_built_where_a_call_would_refuse():
    from paper_2504_12285_b200 import chain as gpu_chain
    from paper_2504_12285_b200 import workloads as wl
    from test_gpu_serving import small_layers

    H, F, n_q, n_kv, hd = 256, 512, 4, 2, 64
    layers, table = small_layers(1, H, F, n_kv * hd, 8700), torch.zeros(500, H, dtype=torch.bfloat16, device=DEV)

    def build(block_rows=16, n_q=n_q, kv_dtype=torch.int8, table=table):
        return gpu_chain.PagedDecodeStep(layers, table, 6, 4, 14, block_rows, 5, H, F, n_q, n_kv, hd, kv_dtype, wl.RMS_EPS, device=DEV)

    for bad in (dict(block_rows=48), dict(n_q=2), dict(kv_dtype=torch.float8_e5m2), dict(table=torch.zeros(bl.SAMPLE_MAX_VOCAB + 1, H, dtype=torch.bfloat16, device=DEV))):
        with pytest.raises((TypeError, ValueError, bl.BitLinearError)):
            build(**bad)
    assert int(build().n_free[0]) == 14


def test_decode_step_refuses_other_numbers_of_tokens():
    from paper_2504_12285_b200 import chain as gpu_chain
    from paper_2504_12285_b200 import workloads as wl
    from test_gpu_serving import small_layers

    table = torch.zeros(500, 256, dtype=torch.bfloat16, device=DEV)
    st = gpu_chain.DecodeStep(small_layers(1, 256, 512, 128, 8700), table, 2, 64, 256, 512, 4, 2, 64, wl.RMS_EPS, device=DEV)
    for n in (1, 3):
        with pytest.raises(ValueError):
            st.step(torch.zeros(n, dtype=torch.int32, device=DEV))
    assert st.step(torch.zeros(2, dtype=torch.int32, device=DEV)).shape == (2, 500)


@pytest.mark.parametrize("recorded", [False, True])
def test_paged_decode_step_keeps_tokens_with_their_places(recorded):
    """A place that outgrows its table is left out and does not hold up the others: the places behind it still get their own tokens, those that
    lie beyond the step's rows none."""
    def run(new, tokens):
        st, _ = paged_step(torch.int8)
        if recorded:
            st.capture()
        # place 1 has 79 of the 80 rows that its table can name, the others start
        st.tables[1] = torch.arange(9, 14, dtype=torch.int32, device=DEV)
        st.lengths[1] = 79
        st.n_free.fill_(9)
        outs = []
        for n, t in zip(new, tokens):
            st.new_tokens.copy_(torch.tensor(n, dtype=torch.int32))
            ids, u = torch.tensor((t + [0] * 6)[:6], dtype=torch.int32, device=DEV), torch.full((6,), 0.4, device=DEV)
            if recorded:
                st.token_buf.copy_(ids), st.u_buf.copy_(u)
                got = st.step_graph()
            else:
                got = st.step(ids, u)
            n = int(st.cu_tokens[-1])
            outs += [got[0][:n].clone(), got[1][:n].clone(), st.logits[:n].clone(), st.served.clone(), st.lengths.clone()]
        return outs

    got = run(([1, 3, 1, 1], [1, 2 ** 31 - 1, 1, 0], [0, 2, 2, 2], [1, 1, 1, 1]), ([11, 21, 22, 23, 31, 41], [12, 24, 25, 26, 27, 28], [29, 29, 32, 33, 42, 43], [13, 20, 34, 44]))
    want = run(([1, 0, 1, 1], [1, 0, 0, 0], [0, 0, 2, 2], [1, 1, 1, 1]), ([11, 31, 41], [12], [32, 33, 42, 43], [13, 20, 34, 44]))
    served = ([1, 0, 1, 1], [1, 0, 0, 1], [1, 0, 1, 1], [1, 1, 1, 1])
    for i, s in enumerate(served):
        assert got[5 * i + 3].tolist() == s
    for i, (a, b) in enumerate(zip(got, want)):
        if i % 5 != 3:
            assert torch.equal(a, b), i
