"""Attention of groups of rows over cache rows that they share, against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = [sv.INT8, sv.E4M3]
DTYPE = {sv.INT8: torch.int8, sv.E4M3: torch.float8_e4m3fn}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Case:
    """groups: [(lengths of the rows, rows shared)] of answers with tables of their own whose first blocks are the same, or, with chunk, of rows of one
    sequence; lone: lengths of rows behind the last group."""

    def __init__(self, kind, n_q, n_kv, D, rows, groups, lone=(), chunk=False, seed=0, size=2.5):
        rng = np.random.default_rng(seed)
        self.kind, self.dims, self.rows = kind, (n_q, n_kv, D), rows
        lengths, seq, starts, self.tables_of, n_blocks = [], [], [0], [], 0
        for lens, shared in groups:
            first = None
            for n in lens:
                if chunk and first is not None:
                    seq.append(first)
                else:
                    own = -(-max(n, shared if chunk else n, max(lens) if chunk else 0) // rows) + 1
                    common = 0 if first is None else min(-(-shared // rows), own)
                    table = list(range(n_blocks, n_blocks + own))
                    n_blocks += own
                    if first is not None:
                        table[:common] = self.tables_of[first][:common]
                        table += [self.tables_of[first][i] for i in range(len(table), common)]
                    seq.append(len(self.tables_of))
                    if first is None:
                        first = len(self.tables_of)
                        table += list(range(n_blocks, n_blocks + max(0, -(-shared // rows) - own)))  # the leader's table names all shared blocks
                        n_blocks += max(0, -(-shared // rows) - own)
                    self.tables_of.append(table)
                lengths.append(n)
            starts.append(len(lengths))
        for n in lone:
            own = -(-max(n, 0) // rows) + 1
            seq.append(len(self.tables_of))
            self.tables_of.append(list(range(n_blocks, n_blocks + own)))
            n_blocks += own
            lengths.append(n)
        n_blocks += 1
        ids = rng.permutation(n_blocks)
        self.tables = np.full((len(self.tables_of), max(map(len, self.tables_of))), -1, np.int32)
        for s, t in enumerate(self.tables_of):
            self.tables[s, :len(t)] = ids[t]
        self.lengths, self.seq = np.array(lengths, np.int32), np.array(seq, np.int32)
        self.starts, self.shared = np.array(starts, np.int32), np.array([s for _, s in groups], np.int32)
        shape = (n_blocks, n_kv, rows, D)
        self.codes = [sv.encode(rng.standard_normal(shape) * (40.0 if kind == sv.INT8 else 100.0), kind) for _ in range(2)]
        self.scales = [np.array([[sv.scale_for(a, kind) for a in row] for row in rng.uniform(0.3, 1.2, shape[:2]) * size], np.float32) for _ in range(2)]
        # rows that no length covers hold the worst bits there are
        live = np.zeros((n_blocks, rows), bool)
        for s, n in zip(self.seq, self.lengths):
            t = np.arange(max(n, 0))
            live[self.tables[s][t // rows], t % rows] = True
        for c in self.codes:
            c[np.broadcast_to(~live[:, None, :, None], shape)] = 0x7F if kind == sv.E4M3 else 0x80
        for x in self.scales:
            x[~live.any(1)] = np.nan
        self.q = (torch.randn(len(lengths), n_q * D, generator=torch.Generator().manual_seed(seed)) * 2.0).to(torch.bfloat16)

    def call(self, **kw):
        pool = [dev(c).view(DTYPE[self.kind]) for c in self.codes] + [dev(s) for s in self.scales]
        return bl.bitlinear_attention_shared_kv8(self.q.to(DEV), *pool, dev(self.tables), dev(self.lengths), dev(self.starts), dev(self.shared), *self.dims, seq_ids=dev(self.seq), **kw)

    def check(self, got, rows=None):
        n_q, n_kv, D = self.dims
        got = got.double().cpu().numpy().reshape(-1, n_q, D)
        assert np.isfinite(got).all()
        qn = self.q.double().numpy().reshape(-1, n_q, D)
        cache = {}
        for m in range(len(self.lengths)) if rows is None else rows:
            s, n = int(self.seq[m]), int(self.lengths[m])
            if n <= 0:
                assert not got[m].any()
                continue
            if s not in cache:
                most = int(self.lengths[self.seq == s].max())
                t = np.arange(most)
                b, r = self.tables[s][t // self.rows], t % self.rows
                ok = (b >= 0) & (b < len(self.codes[0]))
                b = np.where(ok, b, 0)
                k, v = (sv.decode(c[b, :, r], self.kind) * x[b].astype(np.float64)[..., None] for c, x in zip(self.codes, self.scales))
                cache = {s: (k, v, ok)}
            k, v, ok = (x[:n] for x in cache[s])
            k, v = k[ok], v[ok]
            for h in range(n_q):
                g = h // (n_q // n_kv)
                if not ok.any():
                    assert not got[m, h].any()
                    continue
                score = k[:, g] @ qn[m, h] / math.sqrt(D)
                p = np.exp(score - score.max())
                want = (p / p.sum()) @ v[:, g]
                # D products in fp32, each addition off by 2^-23 at most (the tensor cores may cut instead of round), three roundings of the scaled score, and
                # queries that lose what is below 2^-23 of their head's largest
                err = ((D + 4) * 2.0 ** -23 * float((np.abs(k[:, g]) @ np.abs(qn[m, h])).max()) + 2.0 ** -23 * np.abs(qn[m, h]).max() * float(np.abs(k[:, g]).sum(-1).max())) / math.sqrt(D)
                # the weights' rounding to f16 (half a step 2^-12, an eps of 2^-11 with what their scale rounds), both errors of a weight (it stands above and below the
                # line: twice the scores' error), sums in fp32; then half a step of bf16
                tol = (2.0 ** -11 + 2 * err + 1e-6) * np.abs(v[:, g]).max()
                assert (np.abs(got[m, h] - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol)).all(), (m, h, np.abs(got[m, h] - want).max(), tol)


SMALL = [
    ([([1, 1], 1)], []),
    ([([20, 40, 33], 16)], [5, 0, 1]),
    ([([130, 129, 128, 127], 128)], []),
    ([([300] * 5, 300)], [64]),
    ([([256, 300, 511, 513, 700], 256), ([1, 2, 3], 1), ([40], 30)], [200]),
    ([([600, 20, 0, 599, 601], 590)], []),                # rows shorter than what the group shares
    ([([90, 80], 0), ([50, 60], 5000), ([], 64)], [7]),    # nothing shared, more shared than there is, no rows
]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_kv,D,rows", [(20, 5, 128, 64), (8, 8, 64, 16), (7, 1, 128, 16), (16, 2, 64, 128), (5, 1, 64, 32), (6, 2, 128, 128)])
@pytest.mark.parametrize("groups,lone", SMALL)
def test_answers_that_share_a_prompt(kind, n_q, n_kv, D, rows, groups, lone):
    # blocks are shared whole, so what lies between two answers' own rows and the shared ones belongs to each
    groups = [(lens, shared if max(lens, default=0) <= shared or shared == 0 else shared // rows * rows) for lens, shared in groups]
    case = Case(kind, n_q, n_kv, D, rows, groups, lone, seed=len(lone) + D)
    case.check(case.call())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_kv,D,rows", [(20, 5, 128, 64), (8, 2, 64, 16), (3, 1, 128, 32)])
@pytest.mark.parametrize("start,n", [(0, 1), (0, 2), (0, 129), (5, 70), (127, 130), (300, 33)])
def test_tokens_of_a_chunk(kind, n_q, n_kv, D, rows, start, n):
    lens = list(range(start + 1, start + n + 1))
    for shared in sorted({start, start + n, max(1, start - 3), 10 ** 6}):  # all of it, what lies in front of the chunk, a number that fits no block
        case = Case(kind, n_q, n_kv, D, rows, [(lens, start + n)], chunk=True, seed=n)
        case.shared[:] = shared
        case.check(case.call())


@pytest.mark.parametrize("kind", KINDS)
def test_many_query_rows(kind):
    """More than one pair of query tiles, borders inside a token's heads, two chunks at once."""
    case = Case(kind, 15, 3, 64, 32, [(list(range(101, 101 + 217)), 317), (list(range(1, 60)), 59)], lone=[33, 500], chunk=True, seed=4)
    case.check(case.call())
    case = Case(kind, 8, 1, 128, 64, [([700 + 3 * i for i in range(70)], 640)], seed=5)
    case.check(case.call())


@pytest.mark.parametrize("kind,D", [(sv.INT8, 128), (sv.E4M3, 64)])
def test_long_shared_rows(kind, D):
    case = Case(kind, 8, 2, D, 128, [([20000 + 40 * i for i in range(9)], 19968)], lone=[9000], seed=6)
    case.check(case.call(), rows=[0, 4, 8, 9])


@pytest.mark.parametrize("kind", KINDS)
def test_values_and_scales_of_very_different_sizes(kind):
    case = Case(kind, 4, 1, 64, 16, [([200, 180, 90], 64)], seed=7)
    rng = np.random.default_rng(1)
    live = ~np.isnan(case.scales[1])
    case.scales[1] = np.where(live, case.scales[1] * 2.0 ** rng.integers(-40, 3, live.shape), np.nan).astype(np.float32)
    case.check(case.call())
    case.scales[1][live] = 0.0
    assert not case.call().any()
    # keys so large that one row takes all the weight, and scales of zero
    case = Case(kind, 4, 1, 64, 16, [([200, 180, 90], 64)], seed=8, size=400.0)
    case.check(case.call())
    case.scales[0][live] = 0.0
    case.check(case.call())


@pytest.mark.parametrize("kind", KINDS)
def test_queries_of_very_different_sizes(kind):
    case = Case(kind, 8, 2, 128, 64, [([200, 300, 270], 192)], seed=9)
    case.q[0] *= 1e-30
    case.q[1, :128] = 0
    case.q[1, 200] = 300.0
    case.check(case.call())


def test_what_is_not_finite_stays_in_its_row_and_head():
    case = Case(sv.INT8, 8, 2, 64, 32, [([300, 290, 280, 100], 256)], lone=[64], seed=10)
    case.q[1, 64 * 5 + 3] = math.nan
    case.q[3, 0] = math.inf
    got = case.call().float().cpu().reshape(5, 8, 64)
    bad = torch.isnan(got).all(-1)
    want = torch.zeros(5, 8, dtype=torch.bool)
    want[1, 5] = want[3, 0] = True
    assert torch.equal(bad, want) and torch.equal(torch.isnan(got).any(-1), want)
    # a scale that is NaN: the rows that use its block, of that KV head
    case = Case(sv.INT8, 8, 2, 64, 32, [([300, 290, 280, 100], 256)], lone=[64], seed=10)
    for pool in (0, 1):
        for at, rows in ((2, [0, 1, 2, 3]), (5, [0, 1, 2])):  # cache rows 64 .. 95, 160 .. 191
            scales = [s.copy() for s in case.scales]
            block = case.tables[0][at]
            case.scales[pool][block, 1] = math.nan
            got = torch.isnan(case.call().float().cpu().reshape(5, 8, 64))
            want = torch.zeros(5, 8, dtype=torch.bool)
            want[rows, 4:] = True
            assert torch.equal(got.any(-1), want) and torch.equal(got.all(-1), want), (pool, at)
            case.scales = scales


@pytest.mark.parametrize("kind", KINDS)
def test_bad_tables_lengths_and_groups(kind):
    case = Case(kind, 4, 2, 64, 16, [([300, 290, 310], 256)], lone=[100], seed=11)
    # blocks that are none: their rows are left out, of the shared ones for all rows
    for at, bad in ((1, -1), (7, 10 ** 6)):
        for s in range(3):
            case.tables[s, at] = bad
    case.tables[1, 17] = -5
    case.tables[3, 2] = 2 ** 31 - 1
    case.check(case.call())
    # sequences and lengths out of range, the group's first row among them
    case.seq[0], case.lengths[1] = -3, -10
    want = case.call().float().cpu()
    assert not want[:2].any()
    case.lengths[0] = 0
    case.check(case.call(), rows=[1, 2, 3])
    # lengths past the table count as its end; borders of groups outside the rows, decreasing ones: nothing is read or written out of place
    case.lengths[2] = 2 ** 31 - 1
    case.call()
    for starts in ([-7, 99], [3, 1], [2 ** 31 - 1, -2 ** 31], [1, 3]):
        case.starts[:] = starts
        case.call()
    torch.cuda.synchronize()
    assert bl.bitlinear_poll_status() == 0


def test_no_rows_no_groups_and_agreement_with_the_other_attention():
    case = Case(sv.INT8, 20, 5, 128, 64, [([700, 710, 500, 64], 448)], lone=[1, 0, 333], seed=12)
    pool = [dev(c).view(torch.int8) for c in case.codes] + [dev(s) for s in case.scales]
    none = dict(group_starts=torch.zeros(1, dtype=torch.int32, device=DEV), shared_rows=torch.zeros(0, dtype=torch.int32, device=DEV))
    q, tables, lengths, seq = case.q.to(DEV), dev(case.tables), dev(case.lengths), dev(case.seq)
    alone = bl.bitlinear_attention_shared_kv8(q, *pool, tables, lengths, none["group_starts"], none["shared_rows"], *case.dims, seq_ids=seq)
    case.check(alone)
    case.check(bl.bitlinear_attention_decode_kv8(q, *pool, tables, lengths, *case.dims, seq_ids=seq))
    empty = bl.bitlinear_attention_shared_kv8(q[:0], *pool, tables, lengths[:0], none["group_starts"], none["shared_rows"], *case.dims, seq_ids=seq[:0])
    assert empty.shape == (0, 2560)


def test_recorded_repeated_and_on_two_streams():
    cases = [Case(sv.INT8, 20, 5, 128, 64, [([1200 + i for i in range(16)], 1024)], lone=[70], seed=13), Case(sv.E4M3, 20, 5, 128, 64, [(list(range(200, 300)), 300)], chunk=True, seed=14)]
    args = []
    for c in cases:
        pool = [dev(x).view(DTYPE[c.kind]) for x in c.codes] + [dev(s) for s in c.scales]
        args.append((c.q.to(DEV), *pool, dev(c.tables), dev(c.lengths), dev(c.starts), dev(c.shared), *c.dims, dev(c.seq)))
    want = [bl.bitlinear_attention_shared_kv8(*x) for x in args]
    for c, w in zip(cases, want):
        c.check(w)
    for _ in range(20):
        assert all(torch.equal(bl.bitlinear_attention_shared_kv8(*x), w) for x, w in zip(args, want))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = [bl.bitlinear_attention_shared_kv8(*x) for x in args]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    args[0][6].sub_(150)  # the recording reads the lengths that are there when it is replayed
    graph.replay()
    torch.cuda.synchronize()
    cases[0].lengths -= 150
    cases[0].check(got[0])
    args[0][6].add_(150)
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(8):
        streams[i % 2].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(streams[i % 2]):
            outs.append(bl.bitlinear_attention_shared_kv8(*args[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i % 2]) for i, o in enumerate(outs))
    assert bl.bitlinear_poll_status() == 0
