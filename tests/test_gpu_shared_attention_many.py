"""Attention over shared cache rows where a call has hundreds to thousands of rows or groups: the plan takes several rows a thread and keeps its borders outside
shared memory, and a row's parts are joined for all query heads of a KV head together."""
import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from test_gpu_shared_attention import Case

pytestmark = pytest.mark.gpu


def some(case, n, more=()):
    return sorted(set(np.random.default_rng(0).integers(0, len(case.lengths), n).tolist()) | {0, len(case.lengths) - 1} | set(more))


@pytest.mark.parametrize("kind,n_q,n_kv,D", [(sv.INT8, 35, 5, 128), (sv.E4M3, 40, 8, 64), (sv.INT8, 24, 3, 64)])
def test_chunks_answers_and_lone_rows_together(kind, n_q, n_kv, D):
    # 148 SMs times 128 heads and more; groups of heads that cross the borders of tiles and pairs; rows with a shared part, an own part, both and neither
    chunk = list(range(131, 131 + 420))
    answers = [330 + 17 * i % 190 for i in range(90)]
    answers[5] = answers[88] = 0
    case = Case(kind, n_q, n_kv, D, 32, [(answers, 320), ([40, 90], 0), ([64] * 37, 64)], lone=[7 * i % 300 for i in range(700)], seed=2)
    assert len(case.lengths) * n_q >= 128 * 148
    case.check(case.call(), rows=some(case, 40, [5, 88, 18, 36, 37]))
    case = Case(kind, n_q, n_kv, D, 64, [(chunk * 2, 300)], lone=[3, 0], chunk=True, seed=3)
    assert len(case.lengths) * n_q >= 128 * 148
    case.check(case.call(), rows=some(case, 40, [18, 19, 36, 37, 420, 840]))


@pytest.mark.parametrize("kind", [sv.INT8, sv.E4M3])
def test_more_groups_and_pairs_than_a_cta_has_threads(kind):
    # 1100 groups of two or three rows, each a pair of query tiles of its own, then rows on their own
    rng = np.random.default_rng(4)
    groups = [([33 + int(x) for x in rng.integers(0, 40, 2 + g % 2)], 32) for g in range(1100)]
    groups[600] = ([], 5)
    groups[601] = ([50], 48)
    groups[1030] = ([0, 0], 32)
    case = Case(kind, 6, 2, 64, 16, groups, lone=[5, 0, 200], seed=5)
    edges = [int(case.starts[g]) + d for g in (600, 601, 1023, 1024, 1030) for d in (-1, 0, 1)]
    case.check(case.call(), rows=some(case, 60, edges))


def test_thousands_of_rows():
    # more rows than one round of the plan takes, most of them of one chunk; then the same with what does not count between them
    lens = list(range(1, 4301))
    case = Case(sv.INT8, 5, 1, 64, 128, [([150, 140], 128)], lone=[60] * 20, seed=6)
    case.check(case.call(), rows=some(case, 5))
    case = Case(sv.INT8, 5, 1, 64, 128, [([2, 3], 2), (lens, 4300), ([9, 1, 7], 1)], lone=[200, 0], chunk=True, seed=7)
    assert len(case.lengths) > 4096
    case.check(case.call(), rows=some(case, 25, [1, 2, 3, 4098, 4099, 4301, 4302, 4304]))
    case.shared[1] = 1000  # most rows have a part of their own
    case.check(case.call(), rows=some(case, 25, [1000, 1001, 1002, 1128, 4301]))
    case.seq[::7] = -1
    case.lengths[::5] = 0
    got = case.call().float().cpu()
    assert not got[::7].any() and not got[::5].any()
    case.check(case.call(), rows=[m for m in some(case, 40) if m % 7])


def test_repeated_calls_of_many_rows_agree_bit_by_bit():
    case = Case(sv.E4M3, 20, 5, 128, 64, [(list(range(700, 1700)), 1700), ([900 + i for i in range(40)], 832)], lone=[10, 2000], chunk=True, seed=8)
    want = case.call()
    case.check(want, rows=some(case, 12))
    assert all(torch.equal(case.call(), want) for _ in range(5))
    assert bl.bitlinear_poll_status() == 0


@pytest.mark.parametrize("n_q,n_kv,D", [(40, 8, 64), (64, 8, 64), (16, 8, 128), (40, 5, 128)])
@pytest.mark.parametrize("tiles", [1, 3])
@pytest.mark.parametrize("members", [3, 16])
def test_streams_of_uneven_work(n_q, n_kv, D, tiles, members):
    """Groups of at most 128 query rows give the two halves of a CTA different cache tiles: with an odd number of them one has less to do and runs ahead, up to the
    rows' own parts behind the groups."""
    shared = 128 * tiles - 64
    groups = [([shared + 1 + (7 * i + g) % 90 for i in range(members)], shared) for g in range(60)]
    case = Case(sv.INT8, n_q, n_kv, D, 64, groups, lone=[30, 200], chunk=True, seed=tiles)
    case.check(case.call(), rows=some(case, 10))
    assert bl.bitlinear_poll_status() == 0
