"""Groups whose first rows are shorter than what the group shares, with tables that end where they do."""
import numpy as np
import pytest

from oracle import serving as sv
from test_gpu_shared_attention import Case

pytestmark = pytest.mark.gpu


def end_tables(case):
    """Every table names the blocks of its own sequence's rows and no others."""
    for s in range(len(case.tables)):
        case.tables[s, -(-max(int(case.lengths[case.seq == s].max()), 0) // case.rows):] = -1
    return case


@pytest.mark.parametrize("kind,n_q,n_kv,D,rows", [(sv.INT8, 20, 5, 128, 64), (sv.E4M3, 16, 2, 64, 16), (sv.E4M3, 6, 2, 128, 32)])
@pytest.mark.parametrize("lens", [[20, 300, 0, 290], [0, 5, 256, 256], [1, 2, 130], [100] * 70 + [256] * 3, [256] + [3] * 140 + [255, 254]])
def test_short_rows_come_first(kind, n_q, n_kv, D, rows, lens):
    case = end_tables(Case(kind, n_q, n_kv, D, rows, [(lens, 256), (lens[::-1], 128)], lone=[40], seed=len(lens)))
    case.check(case.call())


@pytest.mark.parametrize("kind", [sv.INT8, sv.E4M3])
def test_short_rows_come_first_in_many_groups(kind):
    # more groups and pairs than the plan keeps in shared memory
    case = end_tables(Case(kind, 4, 1, 64, 16, [([5 + g % 20, 64 + g % 7, 70], 48) for g in range(1100)], seed=9))
    case.check(case.call(), rows=sorted(set(np.random.default_rng(0).integers(0, len(case.lengths), 60).tolist()) | {0, 1, 2, 3297, 3298, 3299}))
