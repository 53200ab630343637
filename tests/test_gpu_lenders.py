"""Places of PagedDecodeStep whose blocks other places still read do not finish before those."""
import pytest
import torch

from oracle import serving as sv
from test_gpu_group_answers import bring, check_last_layer, make_step

pytestmark = pytest.mark.gpu


def prompt(st, gen, graph):
    for n in (8, 8, 8, 8, 5):
        bring(st, [n, 0, 0, 0, 0, 0, 0], gen, graph)
    assert st.fork(0, 1, 2) == 32
    st.group_places.copy_(torch.tensor([0, 3, 3], dtype=torch.int32))
    st.shared_rows.copy_(torch.tensor([32, 0], dtype=torch.int32))


@pytest.mark.parametrize("graph", [False, True])
def test_a_lender_waits_for_its_borrowers(graph):
    st = make_step(sv.INT8)
    if graph:
        st.capture()
    gen = torch.Generator().manual_seed(71)
    prompt(st, gen, graph)
    bring(st, [0, 1, 1, 0, 0, 0, 0], gen, graph)
    before = st.tables.clone(), st.lengths.clone(), int(st.n_free[0])
    bring(st, [-1, 0, 0, 0, 0, 0, 0], gen, graph)
    assert st.served[0] == 0 and torch.equal(st.lengths, before[1]) and torch.equal(st.tables, before[0]) and int(st.n_free[0]) == before[2]
    # the others' tokens of such a step are theirs, and so are the rows they read; another request takes blocks that are free
    bring(st, [-1, 1, -1, 4, 0, 0, 0], gen, graph)
    assert st.served.tolist() == [0, 1, 1, 1, 1, 1, 1] and st.lengths.tolist() == [37, 34, 0, 4, 0, 0, 0]
    for _ in range(3):
        bring(st, [-1, 1, 0, 3, 0, 0, 0], gen, graph)
        check_last_layer(st, sv.INT8)
        assert st.lengths[0] == 37
    # the last borrower and the lender together
    bring(st, [-1, -1, 0, -1, 0, 0, 0], gen, graph)
    assert (st.served == 1).all() and not st.lengths.any() and int(st.n_free[0]) == 20 and sorted(st.free_blocks.tolist()) == list(range(20))


def test_what_is_left_out_does_not_disturb_the_attention():
    st = make_step(sv.E4M3)
    gen = torch.Generator().manual_seed(72)
    prompt(st, gen, False)
    for new in ([-1, 2, 1, 3, 0, 0, 0], [-1, 1, -1, 2, 2, 0, 0], [-1, 3, 0, 2, 1, 1, 1]):
        bring(st, new, gen)
        check_last_layer(st, sv.E4M3)


@pytest.mark.parametrize("graph", [False, True])
def test_forks_of_forks(graph):
    st = make_step(sv.INT8)
    if graph:
        st.capture()
    gen = torch.Generator().manual_seed(73)
    prompt(st, gen, graph)
    st.shared_rows.zero_()
    for n in (8, 8, 2):  # place 1 goes on alone, and place 4 begins with all of it
        bring(st, [0, n, 0, 0, 0, 0, 0], gen, graph)
    assert st.fork(1, 4, 1) == 48 and st.fork(0, 3, 1) == 32
    bring(st, [-1, -1, -1, -1, 1, 0, 0], gen, graph)  # place 4 reads blocks of 0 and of 1; those that read none of 2's and 3's let them go
    assert st.served.tolist() == [0, 0, 1, 1, 1, 1, 1] and st.lengths.tolist() == [37, 50, 0, 0, 49, 0, 0]
    bring(st, [1, -1, 0, 0, 1, 0, 0], gen, graph)
    check_last_layer(st, sv.INT8)
    assert st.lengths.tolist() == [38, 50, 0, 0, 50, 0, 0]
    bring(st, [0, -1, 0, 0, -1, 0, 0], gen, graph)
    assert (st.served == 1).all() and st.lengths.tolist() == [38, 0, 0, 0, 0, 0, 0]
    # a place that was a lender may borrow, and one that has nothing of its own to lend may finish
    assert st.fork(0, 1, 1) == 32 and st.fork(1, 2, 1) == 32
    bring(st, [0, -1, 1, 0, 0, 0, 0], gen, graph)
    assert st.served[1] == 1 and st.lengths.tolist() == [38, 0, 33, 0, 0, 0, 0]
    bring(st, [-1, 0, 1, 0, 0, 0, 0], gen, graph)
    assert st.served[0] == 0 and st.lengths[0] == 38
    bring(st, [-1, 0, -1, 0, 0, 0, 0], gen, graph)
    assert not st.lengths.any() and int(st.n_free[0]) == 20 and sorted(st.free_blocks.tolist()) == list(range(20))
