"""A step of PagedDecodeStep with groups that one of its calls would refuse is refused before anything has changed."""
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from test_gpu_group_answers import DEV, ROWS, bring, make_step

pytestmark = pytest.mark.gpu


def state_of(st):
    return [t.clone() for t in (st.lengths, st.tables, st.free_blocks, st.n_free, st.borrowed, st.lenders, *(c.view(torch.uint8) for c in st.cache[0][:2]))]


def test_a_step_with_groups_is_refused_before_it_changes_anything():
    st = make_step(sv.INT8)
    gen = torch.Generator().manual_seed(81)
    for n in (8, 8, 2):
        bring(st, [n, 0, 0, 0, 0, 0, 0], gen)
    assert st.fork(0, 1, 2) == 16
    i32 = dict(dtype=torch.int32, device=DEV)
    st.group_places.copy_(torch.tensor([0, 3, 3], dtype=torch.int32))
    st.shared_rows.copy_(torch.tensor([16, 0], dtype=torch.int32))
    st.new_tokens.copy_(torch.tensor([1, -1, 2, 1, 0, 0, 0], dtype=torch.int32))
    ids, u = torch.zeros(ROWS, **i32), torch.zeros(ROWS, device=DEV)
    before = state_of(st)
    bad = {"shared_rows": [st.shared_rows.long(), st.shared_rows[:1], torch.zeros(4, **i32)[::2], st.shared_rows.cpu(), torch.zeros(2, 1, **i32)],
           "group_places": [st.group_places.float(), st.group_places[:2], st.group_places.cpu(), torch.zeros(4, **i32), torch.zeros(3, 1, **i32)],
           "new_tokens": [st.new_tokens.long(), st.new_tokens[:6], st.new_tokens.cpu(), st.new_tokens[:, None]]}
    for name, values in bad.items():
        kept = getattr(st, name)
        for value in values:
            setattr(st, name, value)
            with pytest.raises((TypeError, ValueError)):
                st.step(ids, u)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(before, state_of(st))), name
        setattr(st, name, kept)
    # 64-bit places are places, and numbers that lie apart are numbers
    st.group_places = st.group_places.long()
    apart = torch.zeros(14, **i32)
    apart[::2] = st.new_tokens
    st.new_tokens = apart[::2]
    st.step(ids, u)
    torch.cuda.synchronize()
    assert st.lengths.tolist() == [19, 0, 18, 1, 0, 0, 0] and bl.bitlinear_poll_status() == 0
