"""Serving entry points: what has to be refused before anything is written, and what the oracle's tolerances can tell apart.
Needs no GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from paper_2504_12285_b200 import chain as gpu_chain
from test_gpu_serving import attend_case


class Recorder:
    """Stands in for the library: notes the calls and launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.mark.parametrize("out", [torch.zeros(6, 64, dtype=torch.bfloat16), torch.zeros(20, 32, dtype=torch.bfloat16), torch.zeros(20 * 64, dtype=torch.bfloat16),
                                 torch.zeros(19, 64, dtype=torch.bfloat16), torch.zeros(20, 64)])
def test_embed_refuses_an_output_that_its_rows_do_not_fit(monkeypatch, out):
    lib = Recorder()
    monkeypatch.setattr(bl, "lib", lambda: lib)
    monkeypatch.setattr(bl, "_stream", lambda: 0)

    def typed(t, dtype, name):
        if t.dtype != dtype:
            raise TypeError(name)
        return t

    monkeypatch.setattr(bl, "_dev", typed)
    ids, table = torch.zeros(20, dtype=torch.int32), torch.zeros(50, 64, dtype=torch.bfloat16)
    with pytest.raises((TypeError, ValueError)):
        bl.bitlinear_embed(ids, table, out=out)
    assert not lib.calls
    for n in (20, 30):
        good = torch.zeros(n, 64, dtype=torch.bfloat16)
        assert bl.bitlinear_embed(ids, table, out=good) is good and lib.calls[-1][1][2] == 20


@pytest.mark.parametrize("rows", [0, -1, 17, 64])
def test_paged_decode_step_refuses_rows_that_the_output_head_cannot_take(rows):
    with pytest.raises(ValueError, match="rows"):
        gpu_chain.PagedDecodeStep([], torch.zeros(50, 64, dtype=torch.bfloat16), rows, 4, 8, 16, 4, 64, 128, 1, 1, 64, device="cpu")


# ------------------------------------------------------------------------------------------------- attention's tolerance

def in_digits(q, units):
    """Queries [M, n_q, D] in whole units, `units` of them to each head's largest magnitude."""
    step = np.abs(q).max(-1, keepdims=True) / units
    return np.rint(q / step) * step


def outlier_case(n_q, n_kv, D, rows, lengths, seed, size):
    """Queries with one channel `size` times the others, over keys that have nothing in that channel and all they have in four others: the small
    channels alone decide the scores."""
    q, codes, scales, tables = attend_case(sv.INT8, n_q, n_kv, D, rows, lengths, seed)
    rng = np.random.default_rng(seed)
    q = q.float().view(len(lengths), n_q, D)
    dims = rng.permutation(D)[:5]
    q[..., int(dims[4])] = float(size)
    keep = np.zeros(D, bool)
    keep[dims[:4]] = True
    codes[0][..., ~keep] = 0
    scales[0] *= 8.0
    return q.reshape(len(lengths), -1).to(torch.bfloat16), codes, scales, tables


def share_of_tolerance(q, codes, scales, tables, lengths, n_q, n_kv, D, units):
    """The largest error that queries of so many units make, as a share of what the GPU tests allow."""
    worst = 0.0
    qn = q.float().numpy().astype(np.float64).reshape(len(lengths), n_q, D)
    for m, n in enumerate(lengths):
        ref, vmax, err = sv.attention8(qn[m], *codes, *scales, tables[m], n, n_q, n_kv, D, sv.INT8)
        got = sv.attention8(in_digits(qn[m], units), *codes, *scales, tables[m], n, n_q, n_kv, D, sv.INT8)[0]
        worst = max(worst, float((np.abs(got - ref) / (2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2 * err + 1e-6) * vmax)).max()))
    return worst


def test_attention_tolerance_notices_coarse_queries():
    # the planted mistakes are the oracle's own: queries of 8 bits on ordinary inputs, of 15 bits beside a channel of 4000
    lengths = [300, 40, 17]
    case = attend_case(sv.INT8, 4, 2, 64, 16, lengths, 7)
    assert share_of_tolerance(*case, lengths, 4, 2, 64, 127) > 1.0
    assert share_of_tolerance(*case, lengths, 4, 2, 64, 127 * 128 * 256) < 0.1
    case = outlier_case(4, 2, 64, 16, lengths, 8, 4000.0)
    assert share_of_tolerance(*case, lengths, 4, 2, 64, 127 * 128) > 2.0
    assert share_of_tolerance(*case, lengths, 4, 2, 64, 127 * 128 * 256) < 0.5


def test_oracle_keeps_what_is_not_a_number_in_sight():
    for kind in (sv.INT8, sv.E4M3):
        for bad in (math.nan, math.inf, -math.inf):
            codes, scale = np.full((2, 1, 16, 64), 5, np.uint8), np.full((2, 1), 0.5, np.float32)
            values = np.ones((2, 1, 64))
            values[1, 0, 3] = bad
            sv.append8(values, [4, 20], codes, scale, kind)
            assert scale[0, 0] == 0.5 and np.isnan(scale[1, 0]) and (codes[0, 0, :4] == 5).all()
            sv.append8(np.ones((1, 1, 64)), [21], codes, scale, kind)
            assert np.isnan(scale[1, 0])  # a finite row does not hide it
            sv.append8(np.ones((1, 1, 64)), [16], codes, scale, kind)
            assert scale[1, 0] == sv.scale_for(1.0, kind)  # the block's next owner does not see it
