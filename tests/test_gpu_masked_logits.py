"""Rows whose tokens are masked by large negative logits, anywhere in the row: log probabilities, statistics, losses and gradients against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import learning as le
from paper_2504_12285_b200 import binding as bl
from test_gpu_token_loss import BF16, DEV, F32, U, check_gradient, host, logp_error, sum_error

pytestmark = pytest.mark.gpu
MASKS = [-1e5, -5e6, -3e9, -1e10, -1e12, -1e20, -1e30, -1e38, -3e38, torch.finfo(BF16).min, torch.finfo(F32).min]
PLACES = ["front", "behind", "scattered", "steps"]


def masked(V, dtype, seed):
    """A row of ordinary logits for every mask and place of it, and a token of each that is not masked.  Free are 200 tokens, or a third of the row behind masks that rise in steps."""
    gen = torch.Generator().manual_seed(seed)
    rows, targets = [], []
    for mask in MASKS:
        if dtype == BF16 and mask == torch.finfo(F32).min:
            continue
        for place in PLACES:
            x = torch.randn(V, generator=gen) * 2.0
            if place == "front":
                x[:-200] = mask
                free = V - 200 + torch.randint(0, 200, (1,), generator=gen)
            elif place == "behind":
                x[200:] = mask
                free = torch.randint(0, 200, (1,), generator=gen)
            elif place == "scattered":
                some = torch.randperm(V, generator=gen)[:200]
                keep = x[some]
                x[:] = mask
                x[some] = keep
                free = some[:1]
            else:
                x[:V // 3], x[V // 3:2 * V // 3] = mask, mask / 3
                free = 2 * V // 3 + torch.randint(0, V // 4, (1,), generator=gen)
            rows.append(x)
            targets.append(int(free))
    x = torch.stack(rows).to(dtype)
    return x, torch.tensor(targets, dtype=torch.int32)


def check_rows(x, targets, logp, stats, d, slopes, dtype):
    """Row by row: the log probability and, where given, (max, sum) and the gradient for a slope."""
    V = x.shape[1]
    for t in range(x.shape[0]):
        r = le.row(host(x[t]), int(targets[t]))
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, V), (t, float(logp[t]), r[0])
        if stats is not None:
            assert float(stats[t, 0]) == r[1] and abs(float(stats[t, 1]) - r[2]) <= r[2] * sum_error(V, r[4]), t
        if d is not None:
            check_gradient(host(d[t]), le.gradient(r[3], int(targets[t]), r[0], slopes[t]), r, V, int(targets[t]), dtype, slopes[t], abs(slopes[t]) * (logp_error(r, V) + 8 * U))


# fewer rows than SMs (rows on chip) and more (rows streamed); a thread has several units of its row either way
@pytest.mark.parametrize("V,copies", [(70001, 1), (20011, 5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_rows(V, copies, dtype):
    x, targets = masked(V, dtype, V)
    n = x.shape[0]
    assert (n * copies < 100) == (copies == 1)
    xd, td = x.to(DEV).repeat(copies, 1), targets.to(DEV).repeat(copies)
    want = torch.tensor([le.row(host(x[t]), int(targets[t]))[0] for t in range(n)])
    logp, stats = bl.bitlinear_token_logprobs(xd, td)
    one = torch.full((n * copies,), 0.7, device=DEV)
    d = bl.bitlinear_token_logprobs_backward(xd, td, stats, one)
    check_rows(x, targets, logp, stats, d, [float(np.float32(0.7))] * n, dtype)
    # the policy loss on the side that is not cut: -r A, which is its slope, too
    old = (want + 0.1).to(torch.float32).to(DEV).repeat(copies)
    got = bl.bitlinear_policy_loss(xd, td, old, one, grad=True)
    slopes = [-math.exp(float(want[t]) - float(old[t])) * float(one[0]) for t in range(n)]
    check_rows(x, targets, got[2], None, got[3], slopes, dtype)
    for t in range(n):
        assert abs(float(got[1][t]) - slopes[t]) <= abs(slopes[t]) * (logp_error(le.row(host(x[t]), int(targets[t])), V) + 10 * U)
    assert abs(float(got[0]) - copies * math.fsum(slopes)) <= 1e-5 * abs(math.fsum(slopes)) * copies
    # pairs of two answers of one token each (and, of an odd number of rows, none in the last)
    pairs = n * copies // 2
    cu = torch.arange(2 * pairs + 1, dtype=torch.int32, device=DEV)
    ref = want.to(torch.float32).repeat(copies)[:2 * pairs].contiguous().to(DEV)
    out = bl.bitlinear_preference_loss(xd, td, cu, ref, beta=0.5, grad=True)
    # the reference is the model itself: every margin is 0, off by the errors of two log probabilities and of two roundings of theirs
    assert torch.isfinite(out[3]).all() and torch.isfinite(out[4].float()).all()
    assert (out[1] - math.log(2)).abs().max() <= 1e-4 and abs(float(out[0]) - math.log(2)) <= 1e-4
    check_rows(x[:2 * pairs], targets[:2 * pairs], out[3], None, None, None, dtype)
    slope = 0.5 / 2 / pairs
    for t in range(0, min(n, 2 * pairs)):
        r = le.row(host(x[t]), int(targets[t]))
        s = slope if t % 2 else -slope
        check_gradient(host(out[4][t]), le.gradient(r[3], int(targets[t]), r[0], s), r, V, int(targets[t]), dtype, s, slope * 1e-4)


@pytest.mark.parametrize("T", [8, 160])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_is_not_a_number_stays_in_sight_behind_masks(T, dtype):
    """A NaN or +infinity among masked tokens, in front of the free ones, between them and behind, is not lost with the masks; the rows around it are as they were."""
    V = 20011
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(T)).to(dtype)
    x[:, :-300] = -1e30
    x[1, 0], x[2, 7000], x[3, V - 1], x[4, 5000], x[5, 8] = math.nan, math.nan, math.nan, math.inf, math.nan
    x[5, :V // 2], x[5, 8] = -1e10, math.nan
    x[6, :] = torch.finfo(dtype).min  # one weight for all
    targets = torch.full((T,), V - 5, dtype=torch.int32, device=DEV)
    xd = x.to(DEV)
    zero, one = torch.zeros(T, device=DEV), torch.ones(T, device=DEV)
    logp, stats = bl.bitlinear_token_logprobs(xd, targets)
    d = bl.bitlinear_token_logprobs_backward(xd, targets, stats, one)
    _, token_loss, logp2, d2 = bl.bitlinear_policy_loss(xd, targets, zero, one, grad=True)
    for got in (logp, logp2, token_loss, d.float().sum(1), d2.float().sum(1)):
        assert torch.isnan(got[1:6]).all() and torch.isfinite(got[[0, 6, 7]]).all()
    for t in (0, 6, 7):
        r = le.row(host(x[t]), V - 5)
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, V) and abs(float(logp2[t]) - r[0]) <= logp_error(r, V)


@pytest.mark.parametrize("V,copies", [(70001, 1), (20011, 60)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_targets(V, copies, dtype):
    """A token that is masked itself: its log probability is as low as its logit, and the gradient is that of a probability of zero."""
    x = torch.randn(3, V, generator=torch.Generator().manual_seed(5)).to(dtype)
    for t, mask in enumerate((-1e10, -1e30, torch.finfo(dtype).min)):
        x[t, : V // 2] = mask
    xd, td = x.to(DEV).repeat(copies, 1), torch.tensor([9, 4000, V // 2 - 1], dtype=torch.int32, device=DEV).repeat(copies)
    logp, stats = bl.bitlinear_token_logprobs(xd, td)
    d = bl.bitlinear_token_logprobs_backward(xd, td, stats, torch.ones(3 * copies, device=DEV))
    check_rows(x, td.cpu()[:3], logp, stats, d, [1.0] * 3, dtype)


@pytest.mark.parametrize("V", [196609, 300001, 360448])
@pytest.mark.parametrize("free", [40, 3000])
def test_masked_rows_of_a_large_vocabulary(V, free):
    """Few tokens are free, so that most threads meet masks alone and go over their part twice, next to threads that do not; masks of several sizes stand among each other."""
    gen = torch.Generator().manual_seed(V + free)
    levels = torch.tensor([-1e7, -1e10, -1e30, -1e38, -3e38, torch.finfo(F32).min, -math.inf])
    x = levels[torch.randint(0, 7, (4, V), generator=gen)]
    for t in range(4):
        some = torch.randperm(V, generator=gen)[:free]
        x[t, some] = torch.randn(free, generator=gen) * 3.0
    x[3] = torch.where(x[3] > -1e6, torch.tensor(-1e7), x[3])  # none is free: those of the highest level share all
    targets = x.argmax(1).to(torch.int32)
    xd, td = x.to(DEV), targets.to(DEV)
    logp, stats = bl.bitlinear_token_logprobs(xd, td)
    d = bl.bitlinear_token_logprobs_backward(xd, td, stats, torch.ones(4, device=DEV))
    check_rows(x, targets, logp, stats, d, [1.0] * 4, F32)
    want = [le.row(host(x[t]), int(targets[t]))[0] for t in range(4)]
    old = torch.tensor(want, dtype=F32)
    got = bl.bitlinear_policy_loss(xd, td, old.to(DEV), torch.ones(4, device=DEV), grad=True)
    check_rows(x, targets, got[2], None, got[3], [-math.exp(w - float(o)) for w, o in zip(want, old)], F32)
