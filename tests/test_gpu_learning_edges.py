"""The losses on drawn tokens where a factor of zero meets what is infinite, against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import learning as le
from paper_2504_12285_b200 import binding as bl
from test_gpu_token_loss import DEV, F32, U, check_gradient, host, logp_error

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("smooth", [0.0, 0.25, 1.0])
@pytest.mark.parametrize("pairs", [2, 12])
def test_answers_of_probability_zero(pairs, smooth):
    """A masked token in the rejected answer (the margin is +infinity) or in the preferred one (-infinity): a term of the loss whose factor is 0 counts for nothing."""
    T, V, beta = 4 * pairs, 301, 0.3
    gen = torch.Generator().manual_seed(pairs)
    x = torch.randn(T, V, generator=gen)
    x[:, 250:] = -math.inf
    targets = torch.randint(0, 250, (T,), generator=gen).to(torch.int32)
    targets[3], targets[4] = 280, 300  # the first pair's rejected answer, the second pair's preferred one
    cu = torch.arange(0, T + 1, 2, dtype=torch.int32)
    ref = torch.randn(2 * pairs, generator=gen) * 3 - 10
    loss, pair_loss, seq, logp, d = bl.bitlinear_preference_loss(x.to(DEV), targets.to(DEV), cu.to(DEV), ref.to(DEV), beta=beta, label_smoothing=smooth, grad=True)
    beta = float(np.float32(beta))
    rows = [le.row(host(x[t]), int(targets[t])) for t in range(T)]
    values = []
    for i in range(pairs):
        s = [sum(rows[t][0] for t in range(4 * i + 2 * k, 4 * i + 2 * k + 2)) for k in (0, 1)]
        value, slope = le.pair(s[0] - float(ref[2 * i]), s[1] - float(ref[2 * i + 1]), beta, smooth, pairs)
        values.append(value)
        assert [float(seq[2 * i + k]) for k in (0, 1)] == [pytest.approx(v, rel=1e-6) for v in s]
        if math.isinf(value):
            assert float(pair_loss[i]) == value
        else:
            assert abs(float(pair_loss[i]) - value) <= 1e-5 * (1 + abs(value)), i
        for t in range(4 * i, 4 * i + 4):
            sign = slope if t < 4 * i + 2 else -slope
            want = le.gradient(rows[t][3], int(targets[t]), rows[t][0], sign)
            if math.isinf(rows[t][0]):
                assert np.abs(host(d[t]) - want).max() <= beta / pairs * 1e-5 and host(d[t])[int(targets[t])] == pytest.approx(sign, rel=1e-6), t
            else:
                check_gradient(host(d[t]), want, rows[t], V, int(targets[t]), F32, sign, beta / pairs * 1e-5)
    assert values[0] == (0.0 if smooth == 0 else math.inf) and values[1] == (0.0 if smooth == 1 else math.inf)
    want = math.fsum(values) / pairs if all(map(math.isfinite, values)) else math.inf
    assert float(loss) == want if math.isinf(want) else abs(float(loss) - want) <= 1e-5 * (1 + want)


@pytest.mark.parametrize("T", [5, 160])
def test_advantages_of_zero(T):
    """Answers that are all rewarded alike have advantages of 0: the ratio, which leaves fp32 where a token was all but impossible when it was drawn, is multiplied by it."""
    V = 700
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(T))
    targets = torch.arange(T, dtype=torch.int32)
    rows = [le.row(host(x[t]), t) for t in range(T)]
    old = torch.tensor([r[0] for r in rows], dtype=F32) + 0.05
    old[1], old[2], old[3] = -150.0, -1e10, -150.0
    adv = torch.ones(T)
    adv[:3], adv[3] = 0.0, 2.0
    ref = torch.tensor([r[0] for r in rows], dtype=F32) - 0.3
    for kl in (0.0, 0.25):
        loss, token_loss, logp, d = bl.bitlinear_policy_loss(x.to(DEV), targets.to(DEV), old.to(DEV), adv.to(DEV), kl_coef=kl, ref_logprobs=ref.to(DEV), grad=True)
        low = float(np.float32(0.2))
        for t in range(T):
            if t in (1, 2):  # (the ratio is multiplied by 0; one of the two is past 64 bits as well)
                value, slope = le.policy_token(rows[t][0], rows[t][0], 0.0, low, low, kl, float(ref[t]))
            else:
                value, slope = le.policy_token(rows[t][0], float(old[t]), float(adv[t]), low, low, kl, float(ref[t]))
            tol = (abs(float(adv[t])) * 1.2 + kl) * (logp_error(rows[t], V) + 10 * U) + abs(value) * 6 * U
            assert abs(float(token_loss[t]) - value) <= tol, t
            check_gradient(host(d[t]), le.gradient(rows[t][3], t, rows[t][0], slope), rows[t], V, t, F32, slope, tol)
        assert abs(float(loss) - float(token_loss.double().sum())) <= U * abs(float(loss))
    # what is not a number stays one
    old[0] = math.nan
    assert torch.isnan(bl.bitlinear_policy_loss(x.to(DEV), targets.to(DEV), old.to(DEV), adv.to(DEV))[1][0])
    old[0], x[0, 5] = 0.0, math.nan
    assert torch.isnan(bl.bitlinear_policy_loss(x.to(DEV), targets.to(DEV), old.to(DEV), adv.to(DEV))[1][0])
