"""Log probabilities of given tokens, the policy loss and the preference loss with their gradients, against the 64-bit oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import learning as le
from paper_2504_12285_b200 import binding as bl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24  # half a step of fp32


def make_logits(T, V, dtype, seed, spread=2.0, offset=0, pad=0):
    """Logits [T, V] whose rows are V + pad apart and start `offset` elements behind a 16-byte border, and targets, mostly likely ones."""
    gen = torch.Generator().manual_seed(seed)
    stride = V + pad
    store = torch.full((offset + T * stride,), float("nan"), dtype=dtype)  # what lies between the rows must not be used
    x = store[offset:].view(T, stride)[:, :V]
    x.copy_(torch.randn(T, V, generator=gen) * spread)
    targets = torch.randint(0, V, (T,), generator=gen)
    x[torch.arange(T), targets] += (torch.rand(T, generator=gen) * 12).to(dtype)
    dev = store.to(DEV)[offset:].view(T, stride)[:, :V]
    return dev, targets.to(torch.int32).to(DEV)


def sum_error(V, mean_distance):
    """Relative error of a row's sum of exponentials: 2 ulp (2^-22) of the exponential, roundings of (l - max) * log2(e) at 2 and of the
    constant at 1 half step of the argument each, on average over the weights; at most V / 256 + 1 additions in a thread (with 4 or 8 elements more), 5 + 3 + 7
    joins of three roundings and an exponential each."""
    return 2.0 ** -22 + 3 * U * 1.45 * mean_distance + (V / 256 + 9) * U + 15 * (2.0 ** -22 + 4 * U)


def logp_error(r, V):
    """... of the log probability: the sum's, that of the logarithm (1 ulp) and the roundings of two differences."""
    logp, top, total, _, mean = r
    return sum_error(V, mean) + 2 * U * abs(math.log(total)) + 2 * U * (abs(logp) + abs(math.log(total)))


def check_gradient(got, want, r, V, target, dtype, slope, slope_error):
    """|got - want| element by element: the weight's and the sum's errors, that of the slope, four roundings, and the result's own."""
    logp, top, total, p, mean = r
    distance = -np.log(np.maximum(p, 1e-300)) - math.log(total)
    rel = 2.0 ** -22 + 3 * U * 1.45 * np.abs(distance) + sum_error(V, mean) + 4 * U
    tol = np.abs(want) * rel + p * slope_error
    # the target's: slope * (1 - p), where p is off by p * (error of logp); expm1 2 ulp
    tol[target] = abs(slope) * math.exp(logp) * logp_error(r, V) + abs(want[target]) * 6 * U - slope_error * math.expm1(logp)
    half = torch.finfo(dtype).eps / 2
    tol = tol + (np.abs(want) + tol) * half + (abs(slope) + 1) * 2.0 ** -125 + 2.0 ** -133  # exponentials below 2^-126 are 0; bf16's smallest step
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.nonzero(bad)[0][:5], got[bad][:5], want[bad][:5], tol[bad][:5])


def host(t):
    return t.double().cpu().numpy()


SHAPES = [(1, 1, F32), (3, 2, BF16), (5, 7, BF16), (4, 9, F32), (2, 33, F32), (6, 257, BF16), (3, 1000, F32), (40, 5003, BF16), (2, 18437, F32), (3, 32003, F32), (2, 128256, F32),
          (5, 128256, BF16), (1, 150001, F32), (2, 360448, F32), (2, 360441, BF16)]


@pytest.mark.parametrize("T,V,dtype", SHAPES)
@pytest.mark.parametrize("offset,pad", [(0, 0), (3, 5), (1, 8)])
def test_token_logprobs_and_gradient(T, V, dtype, offset, pad):
    x, targets = make_logits(T, V, dtype, 7 * V + T, offset=offset, pad=pad)
    if T > 2:
        targets[1] = -1
        targets[2] = V
    grad = torch.randn(T, generator=torch.Generator().manual_seed(3)).to(DEV)
    if T > 3:
        grad[3] = 0.0
    logp, stats = bl.bitlinear_token_logprobs(x, targets)
    out = torch.full((T, V + pad), 7.0, dtype=dtype, device=DEV)
    d = bl.bitlinear_token_logprobs_backward(x, targets, stats, grad, dlogits=out[:, :V])
    d2 = bl.bitlinear_token_logprobs_backward(x, targets, stats, grad)
    assert torch.equal(d, d2)
    assert (out[:, V:] == 7.0).all()  # nothing behind a row is written
    xs, ts, gs = host(x), targets.tolist(), grad.tolist()
    for t in range(T):
        r = le.row(xs[t], ts[t])
        if r is None:
            assert logp[t] == 0 and not d[t].any()
            continue
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, V)
        assert float(stats[t, 0]) == r[1] and abs(float(stats[t, 1]) - r[2]) <= r[2] * sum_error(V, r[4])
        check_gradient(host(d[t]), le.gradient(r[3], ts[t], r[0], gs[t]), r, V, ts[t], dtype, gs[t], 0.0)
    same = x.clone() if pad == 0 else None
    if same is not None:  # the gradient may go where the logits are
        assert bl.bitlinear_token_logprobs_backward(same, targets, stats, grad, dlogits=same) is same and torch.equal(same, d)


def test_logprobs_of_extreme_rows():
    inf, low, nan = math.inf, torch.finfo(F32).min, math.nan
    V = 4099
    x = torch.randn(9, V, generator=torch.Generator().manual_seed(1))
    x[0, 5:] = -inf                # few tokens allowed
    x[1, :] = -inf
    x[1, 7] = 3.0                  # one allowed
    x[2, :] = low                  # the type's lowest everywhere: an even distribution
    x[3, 100:] = low               # masked by the lowest
    x[4, 17] = nan
    x[5, 17] = inf
    x[6, :] = -inf                 # nothing allowed
    x[7] = x[7] * 1e30
    x[8, 0] = 3e38                 # far above the others
    targets = torch.tensor([3, 7, 9, 5, 2, 2, 2, int(x[7].argmax()), 0], dtype=torch.int32)
    xd, td = x.to(DEV), targets.to(DEV)
    logp, stats = bl.bitlinear_token_logprobs(xd, td)
    d = bl.bitlinear_token_logprobs_backward(xd, td, stats, torch.ones(9, device=DEV))
    for t in (0, 1, 2, 3, 7, 8):
        r = le.row(x[t].double().numpy(), int(targets[t]))
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, V), t
        assert abs(host(d[t]) - le.gradient(r[3], int(targets[t]), r[0], 1.0)).max() <= 1e-5, t
    assert torch.isnan(logp[4:7]).all() and torch.isnan(d[4:7]).all()
    # a masked token and a slope of 0 ask nothing of the row
    td[4], td[5], td[6] = -1, V, -5
    logp, stats = bl.bitlinear_token_logprobs(xd, td)
    d = bl.bitlinear_token_logprobs_backward(xd, td, stats, torch.ones(9, device=DEV))
    assert not logp[4:7].any() and not d[4:7].any()
    # a target of no weight
    x0 = xd[:1].contiguous()
    logp, stats = bl.bitlinear_token_logprobs(x0, torch.tensor([100], dtype=torch.int32, device=DEV))
    assert logp[0] == -inf
    d = bl.bitlinear_token_logprobs_backward(x0, torch.tensor([100], dtype=torch.int32, device=DEV), stats, torch.ones(1, device=DEV))
    assert float(d[0, 100]) == 1.0 and not d[0, 6:100].any()


def policy_case(T, V, dtype, seed, kl, **kw):
    x, targets = make_logits(T, V, dtype, seed, **kw)
    gen = torch.Generator().manual_seed(seed + 1)
    now, _ = bl.bitlinear_token_logprobs(x, targets)
    noise = lambda s: (torch.randn(T, generator=gen) * s).to(DEV)  # noqa: E731
    case = dict(old_logprobs=now + noise(0.3), advantages=noise(1.0), weights=torch.rand(T, generator=gen).to(DEV), clip_low=0.2, clip_high=0.3, kl_coef=kl,
                ref_logprobs=now + noise(0.4) if kl else None)
    if kl and T > 2:
        case["ref_logprobs"][1] = now[1] + 1e-3  # next to the reference
    return x, targets, case


def check_policy(x, targets, case, got):
    loss, token_loss, logp, d = got
    T, V = x.shape
    xs, ts = host(x), targets.tolist()
    old, adv = host(case["old_logprobs"]), host(case["advantages"])
    w = host(case["weights"]) if case["weights"] is not None else np.ones(T)
    ref = host(case["ref_logprobs"]) if case["ref_logprobs"] is not None else np.zeros(T)
    total, total_tol, cut = 0.0, 0.0, 0
    for t in range(T):
        r = le.row(xs[t], ts[t])
        if r is None or w[t] == 0:
            assert float(token_loss[t]) == 0 and (d is None or not d[t].any())
            continue
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, V)
        args = (old[t], adv[t], float(np.float32(case["clip_low"])), float(np.float32(case["clip_high"])), float(np.float32(case["kl_coef"])), ref[t])
        value, slope = le.policy_token(r[0], *args)
        e = logp_error(r, V)  # the loss moves by its slope, |A| r + kl |exp(d) - 1|, and rounds ten times
        size = abs(adv[t]) * math.exp(r[0] - old[t]) + args[4] * (math.exp(abs(ref[t] - r[0])))
        tol = w[t] * (size * (e + 10 * U) + abs(value) * 6 * U)
        assert abs(float(token_loss[t]) - w[t] * value) <= tol, t
        total, total_tol, cut = total + w[t] * value, total_tol + tol, cut + (slope == 0)
        if d is not None:
            check_gradient(host(d[t]), le.gradient(r[3], ts[t], r[0], w[t] * slope), r, V, ts[t], x.dtype, w[t] * slope, tol)
    assert abs(float(loss) - total) <= total_tol + abs(total) * U
    return cut


@pytest.mark.parametrize("T,V,dtype", [(1, 1, F32), (2, 5, BF16), (7, 129, F32), (30, 1003, BF16), (3, 32003, F32), (4, 128256, BF16), (2, 128256, F32), (2, 360448, F32)])
@pytest.mark.parametrize("kl", [0.0, 0.1])
def test_policy_loss(T, V, dtype, kl):
    x, targets, case = policy_case(T, V, dtype, 11 * V + T, kl)
    if T > 3:
        targets[0] = -1
        case["weights"][2] = 0.0
    got = bl.bitlinear_policy_loss(x, targets, **case, grad=True)
    check_policy(x, targets, case, got)
    without = bl.bitlinear_policy_loss(x, targets, **case)
    assert without[3] is None and all(torch.equal(a, b) for a, b in zip(got[:3], without[:3]))
    same = x.clone()  # the gradient in the logits' place
    again = bl.bitlinear_policy_loss(same, targets, **case, grad=same)
    assert again[3] is same and all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("offset,pad,d_offset,d_pad", [(1, 3, 0, 0), (5, 8, 2, 1), (0, 0, 1, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_loss_strided(offset, pad, d_offset, d_pad, dtype):
    T, V = 5, 2003
    x, targets, case = policy_case(T, V, dtype, 77, 0.05, offset=offset, pad=pad)
    case["weights"] = None
    store = torch.full((d_offset + T * (V + d_pad),), 7.0, dtype=dtype, device=DEV)
    out = store[d_offset:].view(T, V + d_pad)
    got = bl.bitlinear_policy_loss(x, targets, **case, grad=out[:, :V])
    check_policy(x, targets, case, got)
    assert (store[:d_offset] == 7.0).all() and (out[:, V:] == 7.0).all()


@pytest.mark.parametrize("T,V,dtype", [(148, 5, F32), (400, 1, BF16), (300, 129, BF16), (151, 32003, F32), (200, 8192, BF16), (149, 70001, BF16)])
@pytest.mark.parametrize("offset,pad", [(0, 0), (3, 9)])
def test_many_rows(T, V, dtype, offset, pad):
    """As many rows as SMs and more are streamed."""
    x, targets, case = policy_case(T, V, dtype, 5 * V + T, 0.1, offset=offset, pad=pad)
    targets[2], targets[T - 1] = -1, V
    case["weights"][5] = 0.0
    out = torch.full((T, V + pad), 7.0, dtype=dtype, device=DEV)
    got = bl.bitlinear_policy_loss(x, targets, **case, grad=out[:, :V])
    assert (out[:, V:] == 7.0).all()
    some = torch.tensor(sorted({0, 1, 2, 3, 5, T // 2, T - 2, T - 1}), device=DEV)
    pick = {k: (v[some].contiguous() if torch.is_tensor(v) else v) for k, v in case.items()}
    check_policy(x[some], targets[some], pick, (got[1][some].double().sum(), got[1][some], got[2][some], got[3][some]))
    assert abs(float(got[0]) - float(got[1].double().sum())) <= U * abs(float(got[0])) + 1e-30
    same = x.clone()
    assert torch.equal(bl.bitlinear_policy_loss(same, targets, **case, grad=same)[3], got[3]) or pad  # (rows that start elsewhere are summed in another order)
    assert bl.bitlinear_policy_loss(x, targets, **case)[3] is None
    logp, stats = bl.bitlinear_token_logprobs(x, targets)
    assert torch.equal(logp, got[2])
    xs, ts = host(x[some]), targets[some].tolist()
    for i, t in enumerate(some.tolist()):
        r = le.row(xs[i], ts[i])
        if r is not None:
            assert float(stats[t, 0]) == r[1] and abs(float(stats[t, 1]) - r[2]) <= r[2] * sum_error(V, r[4])


def test_many_extreme_rows():
    inf, low, nan = math.inf, torch.finfo(F32).min, math.nan
    x = torch.randn(160, 4099, generator=torch.Generator().manual_seed(2))
    x[0, 5:], x[1], x[2, 100:], x[3, 17], x[4, 17], x[5] = -inf, low, low, nan, inf, -inf
    x[6] *= 1e30
    x[7, 0], x[8], x[9, 3] = 3e38, x[8] * 1e6, nan
    targets = torch.zeros(160, dtype=torch.int32)
    targets[6] = int(x[6].argmax())
    targets[8] = int(x[8].argmax())
    targets[9] = -1
    args = [torch.zeros(160, device=DEV), torch.ones(160, device=DEV)]
    _, _, logp, d = bl.bitlinear_policy_loss(x.to(DEV), targets.to(DEV), *args, clip_low=1.0, clip_high=1e9, grad=True)  # the loss is -exp(logp), so is its slope
    for t in (0, 1, 2, 6, 7, 8, 10):
        r = le.row(x[t].double().numpy(), int(targets[t]))
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, 4099), t
        assert abs(host(d[t]) - le.gradient(r[3], int(targets[t]), r[0], -math.exp(r[0]))).max() <= 1e-5, t
    assert torch.isnan(logp[3:6]).all() and torch.isnan(d[3:6]).all() and not d[9].any() and not logp[9]


def test_policy_clips_on_both_sides():
    x, targets, case = policy_case(64, 300, F32, 5, 0.0)
    assert 5 < check_policy(x, targets, case, bl.bitlinear_policy_loss(x, targets, **case, grad=True)) < 60


def test_tokens_of_weight_zero_count_for_nothing():
    x, targets, case = policy_case(6, 500, F32, 6, 0.1)
    case["weights"][1:4] = 0.0
    want = bl.bitlinear_policy_loss(x, targets, **case, grad=True)
    case["old_logprobs"][1], case["advantages"][2], case["ref_logprobs"][3] = math.nan, math.inf, -math.inf
    x[3] = math.nan
    got = bl.bitlinear_policy_loss(x, targets, **case, grad=True)
    for i in (0, 1, 3):
        assert torch.equal(got[i], want[i])
    assert not torch.isnan(got[2][:3]).any()


def test_policy_gradient_against_differences():
    """The gradient against differences of the oracle's loss in 64 bits: central differences of step h are off by h^2 / 6 times the third derivative."""
    T, V = 3, 11
    x, targets, case = policy_case(T, V, F32, 8, 0.2)
    d = host(bl.bitlinear_policy_loss(x, targets, **case, grad=True)[3])
    xs, ts = host(x), targets.tolist()
    old, adv, w, ref = (host(case[n]) for n in ("old_logprobs", "advantages", "weights", "ref_logprobs"))

    def loss(row, t):
        return w[t] * le.policy_token(le.row(row, ts[t])[0], old[t], adv[t], 0.2, 0.3, 0.2, ref[t])[0]

    h = 1e-4
    for t in range(T):
        for v in range(V):
            up, down = xs[t].copy(), xs[t].copy()
            up[v] += h
            down[v] -= h
            assert abs((loss(up, t) - loss(down, t)) / (2 * h) - d[t, v]) <= 1e-5


def pairs_case(sizes, V, dtype, seed, **kw):
    T = sum(sizes)
    x, targets = make_logits(max(T, 1), V, dtype, seed, **kw)
    x, targets = x[:T], targets[:T]
    gen = torch.Generator().manual_seed(seed + 1)
    cu = np.concatenate([[0], np.cumsum(sizes)])
    for a, b in zip(cu[:-1], cu[1:]):
        targets[a: a + (b - a) // 4] = -100
    logp = bl.bitlinear_token_logprobs(x, targets)[0]
    ref = torch.stack([logp[a:b].sum() for a, b in zip(cu[:-1], cu[1:])]) + (torch.randn(len(sizes), generator=gen) * 5).to(DEV)
    return x, targets, torch.from_numpy(cu.astype(np.int32)).to(DEV), ref.contiguous()


def check_pairs(x, targets, cu, ref, beta, smooth, got):
    loss, pair_loss, seq_logp, logp, d = got
    T, V = x.shape
    xs, ts, cus, refs = host(x), targets.tolist(), cu.tolist(), host(ref)
    beta, smooth = float(np.float32(beta)), float(np.float32(smooth))
    rows = [le.row(xs[t], ts[t]) for t in range(T)]
    err = [logp_error(r, V) if r else 0.0 for r in rows]
    for t, r in enumerate(rows):
        assert abs(float(logp[t]) - (r[0] if r else 0.0)) <= err[t]
    P, losses, loss_tol, covered = len(refs) // 2, [], 0.0, set()
    for i in range(P):
        span = [range(cus[2 * i + k], cus[2 * i + k + 1]) for k in (0, 1)]
        sums = [math.fsum(rows[t][0] for t in s if rows[t]) for s in span]
        errs = [math.fsum(err[t] for t in s) for s in span]
        for k in (0, 1):
            assert abs(float(seq_logp[2 * i + k]) - sums[k]) <= errs[k] + abs(sums[k]) * U
        value, slope = le.pair(sums[0] - refs[2 * i], sums[1] - refs[2 * i + 1], beta, smooth, P)
        delta = beta * ((sums[0] - refs[2 * i]) - (sums[1] - refs[2 * i + 1]))
        delta_err = beta * sum(errs) + abs(delta) * 2 * U
        tol = delta_err + (abs(delta) + 1) * 12 * U  # |d loss / d delta| <= 1; a dozen roundings of terms no larger than |delta| + 1
        assert abs(float(pair_loss[i]) - value) <= tol
        losses.append(value)
        loss_tol += tol / P
        if d is None:
            continue
        for k in (0, 1):
            for t in span[k]:
                covered.add(t)
                if rows[t] is None:
                    assert not d[t].any()
                    continue
                s = slope if k == 0 else -slope
                # |slope| <= beta / P, its change with delta a quarter of that; eight roundings
                check_gradient(host(d[t]), le.gradient(rows[t][3], ts[t], rows[t][0], s), rows[t], V, ts[t], x.dtype, s, beta / P * (0.25 * delta_err + 8 * U))
    assert abs(float(loss) - math.fsum(losses) / P) <= loss_tol + U * abs(float(loss))
    if d is not None:
        for t in set(range(T)) - covered:
            assert not d[t].any()


@pytest.mark.parametrize("sizes,V,dtype", [([1, 1], 2, F32), ([3, 5], 130, BF16), ([0, 4, 7, 0], 1003, F32), ([40, 1, 2, 300], 517, BF16), ([5, 3, 2, 2, 9, 1], 32003, F32), ([3, 4], 128256, BF16)])
@pytest.mark.parametrize("smooth", [0.0, 0.1])
def test_preference_loss(sizes, V, dtype, smooth):
    case = pairs_case(sizes, V, dtype, 3 * V + len(sizes))
    for beta in (0.1, 1.5):
        got = bl.bitlinear_preference_loss(*case, beta=beta, label_smoothing=smooth, grad=True)
        check_pairs(*case, beta, smooth, got)
        without = bl.bitlinear_preference_loss(*case, beta=beta, label_smoothing=smooth)
        assert without[4] is None and all(torch.equal(a, b) for a, b in zip(got[:4], without[:4]))
        same = case[0].clone()
        again = bl.bitlinear_preference_loss(same, *case[1:], beta=beta, label_smoothing=smooth, grad=same)
        assert torch.equal(again[4], got[4])


def test_preference_loss_rows_of_no_answer_and_many_pairs():
    x, targets, cu, ref = pairs_case([2] * 40, 67, F32, 9, offset=1, pad=3)
    inner = cu[4:13].contiguous()  # answers 4 .. 11 of the rows: those in front and behind belong to none
    check_pairs(x, targets, inner, ref[4:12].contiguous(), 0.3, 0.0, bl.bitlinear_preference_loss(x, targets, inner, ref[4:12].contiguous(), beta=0.3, grad=True))
    sizes = np.random.default_rng(1).integers(0, 3, 2 * 1500).tolist()
    case = pairs_case(sizes, 19, F32, 10)
    check_pairs(*case, 0.2, 0.05, bl.bitlinear_preference_loss(*case, beta=0.2, label_smoothing=0.05, grad=True))
    # offsets outside the rows, and ones that decrease: nothing is read or written out of place
    bad = torch.tensor([-5, 3, 10 ** 6, 2, 1], dtype=torch.int32, device=DEV)
    bl.bitlinear_preference_loss(x, targets, bad, torch.zeros(4, device=DEV), grad=True)
    torch.cuda.synchronize()
    # no rows at all: two empty answers, loss log 2
    empty = bl.bitlinear_preference_loss(x[:0], targets[:0], torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(2, device=DEV), grad=True)
    assert abs(float(empty[0]) - math.log(2)) <= 2 * U and empty[4].shape == (0, 67)
    assert float(bl.bitlinear_policy_loss(x[:0], targets[:0], torch.zeros(0, device=DEV), torch.zeros(0, device=DEV))[0]) == 0.0
    assert bl.bitlinear_token_logprobs(x[:0], targets[:0])[0].numel() == 0


def test_large_differences_of_a_pair():
    x, targets, cu, _ = pairs_case([3, 4], 50, F32, 12)
    for gap in (300.0, -300.0, 3e4):
        ref = torch.tensor([0.0, gap], device=DEV)
        check_pairs(x, targets, cu, ref, 1.0, 0.1, bl.bitlinear_preference_loss(x, targets, cu, ref, beta=1.0, label_smoothing=0.1, grad=True))


def test_losses_recorded_and_on_two_streams():
    x, targets, case = policy_case(33, 5001, BF16, 20, 0.05)
    p = pairs_case([8, 9, 10, 6], 5001, BF16, 21)
    want = bl.bitlinear_policy_loss(x, targets, **case, grad=True), bl.bitlinear_preference_loss(*p, grad=True)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = bl.bitlinear_policy_loss(x, targets, **case, grad=True), bl.bitlinear_preference_loss(*p, grad=True)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    x.copy_(x.flip(1))  # the recording reads what is there when it is replayed
    want = bl.bitlinear_policy_loss(x, targets, **case, grad=True)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(want, got[0]))
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(6):
        streams[i % 2].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(streams[i % 2]):
            outs.append(bl.bitlinear_policy_loss(x, targets, **case, grad=True) if i % 2 else bl.bitlinear_preference_loss(*p, grad=True))
    torch.cuda.synchronize()
    ref = bl.bitlinear_preference_loss(*p, grad=True)
    for i, o in enumerate(outs):
        assert all(torch.equal(s, t) for s, t in zip(o, want if i % 2 else ref))


def test_offsets_past_32_bits():
    """Rows whose elements lie beyond 2^31: the last row of a strided matrix."""
    V, T, stride = 1009, 3, 1 << 30
    store = torch.empty(2 * stride + V, dtype=BF16, device=DEV)
    x = store.as_strided((T, V), (stride, 1))
    small, targets = make_logits(T, V, BF16, 30)
    x.copy_(small)
    logp, stats = bl.bitlinear_token_logprobs(x, targets)
    d = bl.bitlinear_token_logprobs_backward(x, targets, stats, torch.ones(T, device=DEV), dlogits=x)
    xs = host(small)
    for t, target in enumerate(targets.tolist()):  # (rows that start elsewhere are summed in another order: the oracle, not another call)
        r = le.row(xs[t], target)
        assert abs(float(logp[t]) - r[0]) <= logp_error(r, V)
        check_gradient(host(d[t]), le.gradient(r[3], target, r[0], 1.0), r, V, target, BF16, 1.0, 0.0)
