"""Token log probabilities, policy and preference loss: what the host refuses before anything is launched, and the oracle's own pins.  Needs
no GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import learning as le
from paper_2504_12285_b200 import binding as bl

FAKE = 0x1000  # never dereferenced: host checks come first


def logprobs_call(dtype=0, T=4, V=100, stride=100, **p):
    return bl.lib().bitlinear_token_logprobs(p.get("logits", FAKE), dtype, T, V, stride, *(p.get(n, FAKE) for n in ("targets", "logprobs", "stats")), None)


def backward_call(dtype=0, T=4, V=100, stride=100, d_stride=100, logits=FAKE, **p):
    return bl.lib().bitlinear_token_logprobs_backward(logits, dtype, T, V, stride, *(p.get(n, 2 * FAKE) for n in ("targets", "stats", "grad", "dlogits")), d_stride, None)


def policy_call(dtype=0, T=4, V=100, stride=100, d_stride=100, low=0.2, high=0.2, kl=0.1, logits=FAKE, **p):
    a = [p.get(n, 2 * FAKE) for n in ("targets", "old", "adv", "weights", "ref")]
    b = [p.get(n, 2 * FAKE) for n in ("loss", "token_loss", "logprobs", "dlogits")]
    return bl.lib().bitlinear_policy_loss(logits, dtype, T, V, stride, *a, low, high, kl, *b, d_stride, None)


def pairs_call(dtype=0, T=4, V=100, stride=100, d_stride=100, pairs=2, beta=0.1, smooth=0.0, ws=FAKE, ws_bytes=1 << 20, logits=FAKE, **p):
    b = [p.get(n, 2 * FAKE) for n in ("loss", "pair_loss", "seq_logprobs", "logprobs", "dlogits")]
    return bl.lib().bitlinear_preference_loss(logits, dtype, T, V, stride, p.get("targets", FAKE), p.get("cu", FAKE), pairs, p.get("ref", FAKE), beta, smooth, *b, d_stride, ws,
                                              ws_bytes, None)


def test_refusals():
    most = 360448
    for call in (logprobs_call, backward_call, policy_call, pairs_call):
        assert call(dtype=2) == 5 and call(dtype=-1) == 5
        for bad in (dict(T=-1), dict(V=0), dict(V=most + 1, stride=most + 1), dict(stride=99), dict(T=(1 << 24) + 1)):
            assert call(**bad) == 2, bad
        assert call(logits=None) == 1 and call(logits=FAKE + 2) == 3 and call(targets=None) == 1
    assert logprobs_call(T=0) == 0 and backward_call(T=0) == 0
    for name in ("logprobs", "stats"):
        assert logprobs_call(**{name: None}) == 1
    assert logprobs_call(stats=FAKE + 4) == 3
    for name in ("stats", "grad", "dlogits"):
        assert backward_call(**{name: None}) == 1
    assert backward_call(d_stride=99) == 2 and backward_call(dlogits=2 * FAKE + 2) == 3 and backward_call(dlogits=FAKE, d_stride=101) == 2
    for name in ("old", "adv", "ref", "loss", "token_loss", "logprobs"):
        assert policy_call(**{name: None}) == 1, name
    for bad in (dict(low=-0.1), dict(high=math.nan), dict(kl=math.inf), dict(d_stride=99), dict(dlogits=FAKE, d_stride=101)):
        assert policy_call(**bad) == 2, bad
    assert policy_call(dlogits=2 * FAKE + 1) == 3
    for name in ("cu", "ref", "loss", "pair_loss", "seq_logprobs", "logprobs"):
        assert pairs_call(**{name: None}) == 1, name
    for bad in (dict(pairs=0), dict(pairs=-3), dict(beta=math.nan), dict(smooth=-0.1), dict(smooth=1.1), dict(d_stride=99), dict(dlogits=FAKE, d_stride=200)):
        assert pairs_call(**bad) == 2, bad
    need = bl.bitlinear_preference_loss_workspace_bytes(4)
    assert need >= 48 and bl.bitlinear_preference_loss_workspace_bytes(0) == 0 and bl.bitlinear_preference_loss_workspace_bytes(-1) == 0
    assert pairs_call(ws=None) == 4 and pairs_call(ws=FAKE + 8) == 4 and pairs_call(ws_bytes=need - 1) == 4


def test_binding_wants_device_tensors():
    x, t, f = torch.zeros(2, 5), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    for call in (lambda: bl.bitlinear_token_logprobs(x, t), lambda: bl.bitlinear_token_logprobs_backward(x, t, torch.zeros(2, 2), f), lambda: bl.bitlinear_policy_loss(x, t, f, f),
                 lambda: bl.bitlinear_preference_loss(x, t, t, f)):
        with pytest.raises(TypeError):
            call()


def test_oracle_pins():
    # two equal logits: log 1/2, gradient (1/2, -1/2); hand-computed losses
    logp, top, total, p, mean = le.row(np.array([1.0, 1.0]), 0)
    assert logp == -math.log(2) and top == 1.0 and total == 2.0 and mean == 0.0
    assert np.allclose(le.gradient(p, 0, logp, 2.0), [1.0, -1.0], rtol=1e-15)
    assert le.row(np.zeros(3), 3) is None and le.row(np.zeros(3), -1) is None
    assert le.policy_token(math.log(1.5), 0.0, 2.0, 0.2, 0.2) == (-2.4, 0.0)      # above the clip with a gain: cut
    assert np.allclose(le.policy_token(math.log(1.5), 0.0, -2.0, 0.2, 0.2), (3.0, 3.0))  # above with a loss: not cut
    assert le.policy_token(math.log(0.5), 0.0, -2.0, 0.2, 0.2) == (1.6, 0.0)
    loss, slope = le.policy_token(0.0, 0.0, 0.0, 0.2, 0.2, 1.0, 1.0)
    assert np.isclose(loss, math.e - 2) and np.isclose(slope, 1 - math.e)
    assert np.allclose(le.pair(2.0, 2.0, 0.5, 0.0, 1), (math.log(2), -0.25))
    # slopes are the derivatives
    h = 1e-5
    for s in (0.0, 0.2):
        up, down = le.pair(1.0 + h, 0.3, 0.7, s, 1)[0], le.pair(1.0 - h, 0.3, 0.7, s, 1)[0]
        assert abs((up - down) / (2 * h) - le.pair(1.0, 0.3, 0.7, s, 1)[1]) < 1e-9


def shared_call(M=4, G=2, n_q=20, n_kv=5, D=128, kind=0, n_blocks=8, rows=64, n_seq=4, max_blocks=4, ws=FAKE, ws_bytes=1 << 40, seq_ids=FAKE, **p):
    a = [p.get(n, FAKE) for n in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "tables", "lengths")]
    return bl.lib().bitlinear_attention_shared_kv8(*a, seq_ids, p.get("starts", FAKE), p.get("shared", FAKE), M, G, n_q, n_kv, D, kind, n_blocks, rows, n_seq, max_blocks,
                                                   p.get("out", FAKE), ws, ws_bytes, None)


def test_shared_attention_refusals():
    assert shared_call(kind=-1) == 5 and shared_call(kind=2) == 5
    for bad in (dict(M=-1), dict(M=65536), dict(G=-1), dict(G=65536), dict(n_q=21), dict(n_q=45), dict(D=96), dict(rows=8), dict(rows=24), dict(n_blocks=0), dict(n_blocks=1 << 26),
                dict(n_seq=0), dict(max_blocks=0), dict(max_blocks=1 << 25), dict(seq_ids=None, M=5), dict(M=65535, max_blocks=1 << 19), dict(M=65535, n_q=40000, n_kv=5000)):
        assert shared_call(**bad) == 2, bad
    assert shared_call(M=0) == 0
    for name in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "tables", "lengths", "starts", "shared", "out"):
        assert shared_call(**{name: None}) == 1, name
    for name in ("q", "k_cache", "v_cache", "out"):
        assert shared_call(**{name: FAKE + 8}) == 3, name
    need = bl.bitlinear_attention_shared_kv8_workspace_bytes(4, 2, 20, 5, 128)
    assert need > 0 and shared_call(ws_bytes=need - 1) == 4 and shared_call(ws=None) == 4 and shared_call(ws=FAKE + 8) == 4
    for bad in ((-1, 2, 20, 5, 128), (4, -1, 20, 5, 128), (4, 2, 20, 6, 128), (4, 2, 45, 5, 128), (4, 2, 20, 5, 96), (65536, 2, 20, 5, 128)):
        assert bl.bitlinear_attention_shared_kv8_workspace_bytes(*bad) == 0, bad


def test_shared_step_wants_no_more_groups_than_places():
    from paper_2504_12285_b200 import chain as gpu_chain

    for groups in (-1, 5):
        with pytest.raises(ValueError):
            gpu_chain.PagedDecodeStep([], torch.zeros(50, 64, dtype=torch.bfloat16), 4, 4, 8, 16, 4, 64, 128, 1, 1, 64, device="cpu", groups=groups)
