"""Answers sampled in a group and learned from: a prompt in one place of PagedDecodeStep, several answers that share its cache rows, then the losses on what was drawn."""
import math

import numpy as np
import pytest
import torch

from oracle import learning as le
from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl
from paper_2504_12285_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPE = {sv.INT8: torch.int8, sv.E4M3: torch.float8_e4m3fn}
H, F, N_Q, N_KV, HD, V, ROWS, B = 256, 512, 4, 2, 64, 500, 8, 16


def host(t):
    return (t.view(torch.uint8) if t.dtype in (torch.int8, torch.float8_e4m3fn) else t).cpu().numpy()


def make_step(kind, groups=2, layers=2, places=7, n_blocks=20):
    from paper_2504_12285_b200 import chain as gpu_chain

    made = []
    for li in range(layers):
        layer = {}
        for i, (name, n, k) in enumerate((("q", H, H), ("k", N_KV * HD, H), ("v", N_KV * HD, H), ("o", H, H), ("gate", F, H), ("up", F, H), ("down", H, F))):
            packed, s_w = bl.bitlinear_pack_weights(wl.latent_weights(n, k, 8800 + 10 * li + i).to(DEV), wl.WEIGHT_EPS)
            layer[name] = (packed, s_w, wl.gain_random(k, 8900 + 10 * li + i).to(DEV))
        made.append(layer)
    table = (torch.randn(V, H, generator=torch.Generator().manual_seed(51)) * 0.3).to(torch.bfloat16).to(DEV)
    return gpu_chain.PagedDecodeStep(made, table, ROWS, places, n_blocks, B, 6, H, F, N_Q, N_KV, HD, DTYPE[kind], wl.RMS_EPS, device=DEV, groups=groups)


def check_last_layer(st, kind):
    """The last layer's attention against the oracle on the queries and the cache that the GPU made; tolerance as for the call itself."""
    codes, scales = [host(c) for c in st.cache[-1][:2]], [host(s) for s in st.cache[-1][2:]]
    q, got = st.q_rot.double().cpu().numpy().reshape(ROWS, N_Q, HD), st.attn.double().cpu().numpy().reshape(ROWS, N_Q, HD)
    tables, seq, lengths = host(st.tables), host(st.seq_ids), host(st.row_lengths)
    for m in range(int(st.cu_tokens[-1])):
        n = int(lengths[m])
        t = np.arange(n)
        b, r = tables[seq[m]][t // B], t % B
        assert (b >= 0).all()
        k, v = (sv.decode(c[b, :, r], kind) * s[b].astype(np.float64)[..., None] for c, s in zip(codes, scales))
        for h in range(N_Q):
            g = h // (N_Q // N_KV)
            score = k[:, g] @ q[m, h] / math.sqrt(HD)
            p = np.exp(score - score.max())
            want = (p / p.sum()) @ v[:, g]
            err = ((HD + 4) * 2.0 ** -23 * float((np.abs(k[:, g]) @ np.abs(q[m, h])).max()) + 2.0 ** -23 * np.abs(q[m, h]).max() * float(np.abs(k[:, g]).sum(-1).max())) / math.sqrt(HD)
            tol = (2.0 ** -11 + 2 * err + 1e-6) * np.abs(v[:, g]).max()
            assert (np.abs(got[m, h] - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol)).all(), (m, h)


def bring(st, new, gen, graph=False):
    st.new_tokens.copy_(torch.tensor(new, dtype=torch.int32))
    ids, u = torch.randint(0, V, (ROWS,), generator=gen, dtype=torch.int32).to(DEV), torch.rand(ROWS, generator=gen).to(DEV)
    if graph:
        st.token_buf.copy_(ids)
        st.u_buf.copy_(u)
        out = st.step_graph()
    else:
        out = st.step(ids, u)
    torch.cuda.synchronize()
    assert bl.bitlinear_poll_status() == 0
    return [t.clone() for t in out]


@pytest.mark.parametrize("kind", [sv.INT8, sv.E4M3])
def test_places_share_a_prompt(kind):
    st = make_step(kind, groups=3)
    gen = torch.Generator().manual_seed(61)
    for n in (8, 8, 8, 8, 5):  # a prompt of 37 tokens in place 0, one of 18 in place 4
        bring(st, [n, 0, 0, 0, 0, 0, 0], gen)
    bring(st, [0, 0, 0, 0, 8, 0, 0], gen)
    bring(st, [0, 0, 0, 0, 8, 0, 0], gen)
    bring(st, [0, 0, 0, 0, 2, 0, 0], gen)
    free = int(st.n_free[0])
    assert st.fork(0, 1, 2) == 32 and st.fork(4, 5, 2) == 16
    assert int(st.n_free[0]) == free and st.lengths.tolist() == [37, 32, 32, 0, 18, 16, 16]
    st.group_places.copy_(torch.tensor([0, 3, 4, 7], dtype=torch.int32))  # place 3, between the groups, is a request of its own
    st.shared_rows.copy_(torch.tensor([32, 0, 16], dtype=torch.int32))
    for new in ([1, 3, 1, 0, 1, 1, 1], [1, 1, 1, 1, 1, 1, 1], [0, 2, 1, 1, 1, 0, 3], [1, 1, 1, 0, 1, 1, 1]):
        bring(st, new, gen)
        assert (st.served == 1).all()
        check_last_layer(st, kind)
    tables = st.tables.cpu()
    assert torch.equal(tables[0, :2], tables[1, :2]) and torch.equal(tables[0, :2], tables[2, :2]) and tables[4, 0] == tables[5, 0] == tables[6, 0]
    # answers end and others begin; each gives back what it did not borrow, the prompts' places last
    bring(st, [1, -1, 1, 0, 0, 0, -1], gen)
    assert st.lengths[1] == 0 and st.lengths[6] == 0 and st.borrowed[1] == 0
    assert st.fork(0, 1, 1) == 32
    bring(st, [1, 2, 1, 0, 1, 1, 0], gen)
    check_last_layer(st, kind)
    bring(st, [0, -1, -1, -1, 0, -1, -1], gen)
    bring(st, [-1, 0, 0, 0, -1, 0, 0], gen)
    assert not st.lengths.any() and int(st.n_free[0]) == 20 and sorted(st.free_blocks.tolist()) == list(range(20))


def test_forks_that_are_refused():
    st = make_step(sv.INT8)
    gen = torch.Generator().manual_seed(62)
    bring(st, [5, 0, 0, 0, 3, 0, 0], gen)  # (eight rows in all: more would leave place 4 out)
    for source, first, count in ((0, 0, 2), (7, 1, 1), (0, 6, 2), (0, 1, 0), (-1, 1, 1), (0, 4, 1)):
        with pytest.raises(ValueError):
            st.fork(source, first, count)
    assert st.fork(0, 1, 2) == 0  # no whole block yet
    with pytest.raises(ValueError):
        make_step(sv.INT8, groups=0).fork(0, 1, 1)


def test_shared_steps_recorded():
    kind = sv.E4M3
    eager, recorded = make_step(kind), make_step(kind)
    recorded.capture()
    gens = torch.Generator().manual_seed(63), torch.Generator().manual_seed(63)

    def both(new):
        want, got = bring(eager, new, gens[0]), bring(recorded, new, gens[1], graph=True)
        n = int(eager.cu_tokens[-1])
        assert all(torch.equal(w[:n], g[:n]) for w, g in zip(want, got)) and torch.equal(eager.tables, recorded.tables) and torch.equal(eager.free_blocks, recorded.free_blocks)

    for n in (8, 8, 6):
        both([n, 0, 0, 0, 0, 0, 0])
    for st in (eager, recorded):
        assert st.fork(0, 1, 3) == 16
        st.group_places.copy_(torch.tensor([0, 4, 4], dtype=torch.int32))
        st.shared_rows.copy_(torch.tensor([16, 0], dtype=torch.int32))
    for new in ([1, 1, 1, 1, 2, 0, 0], [1, 2, 1, 1, 1, 0, 0], [0, -1, 1, -1, 1, 0, 0], [-1, 0, -1, 0, -1, 0, 0]):
        both(new)
        check_last_layer(recorded, kind)
    assert int(recorded.n_free[0]) == 20


def test_sampled_answers_are_learned_from():
    """Answers drawn from a shared prompt; the loss on their logits, and the gradient against the oracle's: from the weights' gradient of the head on."""
    st = make_step(sv.INT8)
    gen = torch.Generator().manual_seed(64)
    for n in (8, 8, 4):
        bring(st, [n, 0, 0, 0, 0, 0, 0], gen)
    shared = st.fork(0, 1, 5)
    st.group_places.copy_(torch.tensor([0, 6, 7], dtype=torch.int32))
    st.shared_rows.copy_(torch.tensor([shared, 0], dtype=torch.int32))
    logits, drawn, old, hidden = [], [], [], []
    ids = torch.randint(0, V, (ROWS,), generator=gen, dtype=torch.int32).to(DEV)
    for _ in range(3):
        st.new_tokens.copy_(torch.tensor([0, 1, 1, 1, 1, 1, 0], dtype=torch.int32))
        out, logp = st.step(ids, torch.rand(ROWS, generator=gen).to(DEV))
        logits.append(st.logits[:5].clone())
        drawn.append(out[:5].clone())
        old.append(logp[:5].clone())
        hidden.append(st.h_mid[:5].clone())
        ids = torch.cat([out[:5], ids[5:]])
    logits, drawn, old, hidden = (torch.cat(x) for x in (logits, drawn, old, hidden))
    # the same model gives the same log probabilities (the draw's are good to 2^-31 of the total and rounded; the loss's sums to about 2^-20)
    logp, _ = bl.bitlinear_token_logprobs(logits, drawn)
    assert (logp - old).abs().max() <= 1e-5
    adv = torch.randn(15, generator=gen).to(DEV)
    loss, token_loss, _, d = bl.bitlinear_policy_loss(logits, drawn, old - 0.1, adv, weights=torch.full((15,), 1 / 15, device=DEV), kl_coef=0.1, ref_logprobs=old + 0.05, grad=True)
    total = 0.0
    xs = logits.double().cpu().numpy()
    for t in range(15):
        r = le.row(xs[t], int(drawn[t]))
        value, slope = le.policy_token(r[0], float(old[t]) - 0.1, float(adv[t]), 0.2, 0.2, 0.1, float(old[t]) + 0.05)
        total += value / 15
        # |got - want|: the slope follows old and the log probability, each within 1e-5 of what the oracle takes, and is at most 2 |A| + 1 / 10
        want = le.gradient(r[3], int(drawn[t]), r[0], slope / 15)
        assert np.abs(d[t].double().cpu().numpy() - want).max() <= 1e-5 * (2 * abs(float(adv[t])) + 1)
    assert abs(float(loss) - total) <= 1e-4
    grad_table = d.T @ hidden.float()  # what an optimiser of the tied table takes from here
    assert grad_table.shape == (V, H) and torch.isfinite(grad_table).all() and grad_table.abs().max() > 0
    # the answers as pairs, of three rows each: the first preferred to the second, the third to the fourth
    order = torch.arange(15, device=DEV).view(3, 5).T.reshape(-1)[:12]
    ref = torch.tensor([float(old[order[3 * i: 3 * i + 3]].sum()) for i in range(4)], device=DEV)
    out = bl.bitlinear_preference_loss(logits[order], drawn[order], torch.arange(0, 13, 3, dtype=torch.int32, device=DEV), ref, beta=0.5, grad=True)
    assert abs(float(out[0]) - math.log(2)) <= 1e-4  # the reference is the model itself
    for t in range(12):
        r = le.row(xs[int(order[t])], int(drawn[order[t]]))
        want = le.gradient(r[3], int(drawn[order[t]]), r[0], (-1 if (t // 3) % 2 == 0 else 1) * 0.5 / 2 / 2)
        assert np.abs(out[4][t].double().cpu().numpy() - want).max() <= 1e-4


def test_group_places_outside_the_places():
    # they count as the nearest place there is: one group of all places, one of none
    st = make_step(sv.INT8)
    gen = torch.Generator().manual_seed(64)
    st.group_places.copy_(torch.tensor([-5, 99, 2 ** 31 - 1], dtype=torch.int32))
    for new in ([3, 2, 0, 1, 0, 1, 1], [1, 1, 2, 1, 1, 1, 1]):
        bring(st, new, gen)
        check_last_layer(st, sv.INT8)
