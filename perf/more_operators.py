"""Operators around answers that are sampled in groups and learned from, as cases that can be timed: attention of many rows over cache rows
that they share, log probabilities of given tokens with their gradient, a clipped policy loss with a KL term, and a loss over pairs of a
preferred and a rejected answer, both with the gradient of the logits.

`run` computes each of them in plain torch operations, or, with `own` set, through the library's entry points.  Shapes: 20 query / 5 KV heads
of 128 and a vocabulary of 128,256 are this library's 2B configuration; the others are generic.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
Q_MAX = {"int8": 127.0, "e4m3": 448.0}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    b2 = {"heads": 20, "kv_heads": 5, "dim": 128}
    return [
        # four answers to a short question, some tokens in: the latency of a small group's step
        {"name": "share_few", "op": "share", "kind": "int8", **b2, "block": 64, "groups": 1, "rows_from": 4, "rows_to": 4, "shared_from": 300, "shared_to": 300, "own_from": 1, "own_to": 40},
        # sixteen answers to one prompt of 4096 tokens
        {"name": "share_group", "op": "share", "kind": "int8", **b2, "block": 64, "groups": 1, "rows_from": 16, "rows_to": 16, "shared_from": 4096, "shared_to": 4096, "own_from": 50, "own_to": 600},
        # a busy server: groups of 5 to 48 answers with prompts of their own, small heads and blocks
        {"name": "share_ragged", "op": "share", "kind": "e4m3", "heads": 32, "kv_heads": 4, "dim": 64, "block": 16, "groups": 6, "rows_from": 5, "rows_to": 48,
         "shared_from": 1000, "shared_to": 9000, "own_from": 1, "own_to": 1200},
        # 64 answers about a long document
        {"name": "share_long", "op": "share", "kind": "int8", **b2, "block": 32, "groups": 1, "rows_from": 64, "rows_to": 64, "shared_from": 32768, "shared_to": 32768, "own_from": 200, "own_to": 1000},
        # chunks of two prompts, each token seeing those in front of it: the rows of a chunk share all of the cache but their own triangle
        {"name": "share_chunk", "op": "chunk", "kind": "e4m3", **b2, "block": 64, "groups": 2, "tokens_from": 900, "tokens_to": 1100, "context_from": 3000, "context_to": 6000},
        # what the model thinks of a handful of tokens
        {"name": "logp_few", "op": "logp", "type": "f32", "tokens": 7, "vocab": 128256, "grad": False},
        # a reference model's log probabilities of an answer
        {"name": "logp_answers", "op": "logp", "type": "bf16", "tokens": 1200, "vocab": 128256, "grad": False},
        # the gradient of a loss that is not among those below; a vocabulary whose rows start anywhere
        {"name": "logp_grad", "op": "logp", "type": "f32", "tokens": 700, "vocab": 50281, "grad": True},
        # a few sampled tokens
        {"name": "policy_few", "op": "policy", "type": "f32", "tokens": 21, "vocab": 128256, "kl": 0.05},
        # a minibatch of sampled answers
        {"name": "policy_batch", "op": "policy", "type": "bf16", "tokens": 3000, "vocab": 128256, "kl": 0.05},
        # one pair of short answers, a small odd vocabulary
        {"name": "pairs_one", "op": "pairs", "type": "f32", "pairs": 1, "tokens_from": 5, "tokens_to": 20, "vocab": 32003},
        # six pairs with their prompts' tokens among the rows
        {"name": "pairs_batch", "op": "pairs", "type": "bf16", "pairs": 6, "tokens_from": 60, "tokens_to": 250, "vocab": 128256},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["share", "share", "chunk", "logp", "policy", "pairs"])
    if op in ("share", "chunk"):
        heads, kv_heads = rng.choice([(20, 5), (16, 4), (32, 4), (8, 8), (28, 4), (6, 2)])
        c = {"op": op, "kind": rng.choice(["int8", "e4m3"]), "heads": heads, "kv_heads": kv_heads, "dim": rng.choice([64, 128]), "block": rng.choice([16, 32, 64, 128])}
        if op == "chunk":
            groups, most = rng.randint(1, 4), 4000000 * 20 // heads
            tokens = _log(rng, 1, 2000 // groups)
            context = _log(rng, 1, min(20000, max(1, most // (tokens * groups))))
            return {**c, "groups": groups, "tokens_from": max(1, tokens // 2), "tokens_to": tokens, "context_from": context // 2, "context_to": context}
        groups = _log(rng, 1, 12)
        rows = _log(rng, 1, max(1, 160 // groups))
        own_rows = _log(rng, 1, max(1, min(2000, 60000 // (rows * groups))))
        shared = _log(rng, 16, min(32768, 160000 // groups))
        return {**c, "groups": groups, "rows_from": max(1, rows // 3), "rows_to": rows, "shared_from": shared // 3, "shared_to": shared, "own_from": rng.randint(0, own_rows),
                "own_to": own_rows}
    vocab = rng.choice([_log(rng, 100, 160000), 8 * _log(rng, 16, 16000), 128256])
    c = {"op": op, "type": rng.choice(["f32", "bf16"]), "vocab": vocab}
    most = min(4000, max(2, 190000000 // vocab))
    if op == "pairs":
        pairs = _log(rng, 1, 12)
        tokens = _log(rng, 1, max(1, most // (4 * pairs)))
        return {**c, "pairs": pairs, "tokens_from": max(1, tokens // 4), "tokens_to": tokens}
    if op == "logp":
        return {**c, "tokens": _log(rng, 1, most), "grad": rng.random() < 0.5}
    return {**c, "tokens": _log(rng, 1, most), "kl": rng.choice([0.0, 0.02, 0.3])}


# ------------------------------------------------------------------------------------------------------ inputs

def _to(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _spread(rng, lo, hi, n):
    """n lengths between lo and hi, many short and few long ones."""
    return np.rint(np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1), n)) - 1).astype(np.int64).clip(lo, hi)


def _rows(c):
    """The rows of an attention case: [(rows of the group, cache rows they share, lengths)].  These go by the case alone."""
    if c["op"] == "chunk":
        tokens, context = (c["tokens_from"], c["tokens_to"]), (c["context_from"], c["context_to"])
        rng = np.random.default_rng([c["groups"], *tokens, *context])
        out = []
        for g in range(c["groups"]):
            n = tokens[1] if g == 0 else int(rng.integers(tokens[0], tokens[1] + 1))
            start = int(rng.integers(context[0], context[1] + 1))
            out.append((n, start + n, start + 1 + np.arange(n)))
        return out
    rows, prompts, own_rows = (c["rows_from"], c["rows_to"]), (c["shared_from"], c["shared_to"]), (c["own_from"], c["own_to"])
    rng = np.random.default_rng([c["groups"], *rows, *prompts, *own_rows, c["block"]])
    out = []
    for g in range(c["groups"]):
        n = rows[1] if g == 0 else int(rng.integers(rows[0], rows[1] + 1))
        prompt = prompts[1] if g == 0 else int(rng.integers(prompts[0], prompts[1] + 1))
        shared = prompt // c["block"] * c["block"]  # whole blocks are shared, the prompt's rest stands with each answer
        out.append((n, shared, prompt + _spread(rng, *own_rows, n)))
    return out


def _codes(shape, kind, gen):
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
    if kind == "int8":
        return (x * 38.0).round_().clamp_(-127, 127).to(torch.int8)
    return (x * 110.0).clamp_(-448, 448).to(torch.float8_e4m3fn)


def _scales(shape, kind, size, gen):
    s = (torch.rand(shape, generator=gen, device=DEV, dtype=torch.float32) * 0.8 + 0.4) * (size / Q_MAX[kind])
    return s if kind == "int8" else torch.exp2(torch.ceil(torch.log2(s)))


def _prepare_attend(c, seed):
    rng, gen = np.random.default_rng([seed, 1]), _generator(seed)
    B, groups = c["block"], _rows(c)
    M = sum(n for n, _, _ in groups)
    lengths = np.concatenate([x for _, _, x in groups])
    # which blocks each sequence has: one sequence to a group's chunk, one to each answer
    need, share = [], []
    for n, shared, x in groups:
        for r in range(1 if c["op"] == "chunk" else n):
            need.append(-(-int(x[-1] if c["op"] == "chunk" else x[r]) // B))
            share.append(shared // B if c["op"] == "share" and r > 0 else 0)
    n_blocks = sum(a - b for a, b in zip(need, share)) + 3
    ids = rng.permutation(n_blocks).astype(np.int32)
    tables = np.full((len(need), max(1, max(need))), -1, np.int32)
    at, seq = 0, []
    for s, (a, b) in enumerate(zip(need, share)):
        if b:
            tables[s, :b] = tables[first, :b]
        else:
            first = s
        tables[s, b:a] = ids[at: at + a - b]
        at += a - b
    for g, (n, _, _) in enumerate(groups):
        seq += [g] * n if c["op"] == "chunk" else []
    pair = (n_blocks, c["kv_heads"], B, c["dim"])
    starts = np.cumsum([0] + [n for n, _, _ in groups])
    return {"q": (torch.randn((M, c["heads"] * c["dim"]), generator=gen, device=DEV) * 2.0).to(torch.bfloat16), "lengths": _to(lengths.astype(np.int32)), "tables": _to(tables),
            "seq_ids": _to(np.array(seq, np.int32)) if c["op"] == "chunk" else None, "group_starts": _to(starts.astype(np.int32)),
            "shared_rows": _to(np.array([s for _, s, _ in groups], np.int32)), "k_cache": _codes(pair, c["kind"], gen), "v_cache": _codes(pair, c["kind"], gen),
            "k_scale": _scales(pair[:2], c["kind"], 2.5, gen), "v_scale": _scales(pair[:2], c["kind"], 2.5, gen)}


def _prepare_logits(T, V, kind, gen):
    """Logits and the tokens that were drawn from them: tokens are mostly likely ones."""
    x = torch.randn((T, V), generator=gen, device=DEV, dtype=torch.float32).mul_(2.0)
    targets = torch.randint(0, V, (T,), generator=gen, device=DEV)
    x[torch.arange(T, device=DEV), targets] += torch.rand(T, generator=gen, device=DEV) * 14.0
    x = x.to(TYPE[kind])
    logp = torch.empty(T, device=DEV)
    for t in range(0, T, 256):  # what another pass of about the same model gave these tokens
        y = x[t: t + 256].float()
        y = y - y.amax(-1, keepdim=True)
        logp[t: t + 256] = y.gather(1, targets[t: t + 256, None])[:, 0] - y.exp_().sum(-1).log()
    return x, targets.int(), logp


def _answers(c):
    """Rows of each sequence of a case of pairs: by the case alone."""
    rng = np.random.default_rng([c["pairs"], c["tokens_from"], c["tokens_to"]])
    return rng.integers(c["tokens_from"], c["tokens_to"] + 1, 2 * c["pairs"])


def prepare(case, seed):
    c = case
    if c["op"] in ("share", "chunk"):
        return {"case": c, **_prepare_attend(c, seed)}
    gen = _generator(seed)
    sizes = _answers(c) if c["op"] == "pairs" else None
    T = int(sizes.sum()) if c["op"] == "pairs" else c["tokens"]
    logits, targets, logp = _prepare_logits(T, c["vocab"], c["type"], gen)
    s = {"case": c, "logits": logits, "targets": targets}
    noise = lambda size: torch.randn(T, generator=gen, device=DEV) * size  # noqa: E731
    if c["op"] == "logp":
        s["grad"] = noise(1.0)
    elif c["op"] == "policy":
        s["old"], s["ref"] = logp + noise(0.25), logp + noise(0.3)
        s["advantages"] = noise(1.0)
        s["weights"] = torch.full((T,), 1.0 / T, device=DEV)
    else:
        cu = np.concatenate([[0], np.cumsum(sizes)])
        for a, b in zip(cu[:-1], cu[1:]):  # a prompt's last tokens stand in front of an answer: they count for nothing
            targets[a: a + (b - a) // 5] = -1
        live = torch.where(targets >= 0, logp + noise(0.2), 0.0)
        s["cu_tokens"] = _to(cu.astype(np.int32))
        s["ref"] = torch.stack([live[a:b].sum() for a, b in zip(cu[:-1], cu[1:])])
    return s


# ------------------------------------------------------------------------------------------------------ plain forms

def _values(cache, scale):
    return (cache.float() if cache.dtype != torch.int8 else cache) * scale[..., None, None]


def _pick(cache, scale, blocks):
    """Rows of these blocks [..., n] -> [..., H, n * B, D]."""
    x = _values(cache.view(torch.uint8)[blocks].view(cache.dtype), scale[blocks])  # [..., n, H, B, D]
    return x.transpose(-4, -3).flatten(-3, -2)


def _plain_attend(s):
    c = s["case"]
    H, D, B = c["kv_heads"], c["dim"], c["block"]
    G = c["heads"] // H
    out, m0 = torch.empty_like(s["q"]), 0
    for g, (n, shared, _) in enumerate(_rows(c)):
        rows = slice(m0, m0 + n)
        q = s["q"][rows].float().view(n, H, G, D) / math.sqrt(D)
        seq = s["seq_ids"][rows].long() if s["seq_ids"] is not None else torch.arange(m0, m0 + n, device=DEV)
        length = s["lengths"][rows]
        tables = s["tables"][seq].clamp(min=0).long()
        nb = -(-shared // B)
        k = _pick(s["k_cache"], s["k_scale"], tables[0, :nb])[:, :shared]  # [H, shared, D]
        v = _pick(s["v_cache"], s["v_scale"], tables[0, :nb])[:, :shared]
        at = torch.arange(shared, device=DEV)
        score = (q.permute(1, 0, 2, 3).reshape(H, n * G, D) @ k.transpose(1, 2)).view(H, n, G, shared)
        score = torch.where((at < length[:, None])[None, :, None], score, -math.inf).permute(1, 0, 2, 3)
        parts = [score]
        if c["op"] == "share":
            k2, v2 = (_pick(x, y, tables[:, nb:]) for x, y in ((s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"])))  # [n, H, rows, D]
            live = torch.arange(nb * B, nb * B + k2.shape[2], device=DEV) < length[:, None]
            parts.append(torch.where(live[:, None, None], q @ k2.transpose(2, 3), -math.inf))
            v2 = torch.where(live[:, None, :, None], v2, 0.0)
        score = torch.cat(parts, -1)
        if score.shape[-1]:
            p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
            o = (p[..., :shared].permute(1, 0, 2, 3).reshape(H, n * G, shared) @ v).view(H, n, G, D).permute(1, 0, 2, 3)
            if c["op"] == "share":
                o = o + p[..., shared:] @ v2
            o = o / p.sum(-1, keepdim=True)
            o = torch.where((length > 0)[:, None, None, None], o, 0.0)
        else:
            o = torch.zeros_like(q)
        out[rows] = o.reshape(n, -1).to(torch.bfloat16)
        m0 += n
    return out


def _plain_logp(logits, targets):
    """(log probabilities, 0 for a target outside the vocabulary; probabilities; which rows count)"""
    x = logits.float()
    live = (targets >= 0) & (targets < x.shape[1])
    x = x - x.amax(-1, keepdim=True)
    at = torch.where(live, targets, 0).long()[:, None]
    chosen = x.gather(1, at)[:, 0]
    p = x.exp_()
    total = p.sum(-1, keepdim=True)
    return torch.where(live, chosen - total.log()[:, 0], 0.0), p.div_(total), live, at


def _plain_dlogits(p, live, at, grad, dtype):
    grad = torch.where(live, grad, 0.0)[:, None]
    d = p.mul_(-grad)
    return d.scatter_add_(1, at, grad).to(dtype)


def _plain_policy(s):
    logp, p, live, at = _plain_logp(s["logits"], s["targets"])
    ratio = torch.exp(logp - s["old"])
    A, kl = s["advantages"], s["case"]["kl"]
    free, cut = ratio * A, ratio.clamp(0.8, 1.28) * A
    loss = -torch.minimum(free, cut)
    grad = torch.where(free <= cut, -free, 0.0)
    if kl:
        d = s["ref"] - logp
        e = torch.expm1(d)
        loss = loss + kl * (e - d)
        grad = grad - kl * e
    loss = torch.where(live, loss * s["weights"], 0.0)
    return {"loss": loss.sum()[None], "token_loss": loss, "logprobs": logp, "dlogits": _plain_dlogits(p, live, at, grad * s["weights"], s["logits"].dtype)}


BETA, SMOOTH = 0.1, 0.05


def _plain_pairs(s):
    logp, p, live, at = _plain_logp(s["logits"], s["targets"])
    P = s["case"]["pairs"]
    seq = torch.repeat_interleave(torch.arange(2 * P, device=DEV), torch.diff(s["cu_tokens"]), output_size=len(logp))
    sums = torch.zeros(2 * P, device=DEV, dtype=torch.float64).index_add_(0, seq, logp.double())
    d = (sums - s["ref"].double()).view(P, 2)
    delta = BETA * (d[:, 0] - d[:, 1])
    log_sigma = lambda x: -torch.log1p(torch.exp(-x.abs())) + x.clamp(max=0.0)  # noqa: E731
    loss = -(1 - SMOOTH) * log_sigma(delta) - SMOOTH * log_sigma(-delta)
    slope = (-BETA / P) * (1 / (1 + torch.exp(delta)) - SMOOTH)
    grad = torch.stack([slope, -slope], 1).view(-1)[seq].float()
    return {"loss": loss.mean()[None].float(), "pair_loss": loss.float(), "seq_logprobs": sums.float(), "logprobs": logp,
            "dlogits": _plain_dlogits(p, live, at, grad, s["logits"].dtype)}


def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2504_12285_b200 import binding as bl
    if op in ("share", "chunk"):
        if not own:
            return _plain_attend(s)
        return bl.bitlinear_attention_shared_kv8(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["tables"], s["lengths"], s["group_starts"],
                                                 s["shared_rows"], c["heads"], c["kv_heads"], c["dim"], seq_ids=s["seq_ids"])
    if op == "logp":
        if own:
            logp, stats = bl.bitlinear_token_logprobs(s["logits"], s["targets"])
            return {"logprobs": logp, "dlogits": bl.bitlinear_token_logprobs_backward(s["logits"], s["targets"], stats, s["grad"])} if c["grad"] else logp
        logp, p, live, at = _plain_logp(s["logits"], s["targets"])
        return {"logprobs": logp, "dlogits": _plain_dlogits(p, live, at, s["grad"], s["logits"].dtype)} if c["grad"] else logp
    if op == "policy":
        if not own:
            return _plain_policy(s)
        ref = s["ref"] if c["kl"] else None
        loss, token_loss, logp, dlogits = bl.bitlinear_policy_loss(s["logits"], s["targets"], s["old"], s["advantages"], weights=s["weights"], clip_low=0.2, clip_high=0.28,
                                                                   kl_coef=c["kl"], ref_logprobs=ref, grad=True)
        return {"loss": loss, "token_loss": token_loss, "logprobs": logp, "dlogits": dlogits}
    if not own:
        return _plain_pairs(s)
    loss, pair_loss, seq_logp, logp, dlogits = bl.bitlinear_preference_loss(s["logits"], s["targets"], s["cu_tokens"], s["ref"], beta=BETA, label_smoothing=SMOOTH, grad=True)
    return {"loss": loss, "pair_loss": pair_loss, "seq_logprobs": seq_logp, "logprobs": logp, "dlogits": dlogits}


# ------------------------------------------------------------------------------------------------------ what a pass needs

def work(case):
    c = case
    if c["op"] in ("share", "chunk"):
        kv, q = c["kv_heads"] * c["dim"], c["heads"] * c["dim"]
        rows = pairs = M = 0.0  # cache rows that have to be read, and (row, cache row) pairs
        for n, shared, lengths in _rows(c):
            M += n
            rows += shared + np.maximum(lengths - shared, 0).sum()
            pairs += lengths.sum()
        return {"bytes": float(rows * (2.0 * kv + 8.0 * c["kv_heads"] / c["block"]) + 4.0 * M * q), "flops": float(4.0 * pairs * q)}
    T = int(_answers(c).sum()) if c["op"] == "pairs" else c["tokens"]
    size = {"f32": 4.0, "bf16": 2.0}[c["type"]]
    grad = c["op"] != "logp" or c["grad"]
    return {"bytes": T * c["vocab"] * size * (2.0 if grad else 1.0) + 24.0 * T, "flops": T * c["vocab"] * (6.0 if grad else 4.0)}


# ------------------------------------------------------------------------------------------------------ from the definitions, in 64 bits

def _code_values(kind):
    code = np.arange(256)
    if kind == "int8":
        return code.astype(np.uint8).view(np.int8).astype(np.float64)
    e, f = (code >> 3) & 15, code & 7
    x = np.where(e > 0, (8 + f) * 2.0 ** (e - 10.0), f * 2.0 ** -9)
    x[(code & 127) == 127] = np.nan
    return np.where(code < 128, x, -x)


def _exact_attend(s):
    c = s["case"]
    H, D = c["kv_heads"], c["dim"]
    value = torch.from_numpy(_code_values(c["kind"])).to(DEV)
    codes = [s[n].view(torch.uint8) for n in ("k_cache", "v_cache")]
    scales = [s[n].double() for n in ("k_scale", "v_scale")]
    M = s["q"].shape[0]
    out = torch.zeros((M, H, c["heads"] // H, D), dtype=torch.float64, device=DEV)
    lengths = s["lengths"].tolist()
    seq = s["seq_ids"].tolist() if s["seq_ids"] is not None else list(range(M))
    for sequence in sorted(set(seq)):  # each on its own, whatever rows they share
        mine = [m for m in range(M) if seq[m] == sequence]
        n = max(lengths[m] for m in mine)
        if n == 0:
            continue
        at = torch.arange(n, device=DEV)
        block, off = s["tables"][sequence].long()[at // c["block"]], at % c["block"]
        for h in range(H):
            k, v = (value[x[block, h, off].long()] * y[block, h][:, None] for x, y in zip(codes, scales))
            for i in range(0, len(mine), 256):
                rows = torch.tensor(mine[i: i + 256], device=DEV)
                live = at < torch.tensor([lengths[m] for m in mine[i: i + 256]], device=DEV)[:, None]
                a = torch.einsum("rgd,nd->rgn", s["q"][rows].double().view(len(rows), H, -1, D)[:, h], k) / D ** 0.5
                a = torch.softmax(a.masked_fill(~live[:, None], -math.inf), -1).nan_to_num(0.0)
                out[rows, h] = a @ v
    return out.view(M, -1).cpu().numpy()


def _exact_rows(s, slope):
    """Log probabilities and, for the slopes that `slope` makes of them, the logits' gradient."""
    T, V = s["logits"].shape
    targets = s["targets"].cpu().numpy()
    live = (targets >= 0) & (targets < V)
    logp, lse = np.zeros(T), torch.empty(T, dtype=torch.float64, device=DEV)
    for t in range(0, T, 128):
        x = s["logits"][t: t + 128].double()
        lse[t: t + 128] = torch.logsumexp(x, -1)
        there = np.nonzero(live[t: t + 128])[0]
        logp[t + there] = (x[_to(there), _to(targets[t + there].astype(np.int64))] - lse[t + _to(there)]).cpu().numpy()
    out = slope(logp, live)
    if out is None:
        return logp, None
    d = np.zeros((T, V))
    for t in range(0, T, 128):
        w = _to(np.where(live, out, 0.0)[t: t + 128])[:, None]
        part = (-w * torch.exp(s["logits"][t: t + 128].double() - lse[t: t + 128, None])).cpu().numpy()
        for i in np.nonzero(live[t: t + 128])[0]:
            part[i, targets[t + i]] = out[t + i] * -math.expm1(logp[t + i])
        d[t: t + 128] = part
    return logp, d


def _exact_policy(s):
    old, ref, A, w = (s[n].double().cpu().numpy() for n in ("old", "ref", "advantages", "weights"))
    kl, losses = s["case"]["kl"], []

    def slope(logp, live):
        r = np.exp(logp - old)
        bound = np.where(A >= 0, np.minimum(r, 1.28), np.maximum(r, 0.8))
        drift = np.exp(ref - logp)
        losses.append(np.where(live, w * (-bound * A + kl * (drift - 1 - (ref - logp))), 0.0))
        return w * (np.where(bound == r, -r * A, 0.0) + kl * (1 - drift))

    logp, d = _exact_rows(s, slope)
    return {"loss": np.array([math.fsum(losses[0])]), "token_loss": losses[0], "logprobs": logp, "dlogits": d}


def _exact_pairs(s):
    cu, ref, P = s["cu_tokens"].cpu().numpy(), s["ref"].double().cpu().numpy(), s["case"]["pairs"]
    sums, losses = np.zeros(2 * P), np.zeros(P)

    def slope(logp, live):
        out = np.zeros(len(logp))
        for i in range(2 * P):
            sums[i] = math.fsum(logp[cu[i]: cu[i + 1]][live[cu[i]: cu[i + 1]]])
        for i in range(P):
            delta = BETA * ((sums[2 * i] - ref[2 * i]) - (sums[2 * i + 1] - ref[2 * i + 1]))
            losses[i] = (1 - SMOOTH) * np.logaddexp(0, -delta) + SMOOTH * np.logaddexp(0, delta)
            g = -BETA / P * ((1 - SMOOTH) / (1 + math.exp(delta)) - SMOOTH / (1 + math.exp(-delta)))
            out[cu[2 * i]: cu[2 * i + 1]], out[cu[2 * i + 1]: cu[2 * i + 2]] = g, -g
        return out

    logp, d = _exact_rows(s, slope)
    return {"loss": np.array([losses.mean()]), "pair_loss": losses, "seq_logprobs": sums, "logprobs": logp, "dlogits": d}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("share", "chunk"):
        return _exact_attend(s)
    if case["op"] == "policy":
        return _exact_policy(s)
    if case["op"] == "pairs":
        return _exact_pairs(s)
    logp, d = _exact_rows(s, lambda logp, live: s["grad"].double().cpu().numpy() if case["grad"] else None)
    return {"logprobs": logp, "dlogits": d} if case["grad"] else logp
