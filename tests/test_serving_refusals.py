"""The serving entry points (block tables, 8-bit cache, sampling): what the host refuses before anything is launched, and
the oracle's own pins.  Needs no GPU."""
import numpy as np
import pytest
import torch

from oracle import serving as sv
from paper_2504_12285_b200 import binding as bl

FAKE = 0x1000  # never dereferenced: host checks come first


def tables_call(R=4, max_blocks=8, n_blocks=32, rows=16, t_cap=64, **null):
    names = ["lengths", "new", "tables", "free", "n_free", "lengths_out", "n_free_out", "served", "cu", "seq", "pos", "len", "slots"]
    p = {n: null.get(n, FAKE) for n in names}
    return bl.lib().bitlinear_block_tables(p["lengths"], p["new"], R, p["tables"], max_blocks, p["free"], p["n_free"], n_blocks, rows, t_cap, p["lengths_out"],
                                           p["n_free_out"], p["served"], p["cu"], p["seq"], p["pos"], p["len"], p["slots"], None)


def test_block_tables_refusals():
    assert tables_call(R=-1) == 2 and tables_call(max_blocks=0) == 2 and tables_call(n_blocks=0) == 2 and tables_call(rows=0) == 2 and tables_call(t_cap=-1) == 2
    assert tables_call(max_blocks=1 << 16, rows=1 << 15) == 2 and tables_call(n_blocks=1 << 16, rows=1 << 15) == 2
    assert tables_call(R=1 << 16, max_blocks=1 << 15) == 2
    for name in ("lengths", "new", "tables", "free", "n_free", "lengths_out", "n_free_out", "served", "cu", "seq", "pos", "len", "slots"):
        assert tables_call(**{name: None}) == 1, name
    assert tables_call(slots=FAKE + 4) == 3
    assert tables_call(lengths_out=FAKE + 4) == 2  # overlaps lengths without being lengths


def rope_call(T=4, t_max=64, n_q=20, n_kv=5, D=128, kind=0, n_blocks=8, rows=64, **p):
    a = [p.get(n, FAKE) for n in ("q", "k", "v", "positions", "slots", "table")]
    b = [p.get(n, FAKE) for n in ("q_out", "k_cache", "v_cache", "k_scale", "v_scale")]
    return bl.lib().bitlinear_rope_kv8(*a, T, t_max, n_q, n_kv, D, *b, kind, n_blocks, rows, None)


def test_append_refusals():
    assert rope_call(kind=2) == 5
    for bad in (dict(T=-1), dict(t_max=0), dict(n_q=21), dict(n_q=45), dict(D=96), dict(n_blocks=0), dict(rows=48), dict(rows=8), dict(rows=256),
                dict(n_blocks=1 << 26)):
        assert rope_call(**bad) == 2, bad
    assert rope_call(T=0) == 0
    for name in ("q", "k", "v", "positions", "slots", "table", "q_out", "k_cache", "v_cache", "k_scale", "v_scale"):
        assert rope_call(**{name: None}) == 1, name
    for name in ("q", "k", "v", "table", "q_out", "k_cache", "v_cache"):
        assert rope_call(**{name: FAKE + 4}) == 3, name


def attend_call(M=2, n_q=20, n_kv=5, D=128, kind=0, n_blocks=8, rows=64, n_seq=2, max_blocks=4, ws=FAKE, ws_bytes=1 << 30, seq_ids=FAKE, **p):
    a = [p.get(n, FAKE) for n in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "tables", "lengths")]
    return bl.lib().bitlinear_attention_decode_kv8(*a, seq_ids, M, n_q, n_kv, D, kind, n_blocks, rows, n_seq, max_blocks, p.get("out", FAKE), ws, ws_bytes, None)


def test_attention_refusals():
    assert attend_call(kind=-1) == 5
    for bad in (dict(M=-1), dict(M=65536), dict(n_q=21), dict(n_q=45), dict(D=96), dict(rows=8), dict(rows=24), dict(n_blocks=0), dict(n_blocks=1 << 26), dict(n_seq=0),
                dict(max_blocks=0), dict(max_blocks=1 << 25), dict(seq_ids=None, M=3)):
        assert attend_call(**bad) == 2, bad
    assert attend_call(M=0) == 0
    for name in ("q", "k_cache", "v_cache", "k_scale", "v_scale", "tables", "lengths", "out"):
        assert attend_call(**{name: None}) == 1, name
    for name in ("q", "k_cache", "v_cache", "out"):
        assert attend_call(**{name: FAKE + 8}) == 3, name
    need = bl.bitlinear_attention_kv8_workspace_bytes(20, 5, 128)
    assert need > 0 and attend_call(ws_bytes=need - 1) == 4 and attend_call(ws=None) == 4 and attend_call(ws=FAKE + 8) == 4
    assert bl.bitlinear_attention_kv8_workspace_bytes(20, 6, 128) == 0 and bl.bitlinear_attention_kv8_workspace_bytes(20, 5, 96) == 0


def sample_call(M=2, V=100, stride=100, dtype=0, logits=FAKE, u=FAKE, ids=FAKE):
    return bl.lib().bitlinear_sample(logits, dtype, M, V, stride, u, None, None, None, None, ids, None, None)


def test_sample_refusals():
    assert sample_call(dtype=2) == 5
    for bad in (dict(M=-1), dict(V=0), dict(V=bl.SAMPLE_MAX_VOCAB + 1, stride=1 << 20), dict(stride=99)):
        assert sample_call(**bad) == 2, bad
    assert sample_call(M=0) == 0
    assert sample_call(logits=None) == 1 and sample_call(u=None) == 1 and sample_call(ids=None) == 1
    assert sample_call(logits=FAKE + 2) == 3 and sample_call(dtype=1, logits=FAKE + 1) == 3


def test_binding_refuses_tensors_that_are_not_on_the_device():
    t = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        bl.bitlinear_block_tables(t, t, torch.zeros(4, 2, dtype=torch.int32), t, t[:1], 16, 8)
    with pytest.raises(TypeError):
        bl.bitlinear_sample(torch.zeros(2, 8), torch.zeros(2))
    pool = torch.zeros(2, 1, 16, 64, dtype=torch.int8)
    with pytest.raises(TypeError):
        bl.bitlinear_attention_decode_kv8(torch.zeros(1, 64, dtype=torch.bfloat16), pool, pool, torch.zeros(2, 1), torch.zeros(2, 1), t.view(1, 4), t[:1], 1, 1, 64)


def test_oracle_codes():
    # e4m3: every code is its own nearest, values in the middle go to the even code, beyond the range to 448
    codes = np.array([c for c in range(256) if c & 0x7f != 0x7f], np.uint8)
    assert np.array_equal(sv.encode(sv.decode(codes, sv.E4M3), sv.E4M3), codes)
    assert list(sv.decode(np.array([0x38, 0x7e, 0x01, 0xb8], np.uint8), sv.E4M3)) == [1.0, 448.0, 2.0 ** -9, -1.0]
    assert list(sv.encode(np.array([1.0625, 1.1875, 500.0, -1e9, 2.0 ** -10]), sv.E4M3)) == [0x38, 0x3a, 0x7e, 0xfe, 0x00]
    t = torch.randn(4000, generator=torch.Generator().manual_seed(1)) * 30
    assert np.array_equal(sv.encode(t.numpy().astype(np.float64), sv.E4M3), t.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert list(sv.encode(np.array([0.5, 1.5, -2.5, 300.0]), sv.INT8).view(np.int8)) == [0, 2, -2, 127]
    assert sv.scale_for(448.0, sv.E4M3) == 1.0 and sv.scale_for(449.0, sv.E4M3) == 2.0 and sv.scale_for(224.0, sv.E4M3) == 0.5
    assert sv.scale_for(127.0, sv.INT8) == 1.0


def test_oracle_tables_and_draw_by_hand():
    # two requests of block size 4: the first finished (blocks 5, 6), the second gets 6 tokens on top of 3
    out = sv.block_tables([5, 3], [-1, 6], np.array([[5, 6, -1], [2, -1, -1]], np.int32), np.array([9, 8, 0, 0, 0, 0, 0, 0, 0, 0], np.int32), 2, 4, 8)
    assert out["n_free"] == 2 and list(out["free_blocks"][:4]) == [9, 8, 5, 6]
    assert list(out["tables"][1]) == [2, 6, 5] and list(out["lengths"]) == [0, 9]
    assert list(out["slots"]) == [11, 24, 25, 26, 27, 20, -1, -1] and list(out["row_lengths"]) == [4, 5, 6, 7, 8, 9, 0, 0]
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert sv.sample(l, 0.05)[0] == 0 and sv.sample(l, 0.15)[0] == 1 and sv.sample(l, 0.99)[0] == 3
    assert sv.sample(l, 0.0, top_k=2) == (1, pytest.approx(np.log(4 / 7)))
    assert sv.sample(l, 0.999, top_p=0.6)[0] == 3 and sv.sample(l, 0.999, top_p=0.39)[0] == 1
    assert sv.sample(l, 0.0, min_p=0.7)[0] == 1 and sv.sample(l, 0.3, min_p=0.3)[0] == 1 and sv.sample(l, 0.5, temperature=0.0) == (1, 0.0)
