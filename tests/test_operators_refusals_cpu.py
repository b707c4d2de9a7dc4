"""What the operators on tokens refuse on the host, before anything is enqueued, and what their workspaces take (no GPU).  FAKE addresses are never followed."""
import ctypes
import struct

import pytest

from paper_2411_17887_amd import tcuscan

FAKE = 1 << 20
OK, INVALID, UNSUPPORTED, WORKSPACE = tcuscan.OK, tcuscan.ERR_INVALID_ARG, tcuscan.ERR_UNSUPPORTED, tcuscan.ERR_WORKSPACE
BIG = 1 << 40


def shape(rows=2, total=100, heads=4, dk=64, dv=64, q=4, k=4, v=4):
    return struct.pack("22q", rows, total, heads, dk, dv, q, k, v, q * dk, dk, k * dk, dk, v * dv, dv, heads * dv, dv, q * dk, dk, k * dk, dk, v * dv, dv)


def forward(s=None, q=FAKE, k=FAKE * 2, v=FAKE * 3, o=FAKE * 4, decay=FAKE * 5, offsets=FAKE * 6, dt=tcuscan.BF16_F32, state_in=0, state_out=0, slots=0, states=0, ws=FAKE * 7, ws_bytes=BIG):
    return tcuscan.load().tcuscan_decay_attention(shape() if s is None else s, q, k, v, o, decay, offsets, dt, 1.0, state_in, state_out, slots, states, ws, ws_bytes, 0)


def backward(s=None, outs=(FAKE * 5, FAKE * 6, FAKE * 7), ins=(FAKE, FAKE * 2, FAKE * 3, FAKE * 4), decay=FAKE * 8, offsets=FAKE * 9, dt=tcuscan.F32_F32, states=(0, 0, 0), ws=FAKE * 10, ws_bytes=BIG):
    return tcuscan.load().tcuscan_decay_attention_backward(shape() if s is None else s, *ins, *outs, decay, offsets, dt, 1.0, *states, ws, ws_bytes, 0)


def step(s=None, q=FAKE, o=FAKE * 4, state=FAKE * 6, slots=0, states=2, dt=tcuscan.F16_F32, ws=0, ws_bytes=0):
    return tcuscan.load().tcuscan_decay_attention_step(shape(2, 2) if s is None else s, q, FAKE * 2, FAKE * 3, o, FAKE * 5, dt, 1.0, state, slots, states, ws, ws_bytes, 0)


def test_attention_shapes_that_no_call_takes():
    for call in (forward, backward, lambda s: step(s)):
        for bad in (dict(heads=0), dict(dk=0), dict(dv=-1), dict(q=3), dict(k=0), dict(v=8), dict(rows=-1), dict(total=-5)):
            assert call(shape(**{**(dict(rows=2, total=2) if call not in (forward, backward) else {}), **bad})) == INVALID, bad
        for bad in (dict(dk=257), dict(dv=300), dict(total=1 << 40), dict(rows=1 << 30), dict(heads=1 << 17, q=1, k=1, v=1)):
            assert call(shape(**bad)) == UNSUPPORTED, bad
    for dt in (tcuscan.I32_I32, tcuscan.I8_I32, 7, -1):
        assert forward(dt=dt) == UNSUPPORTED and backward(dt=dt) == UNSUPPORTED and step(dt=dt) == UNSUPPORTED
    assert tcuscan.load().tcuscan_decay_attention(None, *[FAKE] * 6, tcuscan.F32_F32, 1.0, 0, 0, 0, 0, FAKE, BIG, 0) == INVALID


def test_attention_pointers_that_no_call_takes():
    for name in ("q", "k", "v", "o", "decay", "offsets"):
        assert forward(**{name: 0}) == INVALID, name
    for name, by in (("q", 1), ("k", 1), ("v", 1), ("o", 1), ("decay", 2), ("offsets", 4), ("state_in", 8), ("state_out", 4), ("slots", 4)):
        assert forward(**{name: FAKE * 20 + by, "states": 2}) == INVALID, name
    assert forward(o=FAKE) == INVALID and forward(o=FAKE * 3) == INVALID                          # in place
    assert forward(state_in=FAKE * 30, states=1) == INVALID                                       # fewer states than rows
    assert forward(ws=0) == WORKSPACE and forward(ws=FAKE + 8) == WORKSPACE
    need = tcuscan.decay_attention_workspace_bytes(2, 100, 4, 64, 64)
    assert need >= 256 and forward(ws_bytes=need - 1) == WORKSPACE
    assert forward(shape(rows=0), q=0, k=0, v=0, o=0, decay=0, offsets=0, ws=0) == OK             # nothing to do
    assert forward(shape(total=0), q=0, k=0, v=0, o=0, ws=0) == OK
    for i in range(4):
        ins = [FAKE, FAKE * 2, FAKE * 3, FAKE * 4]
        ins[i] = 0
        assert backward(ins=ins) == INVALID
    assert backward(outs=(FAKE * 5, FAKE * 5, FAKE * 7)) == INVALID and backward(outs=(FAKE, FAKE * 6, FAKE * 7)) == INVALID
    assert backward(outs=(FAKE * 5, 0, FAKE * 7)) == INVALID and backward(outs=(FAKE * 5 + 2, FAKE * 6, FAKE * 7)) == INVALID
    assert backward(states=(FAKE * 20, FAKE * 21, FAKE * 20)) == INVALID and backward(states=(0, FAKE * 21 + 4, 0)) == INVALID
    assert backward(ws_bytes=100) == WORKSPACE
    assert step(shape(2, 3)) == INVALID and step(q=0) == INVALID and step(state=0) == INVALID and step(state=FAKE + 4) == INVALID
    assert step(o=FAKE) == INVALID and step(states=1) == INVALID and step(ws=FAKE, ws_bytes=255) == WORKSPACE
    assert step(shape(0, 0), q=0, o=0, state=0) == OK


def test_attention_workspaces_grow_with_what_a_call_keeps():
    size = tcuscan.decay_attention_workspace_bytes
    assert size(1, 0, 1, 1, 1) == 256 and size(3, 512, 4, 64, 64) == 256                          # short calls are not cut
    cut = size(1, 4096, 4, 64, 64)
    assert cut >= 256 + 4 * 64 * 64 * 4 * 2 and size(1, 8192, 4, 64, 64) >= cut
    assert size(1, 4096, 4, 64, 64, backward=True) >= 2 * (cut - 256)
    assert size(3, 100, 8, 64, 32, backward=True) == 256
    assert size(3, 100, 8, 64, 32, 8, 2, 8, backward=True) == 256 + 100 * 8 * 64 * 4              # keys shared: a part for each head
    assert size(3, 100, 8, 64, 32, 8, 8, 2, backward=True) == 256 + 100 * 8 * 32 * 4
    assert size(3, 100, 8, 300, 32) == 0 and size(3, 100, 8, 64, 32, 3) == 0


def lookup(ids=FAKE, id_bytes=8, n=10, w=FAKE * 2, vocab=100, dim=16, ws_=16, w_dt=tcuscan.F32_F32, o=FAKE * 3, os_=16, o_dt=tcuscan.BF16_F32, ws=0, ws_bytes=0):
    return tcuscan.load().tcuscan_embedding(ids, id_bytes, n, w, vocab, dim, ws_, w_dt, o, os_, o_dt, 1.0, ws, ws_bytes, 0)


def gradient(ids=FAKE, id_bytes=8, n=10, g=FAKE * 2, gs=16, g_dt=tcuscan.BF16_F32, w=FAKE * 3, vocab=100, dim=16, ws_=16, w_dt=tcuscan.F32_F32, flags=0, ws=FAKE * 4, ws_bytes=BIG):
    return tcuscan.load().tcuscan_embedding_backward(ids, id_bytes, n, g, gs, g_dt, w, vocab, dim, ws_, w_dt, 1.0, -1, flags, ws, ws_bytes, 0)


def test_embedding_arguments_that_no_call_takes():
    for call in (lookup, gradient):
        assert call(n=0, **({} if call is lookup else {"flags": 1})) == OK and call(dim=0) == OK
        for bad in (dict(ids=0), dict(ids=FAKE + 4), dict(id_bytes=2), dict(w=0), dict(w=FAKE * 3 + 2), dict(ws_=15)):
            assert call(**bad) == INVALID, bad
        for bad in (dict(vocab=1 << 31), dict(w_dt=tcuscan.I8_I32)):
            assert call(**bad) == UNSUPPORTED, bad
    assert lookup(o=0) == INVALID and lookup(os_=3) == INVALID and lookup(o=FAKE * 2) == INVALID and lookup(vocab=0) == INVALID
    assert lookup(o_dt=0) == UNSUPPORTED and lookup(ws=FAKE, ws_bytes=8) == WORKSPACE and lookup(ws=FAKE + 4, ws_bytes=256) == WORKSPACE
    assert gradient(g=0) == INVALID and gradient(gs=1) == INVALID and gradient(g=FAKE * 3) == INVALID and gradient(flags=2) == INVALID
    assert gradient(n=1 << 32) == UNSUPPORTED and gradient(ws=0) == WORKSPACE and gradient(ws=FAKE + 8) == WORKSPACE
    for n in (10, 5000, 100_000):
        need = tcuscan.embedding_backward_workspace_bytes(n, 100, 16)
        assert need >= 256 and gradient(n=n, ws_bytes=need - 1) == WORKSPACE
    assert tcuscan.embedding_backward_workspace_bytes(1 << 32, 5, 5) == 0


def test_the_binding_checks_shapes_types_and_strides():
    torch = pytest.importorskip("torch")
    q, v = torch.zeros(6, 2, 8), torch.zeros(6, 2, 4)
    g, off, out = torch.zeros(2), torch.tensor([0, 6]), torch.zeros(6, 2, 4)
    good = dict(q=q, k=q.clone(), v=v, out=out, log_decay=g, offsets=off)

    def refused(**change):
        with pytest.raises(ValueError):
            tcuscan.decay_attention(**{**good, **change})

    refused(k=torch.zeros(5, 2, 8))
    refused(k=torch.zeros(6, 2, 7))
    refused(out=torch.zeros(6, 2, 8))
    refused(v=v.bfloat16())
    refused(log_decay=torch.zeros(3))
    refused(log_decay=g.double())
    refused(offsets=off.int())
    refused(q=torch.zeros(6, 8, 2).transpose(1, 2))
    refused(state_in=torch.zeros(1, 2, 4, 8))
    refused(state_out=torch.zeros(1, 2, 8, 4, dtype=torch.float64))
    refused(state_in=torch.zeros(1, 2, 8, 4), state_out=torch.zeros(2, 2, 8, 4))
    refused(slots=torch.zeros(2, dtype=torch.int64), state_in=torch.zeros(3, 2, 8, 4))
    with pytest.raises(ValueError):
        tcuscan.decay_attention_backward(q, q.clone(), v, out, torch.zeros(6, 2, 8), torch.zeros(6, 1, 8), torch.zeros_like(v), g, off)
    with pytest.raises(ValueError):
        tcuscan.decay_attention_step(q, q.clone(), v, out, g, torch.zeros(6, 2, 8, 5))
    table, rows, ids = torch.zeros(9, 5), torch.zeros(3, 5), torch.zeros(3, dtype=torch.int64)
    for bad in ((ids.float(), table, rows), (ids.short(), table, rows), (ids, table, torch.zeros(2, 5)), (ids, table, torch.zeros(3, 4)), (ids, torch.zeros(5, 9).T, rows)):
        with pytest.raises(ValueError):
            tcuscan.embedding(*bad)
        with pytest.raises(ValueError):
            tcuscan.embedding_backward(bad[0], bad[2], bad[1])


def test_an_error_names_the_call():
    with pytest.raises(tcuscan.TcuscanError) as e:
        torch = pytest.importorskip("torch")
        tcuscan.embedding_backward(torch.zeros(3, dtype=torch.int64), torch.zeros(3, 5), torch.zeros(9, 5), stream=0)
    assert e.value.code == WORKSPACE and "tcuscan_embedding_backward" in str(e.value)
    assert ctypes.sizeof(ctypes.c_longlong) * 22 == len(shape())
