"""Host-only checks of the language-model entry points: argument errors are found before any launch, sizes are as documented,
and the Python layer refuses what the library does not take."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


# addresses that are never dereferenced: every call below fails a host check, or has nothing to do
Q, K, V, O, G, WS, S0, S1 = (0x1000_0000 * i for i in range(1, 9))


def dense(ptr, t, h, d):
    return (ptr, t * h * d, h * d, d)


def args(B, **change):
    b, t, h, dk, dv = 2, 100, 3, 64, 64
    a = dict(dtype=B.TCU_BF16, batch=b, tokens=t, heads=h, dk=dk, dv=dv, scale=1.0, d_log_decay=G, q=dense(Q, t, h, dk), k=dense(K, t, h, dk),
             v=dense(V, t, h, dv), o=dense(O, t, h, dv))
    a.update(change)
    return B.tcu_linattn_args(**a)


def test_struct_size_is_checked(B):
    good = args(B, batch=0)
    assert B.tcu_linattn_forward(good, WS, 256) == B.TCU_OK                       # nothing to do
    assert B.tcu_linattn_forward((0).to_bytes(4, "little") + good[4:], WS, 256) == B.TCU_ERR_INVALID_ARG
    assert B.tcu_linattn_forward(None, WS, 256) == B.TCU_ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["forward", "backward"])
def test_linear_attention_refusals(B, call):
    grads = dict(d_o=dense(0x9000_0000, 100, 3, 64), d_q=dense(0xA000_0000, 100, 3, 64), d_k=dense(0xB000_0000, 100, 3, 64), d_v=dense(0xC000_0000, 100, 3, 64))
    fn = B.tcu_linattn_forward if call == "forward" else B.tcu_linattn_backward
    bad = lambda ws=WS, ws_bytes=256, **change: fn(args(B, **{**grads, **change}), ws, ws_bytes)  # noqa: E731
    assert bad(ws=None) == B.TCU_ERR_WORKSPACE
    assert bad(ws_bytes=255) == B.TCU_ERR_WORKSPACE
    assert bad(dtype=B.TCU_F32) == B.TCU_ERR_INVALID_ARG
    assert bad(dtype=7) == B.TCU_ERR_INVALID_ARG
    assert bad(heads=0) == B.TCU_ERR_INVALID_ARG
    assert bad(dk=0) == B.TCU_ERR_INVALID_ARG
    assert bad(dk=136) == B.TCU_ERR_UNSUPPORTED
    assert bad(dv=129) == B.TCU_ERR_UNSUPPORTED
    assert bad(tokens=1 << 31) == B.TCU_ERR_UNSUPPORTED
    assert bad(batch=1 << 30) == B.TCU_ERR_UNSUPPORTED
    assert bad(d_log_decay=0) == B.TCU_ERR_INVALID_ARG
    assert bad(d_offsets=0x1004) == B.TCU_ERR_INVALID_ARG
    assert bad(d_state_in=S0 + 4) == B.TCU_ERR_INVALID_ARG
    for name, ptr in (("q", Q), ("k", K), ("v", V)):
        assert bad(**{name: (0, 19200, 192, 64)}) == B.TCU_ERR_INVALID_ARG                # no pointer
        assert bad(**{name: (ptr + 2, 19200, 192, 64)}) == B.TCU_ERR_INVALID_ARG          # off a 16-byte boundary
        assert bad(**{name: (ptr, 19200, 196, 64)}) == B.TCU_ERR_INVALID_ARG              # so is every second row
        assert bad(**{name: (ptr, 19200, -192, 64)}) == B.TCU_ERR_INVALID_ARG
        assert bad(**{name: (ptr, 19200, 0, 64)}) == B.TCU_ERR_INVALID_ARG                # one token for all
    if call == "forward":
        assert bad(o=dense(Q + 64, 100, 3, 64)) == B.TCU_ERR_INVALID_ARG                  # overlaps an input
        assert bad(o=(O, 19200, 192, 0)) == B.TCU_ERR_INVALID_ARG                         # heads written over one another
    else:
        assert bad(d_k=dense(0x9000_0000, 100, 3, 64)) == B.TCU_ERR_INVALID_ARG           # overlaps d_o
        assert bad(d_v=(0xC000_0000, 0, 192, 64)) == B.TCU_ERR_INVALID_ARG
        assert bad(d_dstate_in=S0, d_dstate_out=S0) == B.TCU_ERR_INVALID_ARG


def test_step_refusals(B):
    bad = lambda **change: B.tcu_linattn_step(args(B, **{**dict(d_state_out=S0, pool_slots=2), **change}))  # noqa: E731
    assert bad(batch=0) == B.TCU_OK
    assert bad(d_state_out=0) == B.TCU_ERR_INVALID_ARG
    assert bad(d_state_out=S0 + 8) == B.TCU_ERR_INVALID_ARG
    assert bad(pool_slots=1) == B.TCU_ERR_INVALID_ARG                 # fewer entries than sequences, and no slots
    assert bad(d_slots=0x1002) == B.TCU_ERR_INVALID_ARG
    assert bad(dk=200) == B.TCU_ERR_UNSUPPORTED
    assert bad(dtype=B.TCU_F32) == B.TCU_ERR_INVALID_ARG
    assert bad(q=(Q + 1, 192, 0, 64)) == B.TCU_ERR_INVALID_ARG
    assert bad(o=(O, 0, 0, 64)) == B.TCU_ERR_INVALID_ARG


def test_embedding_refusals(B):
    f = lambda ids=Q, idb=8, n=10, table=K, rows=5, d=16, stride=16, dt=B.TCU_BF16, out=V: B.tcu_embedding_forward(ids, idb, n, table, rows, d, stride, dt, 1.0, out)  # noqa: E731
    assert f(n=0) == B.TCU_OK
    for bad in (dict(ids=None), dict(table=None), dict(out=None), dict(idb=2), dict(dt=3), dict(stride=15), dict(ids=Q + 4), dict(table=K + 1), dict(out=K)):
        assert f(**bad) == B.TCU_ERR_INVALID_ARG, bad
    assert f(n=1 << 30) == B.TCU_ERR_UNSUPPORTED
    assert f(d=1 << 21, stride=1 << 21) == B.TCU_ERR_UNSUPPORTED
    need = B.tcu_embedding_workspace_bytes(10, 5, 16)
    assert need > 0 and B.tcu_embedding_workspace_bytes(0, 0, 0) > 0

    def g(out=Q, dt=B.TCU_BF16, ids=K, idb=8, n=10, rows=5, d=16, table=V, tt=B.TCU_F32, ws=WS, ws_bytes=need):
        return B.tcu_embedding_backward(out, dt, ids, idb, n, rows, d, 1.0, 0, table, tt, ws, ws_bytes)
    assert g(rows=0) == B.TCU_OK
    for bad in (dict(out=None), dict(ids=None), dict(table=None), dict(idb=3), dict(dt=5), dict(tt=-1), dict(out=Q + 1), dict(table=V + 2), dict(ws=WS + 16), dict(table=Q)):
        assert g(**bad) == B.TCU_ERR_INVALID_ARG, bad
    assert g(tt=B.TCU_F16) == B.TCU_ERR_UNSUPPORTED
    assert g(n=1 << 30) == B.TCU_ERR_UNSUPPORTED
    assert g(ws=None) == B.TCU_ERR_WORKSPACE
    assert g(ws_bytes=need - 1) == B.TCU_ERR_WORKSPACE


def test_python_layer_refuses(B):
    from paper_2411_17887_b200 import api
    q = torch.zeros((2, 10, 3, 64), dtype=torch.bfloat16)
    decay = torch.zeros(3)
    with pytest.raises(TypeError):
        api.linear_attention(q.float(), q.float(), q.float(), decay)
    with pytest.raises(TypeError):
        api.linear_attention(q, q.half(), q, decay)
    with pytest.raises(ValueError):
        api.linear_attention(q, q[:, :9], q, decay)
    with pytest.raises(ValueError):
        api.linear_attention(q, q, q, torch.zeros(4))
    with pytest.raises(ValueError):
        api.linear_attention(q, q, q, decay, initial_state=torch.zeros((2, 3, 64, 63)))
    with pytest.raises(ValueError):
        api.linear_attention(q, q, q, decay, offsets=torch.tensor([0, 10]))                # packed arrays have three axes
    with pytest.raises(ValueError):
        api.linear_attention(q, q, q, decay)                                               # not on a GPU
    with pytest.raises(ValueError):
        api.linear_attention_step(q[:, 0], q[:, 0], q[:, 0], decay, torch.zeros((2, 3, 64, 32)))
    with pytest.raises(ValueError):
        api.embedding(torch.zeros(3), torch.zeros((5, 8)))
    with pytest.raises(ValueError):
        api.embedding(torch.zeros(3, dtype=torch.int64), torch.zeros((5, 8)))
    with pytest.raises(TypeError):
        api.embedding_backward(torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int64), 5, dtype=torch.float16)
