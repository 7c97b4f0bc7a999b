"""Host-only checks of layer norm: argument errors are found before any launch, and the Python layer refuses what the library does not take."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


X, W, C, Y, DY, DX, DW, DB, WS = (0x1000_0000 * i for i in range(1, 10))


def test_forward_refusals(B):
    def f(x=X, rows=10, d=64, stride=64, dt=B.TCU_BF16, w=W, b=C, pt=B.TCU_F32, eps=1e-5, y=Y):
        return B.tcu_layer_norm_forward(x, rows, d, stride, dt, w, b, pt, eps, y)
    assert f(rows=0) == B.TCU_OK
    for bad in (dict(x=None), dict(y=None), dict(x=X + 1), dict(y=Y + 1), dict(w=W + 2), dict(b=C + 1), dict(d=0), dict(dt=3), dict(pt=-1), dict(eps=-1e-5), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(stride=(1 << 38) + 1), dict(y=X + 128), dict(y=X, stride=72), dict(y=W), dict(y=C - 1270), dict(rows=(1 << 31) - 1, stride=1 << 38, dt=B.TCU_F32)):
        assert f(**bad) == B.TCU_ERR_INVALID_ARG, bad
    for bad in (dict(pt=B.TCU_F16), dict(d=16385, stride=16385), dict(rows=1 << 31)):
        assert f(**bad) == B.TCU_ERR_UNSUPPORTED, bad


def test_backward_refusals(B):
    need = B.tcu_layer_norm_workspace_bytes(10, 64)
    assert need > 0 and B.tcu_layer_norm_workspace_bytes(10, 16385) == 0

    def f(dy=DY, dys=64, x=X, xs=64, rows=10, d=64, dt=B.TCU_BF16, w=W, pt=B.TCU_F32, eps=1e-5, dx=DX, dw=DW, db=DB, ws=WS, ws_bytes=need):
        return B.tcu_layer_norm_backward(dy, dys, x, xs, rows, d, dt, w, pt, eps, dx, dw, db, ws, ws_bytes)
    assert f(dx=None, dw=None, db=None) == B.TCU_OK
    assert f(rows=0, dw=None, db=None) == B.TCU_OK
    for bad in (dict(dy=None), dict(x=None), dict(dy=DY + 1), dict(dx=DX + 1), dict(dw=DW + 2), dict(db=DB + 2), dict(ws=WS + 8), dict(dx=X), dict(dx=DY + 64), dict(dx=DY, dys=65),
                dict(dw=DB), dict(dw=X), dict(dw=DY), dict(dw=DX), dict(dw=W), dict(ws=X), dict(ws=DY), dict(ws=DX), dict(ws=DW), dict(d=0), dict(dt=4), dict(eps=-1.0),
                dict(xs=(1 << 38) + 1), dict(dys=(1 << 38) + 1)):
        assert f(**bad) == B.TCU_ERR_INVALID_ARG, bad
    assert f(ws=None) == B.TCU_ERR_WORKSPACE
    assert f(ws_bytes=need - 1) == B.TCU_ERR_WORKSPACE
    assert f(pt=B.TCU_F16) == B.TCU_ERR_UNSUPPORTED


def test_python_layer_refuses(B):
    from paper_2411_17887_b200 import api
    x, w = torch.zeros((4, 6)), torch.ones(6)
    for error, call in ((TypeError, lambda: api.layer_norm(x.double())), (ValueError, lambda: api.layer_norm(x[:, :0])), (ValueError, lambda: api.layer_norm(torch.zeros(()))),
                        (ValueError, lambda: api.layer_norm(x, w[:5])), (TypeError, lambda: api.layer_norm(x, w.half())), (TypeError, lambda: api.layer_norm(x.half(), w.half(), w)),
                        (ValueError, lambda: api.layer_norm(x, w, eps=-1.0)), (ValueError, lambda: api.layer_norm(x, w, eps=float("nan"))),
                        (ValueError, lambda: api.layer_norm(x, torch.ones(12)[::2])), (ValueError, lambda: api.layer_norm(x, w)),
                        (ValueError, lambda: api.layer_norm_backward(x[:3], x, w)), (TypeError, lambda: api.layer_norm_backward(x.half(), x, w))):
        with pytest.raises(error):
            call()
