"""Host-only checks of the gated recurrence: argument errors are found before any launch, the Python layer refuses what the library does
not take, and the 64-bit gradients that the GPU tests compare with are the formula's differences."""
import numpy as np
import pytest
import torch

from tests import gated_reference as ref


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


X, G, Y, S0, S1, M, DY, DX, DG = (0x1000_0000 * i for i in range(1, 10))
N = dict(batch=2, tokens=100, channels=64)


def rows(ptr):
    return (ptr, 6400, 64)


def args(B, **change):
    a = dict(dtype=B.TCU_BF16, input_gate=0, x=rows(X), gate=rows(G), y=rows(Y), **N)
    a.update(change)
    return B.tcu_gated_args(**a)


def test_forward_refusals(B):
    bad = lambda **change: B.tcu_gated_forward(args(B, **change))  # noqa: E731
    assert bad(batch=0) == B.TCU_OK
    good = args(B, batch=0)
    assert B.tcu_gated_forward((8).to_bytes(4, "little") + good[4:]) == B.TCU_ERR_INVALID_ARG
    assert B.tcu_gated_forward(None) == B.TCU_ERR_INVALID_ARG
    for change in (dict(dtype=3), dict(input_gate=3), dict(channels=0), dict(x=B.NO_ROWS), dict(gate=B.NO_ROWS), dict(x=(X + 1, 6400, 64)), dict(x=(X, 6400, -64)),
                   dict(gate=(G, -1, 64)), dict(x=(X, (1 << 38) + 1, 64)), dict(y=(Y, 0, 64)), dict(y=(Y, 6400, 0)), dict(y=rows(X)), dict(y=rows(G + 128)),
                   dict(d_offsets=0x1004), dict(d_state_in=S0 + 2), dict(d_state_out=S1 + 1), dict(d_state_in=S0, d_state_out=S0 + 4), dict(d_state_out=Y), dict(d_state_in=Y),
                   dict(d_state_out=X + 64)):
        assert bad(**change) == B.TCU_ERR_INVALID_ARG, change
    need = B.tcu_gated_marks_bytes(2, 200, 64)
    assert need == (200 // 64 + 2) * 64 * 4
    assert bad(d_marks=M, marks_bytes=need - 1) == B.TCU_ERR_WORKSPACE
    for at in (X, Y, Y + 25536, S0 + 256):
        assert bad(d_marks=at, marks_bytes=need, d_state_in=S0) == B.TCU_ERR_INVALID_ARG
    assert bad(channels=(1 << 30) + 1) == B.TCU_ERR_UNSUPPORTED
    assert bad(tokens=(1 << 31) - 8191) == B.TCU_ERR_UNSUPPORTED
    assert bad(batch=1 << 31) == B.TCU_ERR_UNSUPPORTED
    assert bad(batch=1 << 63, channels=1 << 30) == B.TCU_ERR_UNSUPPORTED
    assert B.tcu_gated_marks_bytes(1 << 62, 1 << 40, 1 << 30) == 0


def test_backward_refusals(B):
    need = B.tcu_gated_marks_bytes(2, 200, 64)
    base = dict(y=B.NO_ROWS, d_y=rows(DY), d_x=rows(DX), d_gate=rows(DG), d_marks=M, marks_bytes=need)
    bad = lambda **change: B.tcu_gated_backward(args(B, **{**base, **change}))  # noqa: E731
    assert bad(batch=0) == B.TCU_OK
    assert bad(d_marks=0) == B.TCU_ERR_WORKSPACE
    assert bad(marks_bytes=need - 1) == B.TCU_ERR_WORKSPACE
    for change in (dict(x=B.NO_ROWS), dict(d_y=B.NO_ROWS), dict(d_x=B.NO_ROWS), dict(d_gate=B.NO_ROWS), dict(d_gate=rows(DX)), dict(d_x=rows(X)), dict(d_gate=rows(DY)),
                   dict(d_x=(DX, 0, 64)), dict(d_x=rows(M)), dict(d_dstate_in=S0, d_dstate_out=S0 + 4), dict(d_dstate_in=DX), dict(d_dstate_out=DG), dict(d_dstate_in=X),
                   dict(d_dstate_in=M), dict(d_y=(DY + 1, 6400, 64))):
        assert bad(**change) == B.TCU_ERR_INVALID_ARG, change


def test_step_refusals(B):
    bad = lambda **change: B.tcu_gated_step(args(B, **{**dict(d_state_out=S0, pool_slots=2, x=(X, 64, 0), gate=(G, 64, 0), y=(Y, 64, 0)), **change}))  # noqa: E731
    assert bad(batch=0) == B.TCU_OK
    for change in (dict(d_state_out=0), dict(pool_slots=1), dict(d_slots=0x1002), dict(d_offsets=0x1000), dict(y=(Y, 0, 0)), dict(y=(S0, 64, 0)), dict(x=(S0, 64, 0)),
                   dict(y=(X + 2, 64, 0)), dict(y=(G, 128, 0)), dict(x=B.NO_ROWS), dict(input_gate=9)):
        assert bad(**change) == B.TCU_ERR_INVALID_ARG, change
    assert bad(batch=1 << 31, pool_slots=1 << 31) == B.TCU_ERR_UNSUPPORTED


def test_python_layer_refuses(B):
    from paper_2411_17887_b200 import api
    x = torch.zeros((2, 10, 6))
    for error, call in ((TypeError, lambda: api.gated_recurrence(x.double(), x.double())), (TypeError, lambda: api.gated_recurrence(x, x.half())),
                        (ValueError, lambda: api.gated_recurrence(x, x[:, :9])), (ValueError, lambda: api.gated_recurrence(x[0], x[0])),
                        (ValueError, lambda: api.gated_recurrence(x, x, offsets=torch.tensor([0, 10]))), (ValueError, lambda: api.gated_recurrence(x, x, input_gate="none")),
                        (ValueError, lambda: api.gated_recurrence(x, x, torch.zeros((2, 5)))), (ValueError, lambda: api.gated_recurrence(x, x, torch.zeros((2, 6)).half())),
                        (ValueError, lambda: api.gated_recurrence(x[0], x[0], offsets=torch.tensor([0, 10], dtype=torch.int32))),
                        (ValueError, lambda: api.gated_recurrence(x[..., :0], x[..., :0])), (ValueError, lambda: api.gated_recurrence(x, x)),
                        (ValueError, lambda: api.gated_recurrence_backward(x[:, :9], x, x)), (ValueError, lambda: api.gated_recurrence_backward(x, x, x, marks=torch.zeros((1, 6)))),
                        (TypeError, lambda: api.gated_recurrence_backward(x.half(), x, x)), (ValueError, lambda: api.gated_recurrence_step(x, x, torch.zeros((2, 6)))),
                        (ValueError, lambda: api.gated_recurrence_step(x[:, 0], x[:, 0], torch.zeros((2, 5)))),
                        (ValueError, lambda: api.gated_recurrence_step(x[:, 0], x[:, 0], torch.zeros((2, 6)), torch.zeros(2))),
                        (ValueError, lambda: api.gated_recurrence_step(x[:, 0], x[:, 0], torch.zeros((2, 6))))):
        with pytest.raises(error):
            call()


@pytest.mark.parametrize("kind", ["complement", "one", "root"])
def test_reference_gradients_are_differences(kind):
    rng = np.random.default_rng(5)
    x, g, d_y = (rng.standard_normal((9, 4)) for _ in range(3))
    first, d_last = rng.standard_normal(4), rng.standard_normal(4)
    want = ref.backward(x, g, d_y, kind, first, d_last, torch.float32)

    def loss(x, g, s):
        (h, _), (last, _) = ref.forward(x, g, kind, s, torch.float32)
        return (h * d_y).sum() + (last * d_last).sum()

    for which, (value, _) in enumerate(want):
        for at in np.ndindex(value.shape):
            moved = []
            for step in (1e-5, -1e-5):
                some = [x.copy(), g.copy(), first.copy()]
                some[which][at] += step
                moved.append(loss(*some))
            assert abs((moved[0] - moved[1]) / 2e-5 - value[at]) < 1e-8
