"""What the gated recurrence's host code takes and refuses besides: fields that a call does not use are not looked at, and nothing is written over the indices it reads."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


X, G, Y, S0, S1, M, DY, DX, DG, OFF, SLOTS = (0x1000_0000 * i for i in range(1, 12))


def rows(at):
    return (at, 0, 64)


def test_a_step_does_not_look_at_tokens(B):
    for tokens in (0, 1, 1 << 31, 1 << 63):
        args = B.tcu_gated_args(B.TCU_BF16, 0, 64, 0, tokens, (X, 64, 0), (G, 64, 0), (Y, 64, 0), d_state_out=S0)
        assert B.tcu_gated_step(args) == B.TCU_OK, tokens


def test_nothing_is_written_over_offsets(B):
    """3 sequences: 4 offsets, 32 bytes."""
    marks = B.tcu_gated_marks_bytes(3, 100, 64)

    def forward(**change):
        a = dict(y=rows(Y), d_offsets=OFF, d_state_in=S0, d_state_out=S1, d_marks=M, marks_bytes=marks)
        a.update(change)
        return B.tcu_gated_forward(B.tcu_gated_args(B.TCU_BF16, 0, 64, 3, 100, rows(X), rows(G), **a))

    def backward(**change):
        a = dict(d_y=rows(DY), d_x=rows(DX), d_gate=rows(DG), d_offsets=OFF, d_dstate_out=S0, d_dstate_in=S1, d_marks=M, marks_bytes=marks)
        a.update(change)
        return B.tcu_gated_backward(B.tcu_gated_args(B.TCU_BF16, 0, 64, 3, 100, rows(X), rows(G), **a))

    for at in (0, -8, 8, 24):
        back = 8 + max(at, 0)                                   # offsets that begin so many bytes ahead of an array's end
        for change in (dict(y=rows(OFF + at)), dict(d_state_out=OFF + at), dict(d_marks=OFF + at), dict(d_offsets=Y + 12800 - back), dict(d_offsets=S1 + 768 - back), dict(d_offsets=M + marks - back)):
            assert forward(**change) == B.TCU_ERR_INVALID_ARG, change
        for change in (dict(d_x=rows(OFF + at)), dict(d_gate=rows(OFF + at)), dict(d_dstate_in=OFF + at), dict(d_offsets=DX + 12800 - back), dict(d_offsets=DG + 12800 - back)):
            assert backward(**change) == B.TCU_ERR_INVALID_ARG, change


def test_nothing_is_written_over_slots(B):
    """5 sequences: 20 bytes."""
    def step(**change):
        a = dict(y=(Y, 64, 0), d_slots=SLOTS, pool_slots=7, d_state_out=S0)
        a.update(change)
        return B.tcu_gated_step(B.tcu_gated_args(B.TCU_BF16, 0, 64, 5, 1, (X, 64, 0), (G, 64, 0), **a))

    for change in (dict(y=(SLOTS, 64, 0)), dict(y=(SLOTS + 16, 64, 0)), dict(d_slots=Y + 636), dict(d_state_out=SLOTS + 16), dict(d_slots=S0 + 1788), dict(d_slots=S0)):
        assert step(**change) == B.TCU_ERR_INVALID_ARG, change
