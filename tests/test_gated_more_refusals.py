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
