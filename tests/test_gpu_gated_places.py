"""What the gated recurrence may write in the place of what it reads: the final state over the initial one, the gradient of one over that of the other, and a
step's output over x or the gate.  The same bits as in places of their own."""
import pytest
import torch

from paper_2411_17887_b200 import api
from paper_2411_17887_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"f32": (torch.float32, B.TCU_F32), "f16": (torch.float16, B.TCU_F16), "bf16": (torch.bfloat16, B.TCU_BF16)}


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def draw(dtype, *shape):
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    return [torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(3)]


def stream():
    return torch.cuda.current_stream().cuda_stream


# (lens of packed sequences, or None; batch, tokens, channels): one block a walk, clusters, short and empty sequences, sequences in the order of their lengths
CASES = [(None, 3, 1, 5), (None, 2, 700, 66), (None, 1, 5000, 130), (None, 300, 130, 64), ([0, 0], 2, 0, 9), ([0, 5, 300, 0, 64], 5, 369, 200), ([7] * 30, 30, 210, 710),
         ([100, 0, 3] * 20, 60, 2060, 330)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,batch,t,d", CASES, ids=lambda v: str(v)[:16])
def test_states(lens, batch, t, d, dtype):
    kind, code = TYPES[dtype]
    x, gate, d_y = draw(kind, *((t, d) if lens else (batch, t, d)))
    offsets = torch.tensor([0] + lens, device="cuda").cumsum(0) if lens else None
    first, d_last = torch.randn((2, batch, d), device="cuda")
    y, last, marks = api.gated_recurrence(x, gate, first, offsets, True, output_marks=True)
    d_x, d_gate, d_first = api.gated_recurrence_backward(d_y, x, gate, first, offsets, d_last, marks=marks)
    row = lambda z: (z.data_ptr(), 0 if lens else t * d, d)  # noqa: E731
    outs, state = [torch.zeros_like(x) for _ in range(3)], first.clone()
    more = dict(d_offsets=offsets.data_ptr() if lens else 0, d_marks=marks.data_ptr(), marks_bytes=marks.numel() * 4)
    for _ in range(3):                                         # (a race need not show at once)
        state.copy_(first)
        args = B.tcu_gated_args(code, 0, d, batch, t, row(x), row(gate), row(outs[0]), d_state_in=state.data_ptr(), d_state_out=state.data_ptr(), **more)
        assert B.tcu_gated_forward(args, stream()) == B.TCU_OK
        assert torch.equal(state, last) and torch.equal(outs[0], y)
        state.copy_(d_last)
        args = B.tcu_gated_args(code, 0, d, batch, t, row(x), row(gate), d_y=row(d_y), d_x=row(outs[1]), d_gate=row(outs[2]), d_dstate_out=state.data_ptr(), d_dstate_in=state.data_ptr(), **more)
        assert B.tcu_gated_backward(args, stream()) == B.TCU_OK
        assert torch.equal(state, d_first) and torch.equal(outs[1], d_x) and torch.equal(outs[2], d_gate)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,d,pad", [(1, 1, 0), (5, 130, 0), (70, 1000, 7), (3, 4099, 1)])
def test_step(b, d, pad, dtype):
    kind, code = TYPES[dtype]
    x, gate, _ = draw(kind, b, d + pad)
    pool = torch.randn((b + 2, d), device="cuda")
    slots = torch.randperm(b + 2, device="cuda")[:b].to(torch.int32)
    if b > 2:
        slots[1] = -1                                          # skipped: zeros in its place
    want_pool = pool.clone()
    want = api.gated_recurrence_step(x[:, :d], gate[:, :d], want_pool, slots)
    for place in range(2):
        both, state = [x.clone(), gate.clone()], pool.clone()
        row = lambda z: (z.data_ptr(), d + pad, 0)  # noqa: E731
        args = B.tcu_gated_args(code, 0, d, b, 1, row(both[0]), row(both[1]), row(both[place]), d_slots=slots.data_ptr(), pool_slots=b + 2, d_state_out=state.data_ptr())
        assert B.tcu_gated_step(args, stream()) == B.TCU_OK
        assert torch.equal(both[place][:, :d], want) and torch.equal(state, want_pool)
        assert torch.equal(both[place][:, d:], (x, gate)[place][:, d:]) and torch.equal(both[1 - place], (x, gate)[1 - place])
    # one array for x, gate and y
    same, state = x.clone(), pool.clone()
    args = B.tcu_gated_args(code, 0, d, b, 1, row(same), row(same), row(same), d_slots=slots.data_ptr(), pool_slots=b + 2, d_state_out=state.data_ptr())
    assert B.tcu_gated_step(args, stream()) == B.TCU_OK
    other = pool.clone()
    assert torch.equal(same[:, :d], api.gated_recurrence_step(x[:, :d], x[:, :d], other, slots)) and torch.equal(state, other)
