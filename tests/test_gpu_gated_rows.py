"""Gradients of the packed recurrence in the rows that belong to no sequence: zero, without a pass over the arrays of its own."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2411_17887_b200 import api

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def draw(t, d, dtype, lens, ahead):
    g = torch.Generator(device="cuda").manual_seed(t + d)
    x, gate, d_y = (torch.randn((t, d), generator=g, device="cuda").to(dtype) for _ in range(3))
    offsets = torch.tensor([ahead] + lens, device="cuda").cumsum(0)
    for z in (x, gate, d_y):                                   # what lies outside must not matter
        z[:ahead] = z[ahead + sum(lens):] = float("nan")
    return x, gate, d_y, offsets


class Ops(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.names = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        self.names.append(func.overloadpacket.__name__)
        return func(*args, **(kwargs or {}))


def test_nothing_is_cleared_ahead():
    x, gate, d_y, offsets = draw(100, 24, torch.bfloat16, [30, 40], 0)
    marks = api.gated_recurrence(x, gate, None, offsets, output_marks=True)[2]
    with Ops() as ops:
        api.gated_recurrence_backward(d_y, x, gate, None, offsets, marks=marks)
    assert ops.names and not [name for name in ops.names if "zero" in name or "fill" in name or "full" in name]


CASES = [([30, 40], 0, 30, 24), ([30, 40], 5, 0, 33), ([0], 70, 13, 64), ([0, 0, 0], 0, 100, 130), ([1], 0, 1, 1), ([700, 3, 1500], 2, 900, 66), ([5000], 17, 3000, 72), ([3, 0, 5] * 30, 1, 2000, 330),
         ([64] * 66, 3, 700, 200)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,ahead,behind,d", CASES, ids=lambda v: str(v)[:20])
def test_rows_of_no_sequence(lens, ahead, behind, d, dtype):
    from paper_2411_17887_b200 import binding as B
    t = ahead + sum(lens) + behind
    x, gate, d_y, offsets = draw(t, d, TYPES[dtype], lens, ahead)
    inside = slice(ahead, t - behind)
    first, d_last = torch.randn((2, len(lens), d), device="cuda")
    marks = api.gated_recurrence(x, gate, first, offsets, output_marks=True)[2]
    junk = [torch.full((t, d), float("nan"), device="cuda", dtype=TYPES[dtype]) for _ in range(4)]     # what fresh memory may hold
    del junk
    got = api.gated_recurrence_backward(d_y, x, gate, first, offsets, d_last, marks=marks)
    want = api.gated_recurrence_backward(d_y[inside], x[inside], gate[inside], first, offsets - ahead, d_last)
    for z, w in zip(got[:2], want[:2]):
        assert (z[:ahead] == 0).all() and (z[t - behind:] == 0).all() and torch.isfinite(z).all()
        assert z[inside].shape == w.shape
    assert torch.isfinite(got[2]).all()
    # from C, into a part of a larger array: what lies beside it is left alone, and with 0 so are the rows
    stream = torch.cuda.current_stream().cuda_stream
    for pad in (0, 3, 8):
        wide = d + pad
        for clear in (0, 1):
            held = torch.full((2, t + 4, wide), 7.0, device="cuda", dtype=TYPES[dtype])
            row = lambda z: (z.data_ptr(), 0, z.stride(0))  # noqa: E731
            args = B.tcu_gated_args({"f32": B.TCU_F32, "f16": B.TCU_F16, "bf16": B.TCU_BF16}[dtype], 0, d, len(lens), t, row(x), row(gate), d_y=row(d_y), d_x=row(held[0, 2:]),
                                    d_gate=row(held[1, 2:]), d_offsets=offsets.data_ptr(), d_marks=marks.data_ptr(), marks_bytes=marks.numel() * 4, d_dstate_out=d_last.data_ptr(),
                                    clear_rows=clear)
            assert B.tcu_gated_backward(args, stream) == B.TCU_OK
            assert (held[:, :2] == 7.0).all() and (held[:, t + 2:] == 7.0).all() and (held[..., d:] == 7.0).all()
            for z, w in zip(held[:, 2:t + 2, :d], got[:2]):
                assert torch.equal(z[inside], w[inside])
                assert (z[:ahead] == (7.0 if clear == 0 else 0.0)).all() and (z[t - behind:] == (7.0 if clear == 0 else 0.0)).all()


def test_no_sequences():
    x, gate, d_y, _ = draw(50, 8, torch.float16, [50], 0)
    d_x, d_gate, _ = api.gated_recurrence_backward(d_y, x, gate, offsets=torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert (d_x == 0).all() and (d_gate == 0).all()


def test_offsets_that_are_not_as_they_should_be():
    """Wrong results, but nothing is written outside the arrays, and the call returns."""
    from paper_2411_17887_b200 import binding as B
    x, gate, d_y, _ = draw(100, 64, torch.bfloat16, [100], 0)
    marks = torch.zeros((100 // 64 + 3, 64), device="cuda")
    row = lambda z: (z.data_ptr(), 0, 64)  # noqa: E731
    for wrong in ([0, 50, 20, 1 << 40], [-5, 10, 90, 100], [100, 80, 60, 0], [1 << 62, -(1 << 62), 3, 500], [40, 30, 20, 10]):
        guard = torch.full((2, 300, 64), 7.0, device="cuda", dtype=torch.bfloat16)
        offsets = torch.tensor(wrong, device="cuda")
        args = B.tcu_gated_args(B.TCU_BF16, 0, 64, 3, 100, row(x), row(gate), d_y=row(d_y), d_x=row(guard[0, 100:200]), d_gate=row(guard[1, 100:200]), d_offsets=offsets.data_ptr(),
                                d_marks=marks.data_ptr(), marks_bytes=marks.numel() * 4, clear_rows=1)
        assert B.tcu_gated_backward(args, torch.cuda.current_stream().cuda_stream) == B.TCU_OK
        torch.cuda.synchronize()
        assert (guard[:, :100] == 7.0).all() and (guard[:, 200:] == 7.0).all()


def test_structure():
    """Only 0 and 1; a structure that ends ahead of the field leaves the rows as they are."""
    from paper_2411_17887_b200 import binding as B
    x, gate, d_y, offsets = draw(100, 24, torch.bfloat16, [30, 40], 0)
    marks = api.gated_recurrence(x, gate, None, offsets, output_marks=True)[2]
    held = torch.full((2, 100, 24), 7.0, device="cuda", dtype=torch.bfloat16)
    row = lambda z: (z.data_ptr(), 0, 24)  # noqa: E731
    call = lambda clear: B.tcu_gated_args(B.TCU_BF16, 0, 24, 2, 100, row(x), row(gate), d_y=row(d_y), d_x=row(held[0]), d_gate=row(held[1]), d_offsets=offsets.data_ptr(),  # noqa: E731
                                          d_marks=marks.data_ptr(), marks_bytes=marks.numel() * 4, clear_rows=clear)
    stream = torch.cuda.current_stream().cuda_stream
    assert B.tcu_gated_backward(call(2), stream) == B.TCU_ERR_INVALID_ARG
    whole = call(1)
    former = (len(whole) - 8).to_bytes(4, "little") + whole[4:-8]
    assert B.tcu_gated_backward(former, stream) == B.TCU_OK and (held[:, 70:] == 7.0).all() and (held[:, :70] != 7.0).any()
    assert B.tcu_gated_backward(whole, stream) == B.TCU_OK and (held[:, 70:] == 0.0).all()


def test_capture():
    """A captured call clears by the offsets that it finds when it is replayed."""
    x, gate, d_y, offsets = draw(300, 40, torch.float16, [100, 150], 0)
    x.nan_to_num_(), gate.nan_to_num_(), d_y.nan_to_num_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call = lambda: api.gated_recurrence_backward(d_y, x, gate, None, offsets)  # noqa: E731
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call()
    for lens in ([100, 150], [10, 20], [0, 300], [0, 0]):
        offsets.copy_(torch.tensor([0] + lens).cumsum(0))
        outs[0].fill_(7.0), outs[1].fill_(7.0)
        graph.replay()
        for got, want in zip(outs[:2], call()):
            assert torch.equal(got, want) and (got[sum(lens):] == 0).all()
