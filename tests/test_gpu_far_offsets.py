"""The recurrence, the norm and the sampling on arrays of more than 2^31 elements: both ends give what copies of them give alone."""
import pytest
import torch

from paper_2411_17887_b200 import api

pytestmark = pytest.mark.gpu
TOKENS, CHANNELS = 530000, 4096            # 2.17e9 elements


@pytest.fixture(scope="module")
def array():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((TOKENS, CHANNELS), generator=g, device="cuda", dtype=torch.bfloat16)
    yield x
    del x
    torch.cuda.empty_cache()


def test_recurrence(array):
    """Channels do not meet, and 64 channels alone are walked by as many blocks in the same order."""
    x = array[None]
    gate, d_y = x.flip(2), x.neg()
    y, last, marks = api.gated_recurrence(x, gate, None, None, True, output_marks=True)
    d_x, d_gate, _ = api.gated_recurrence_backward(d_y, x, gate, marks=marks)
    for at in (0, CHANNELS - 64):
        some = [z[..., at:at + 64].contiguous() for z in (x, gate, d_y)]
        want = api.gated_recurrence(*some[:2], None, None, True, output_marks=True)
        grads = api.gated_recurrence_backward(some[2], *some[:2], marks=want[2])
        for name, got, one in (("y", y, want[0]), ("state", last, want[1]), ("d_x", d_x, grads[0]), ("d_gate", d_gate, grads[1])):
            # the bounds of two blocks' walk are those of one: 2^-8 of a value for the rounding, sums of other orders 2^-20 of the largest
            got, one = got[..., at:at + 64].float(), one.float()
            assert torch.isfinite(one).all() and ((got - one).abs() <= one.abs() * 2.0 ** -7 + one.abs().max() * 2.0 ** -20).all(), (name, at)


def test_norm(array):
    x = array.view(-1, 2048)
    d_y, weight = x.flip(1), torch.linspace(-2, 2, 2048, device="cuda")
    y = api.layer_norm(x, weight)
    d_x, _, _ = api.layer_norm_backward(d_y, x, weight)
    for rows in (slice(0, 700), slice(x.shape[0] - 700, x.shape[0])):
        assert torch.equal(y[rows], api.layer_norm(x[rows].clone(), weight))
        assert torch.equal(d_x[rows], api.layer_norm_backward(d_y[rows].clone(), x[rows].clone(), weight)[0])


def test_sample(array):
    rows, vocabulary = 17000, 127000                                       # 2.16e9
    logits = array.view(-1)[:rows * vocabulary].view(rows, vocabulary)
    uniform = torch.rand(rows, device="cuda")
    tokens = api.sample(logits, uniform, 0.8, top_k=50)
    for part in (slice(0, 200), slice(rows - 200, rows)):
        assert torch.equal(tokens[part], api.sample(logits[part].clone(), uniform[part], 0.8, top_k=50))
    far = array.view(-1).as_strided((2, 1000), (TOKENS * CHANNELS - 2000, 1))           # a row's stride of more than 31 bits
    assert torch.equal(api.sample(far, uniform[:2], 0.0), far.float().argmax(1))
