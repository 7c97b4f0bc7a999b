"""Linear attention where calls begin and end: blocks leave nothing under way when they end."""
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.test_gpu_linattn import draw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert api.linear_attention_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 64, 64), (1, 37, 4, 64, 64), (2, 129, 3, 128, 128), (1, 2100, 1, 128, 128), (1, 300, 160, 16, 16), (300, 5, 1, 16, 72)], ids=str)
def test_short_calls_one_after_another(shape, dtype):
    """Nobody but the block itself waits for the commits of a walk's last group, least of all where no state is wanted.  The blocks of
    the next call, and of a scan with barriers in other places, take over the shared memory at once."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, _, _ = draw(t + h, b, t, h, dk, dv, dtype)
    x = torch.ones(40 * 16384, dtype=torch.int8, device="cuda")
    o, grads = api.linear_attention(q, k, v, decay)[0], api.linear_attention_backward(d_o, q, k, v, decay)[:3]
    want = api.scan(x)
    got = []
    for _ in range(30):
        got.append((api.linear_attention(q, k, v, decay)[0], api.linear_attention(q, k, v, decay)[0], api.scan(x), *api.linear_attention_backward(d_o, q, k, v, decay)[:3]))
    torch.cuda.synchronize()
    for one in got:
        for a, w in zip(one, (o, o, want, *grads)):
            assert torch.equal(a, w)
