"""Layer norm where every block, or group of lanes, goes through several rows, in all types and shapes of a row: rows that come after one another through the same
registers and shared memory, and sums of the parameters' gradients over all of them."""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests import norm_reference as ref
from tests.lm_reference import assert_within, f64

pytestmark = pytest.mark.gpu
TYPES = [(torch.float32, torch.float32), (torch.float16, torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def sums(d_y, x, eps, param_type):
    """The parameters' gradients and their bounds.  In a block at most rows / 100 + 8 are added in order (of the blocks' 148 or more, some lanes of a warp and its eight warps),
    then the blocks' parts, at most 1184: 32 groups of 37 in order, 5 levels."""
    v, dv, r, loose = ref.parts(x, eps)
    n = v * r
    dn = r * dv + loose * np.abs(n) + ref.u * np.abs(n)
    many = x.shape[0] / 100 + 8 + 1184 / 32 + 5
    e_w = (np.abs(d_y) * dn).sum(0) + (many + 1) * ref.u * np.abs(d_y * n).sum(0)
    d_w, d_b = (d_y * n).sum(0), d_y.sum(0)
    return (d_w, ref.rounded(d_w, e_w, param_type)), (d_b, ref.rounded(d_b, many * ref.u * np.abs(d_y).sum(0), param_type))


# widths of 8, 16 and 32 lanes, of a block with 16 elements a thread and with 32, read 16 bytes, 4 bytes and one element at a time, full and not
@pytest.mark.parametrize("dtype,param_type", TYPES, ids=str)
@pytest.mark.parametrize("rows,d", [(20000, 64), (9500, 129), (12000, 300), (5000, 512), (5000, 1000), (5000, 1024), (3000, 1537), (1300, 2050), (700, 8192), (400, 10000), (400, 12002), (330, 16384),
                                    (330, 9001), (310, 8200), (500, 12288)])
def test_rows_after_one_another(rows, d, dtype, param_type):
    g = torch.Generator(device="cuda").manual_seed(rows + d)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, d_y = (normal(rows, d) * (0.1 + normal(rows, 1).abs()) + normal(rows, 1)).to(dtype), normal(rows, d).to(dtype)
    weight, bias = (1.0 + 0.5 * normal(d)).to(param_type), normal(d).to(param_type)
    y, (d_x, d_w, d_b) = api.layer_norm(x, weight, bias), api.layer_norm_backward(d_y, x, weight)
    some = np.unique(np.concatenate([np.arange(0, rows, max(1, rows // 97)), np.arange(max(0, rows - 40), rows)]))       # rows looked at
    pick = lambda z: f64(z[torch.from_numpy(some).cuda()])  # noqa: E731
    assert_within(pick(y), *ref.forward(pick(x), f64(weight), f64(bias), 1e-5, dtype), "y")
    assert_within(pick(d_x), *ref.backward(pick(d_y), pick(x), f64(weight), 1e-5, dtype, param_type)[0], "d_x")
    for name, got, (value, bound) in zip(("d_weight", "d_bias"), (d_w, d_b), sums(f64(d_y), f64(x), 1e-5, param_type)):
        assert_within(got, value, bound, name)
    # every row as it is alone
    at = int(some[len(some) // 2])
    assert torch.equal(api.layer_norm(x[at:at + 1], weight, bias), y[at:at + 1])
    assert torch.equal(api.layer_norm_backward(d_y[at:at + 1], x[at:at + 1], weight, params=False)[0], d_x[at:at + 1])
