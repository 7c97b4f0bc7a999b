"""States of linear attention are results in 32 bits: keys enter them in as many 16-bit terms as that takes.

lm_reference.py bounds states by 2^-16 of the sum of absolute products, which two bfloat16 terms of a key keep.  Here a few tokens are
all there is, so that little else is rounded, and the bounds tell three terms (2^-24 of a key) from two (up to 2^-18):
 - without decay the powers are exact.  A key is a 16-bit value times the scale, in three terms off by 2 * 2^-24; 16 tokens of one
   value are one step of a product for each term, in which no more than 2^-23 of the sum is lost: 2^-24 (2 + 3 * 2) in all, and as much
   again where a state is taken out of one block into another and back;
 - with decay a state is k a^m, with a^m a product of at most three powers, each off by two units in the last place (4 * 2^-24) and
   what the logarithm's rounding makes of it (2 * 2^-24 |m log2 a|), six more roundings, and the key's own as above."""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.lm_reference import assert_within, f64

pytestmark = pytest.mark.gpu
UNIT = 2.0 ** -24


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert api.linear_attention_status() == 0


def bf16(x):
    return f64(torch.from_numpy(np.asarray(x, np.float64)).to(torch.bfloat16))


def off_in_two_terms(k, f):
    """Relative error of k f as two bfloat16 terms."""
    f1 = bf16(f)
    hi = bf16(k * f1)
    return np.abs(k * f - hi - bf16(k * bf16(f - f1) + (k * f1 - hi))) / (k * f)


# whole walks, parts of a cluster, walks cut over blocks
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("b,t,h,dk,dv", [(1, 100, 1, 128, 64), (1, 300, 2, 64, 64), (1, 2100, 1, 128, 64), (2, 700, 80, 64, 24)])
@pytest.mark.parametrize("where", [0.0, 0.4, 1.0])
def test_without_decay(b, t, h, dk, dv, where, dtype):
    """The gradient of the first state: sum of scale q do^T."""
    scale = float(np.float32(0.3))
    at = int((t - 16) * where)
    q = torch.zeros((b, t, h, dk), device="cuda", dtype=dtype)
    values = 1 + (torch.arange(dk, device="cuda") % 128) / 128.0                 # every mantissa of bfloat16
    q[:, at:at + 16] = values.to(dtype)
    d_o = torch.zeros((b, t, h, dv), device="cuda", dtype=dtype)
    d_o[:, at:at + 16] = 1.0
    decay = torch.zeros(h, device="cuda")
    d_first = api.linear_attention_backward(d_o, q, q, d_o, decay, scale, torch.zeros((b, h, dk, dv), device="cuda"))[3]
    want = np.broadcast_to(16 * scale * f64(values)[:, None], (b, h, dk, dv))
    bound = 2 * UNIT * (2 + 3 * 2) * want
    assert off_in_two_terms(f64(values), scale).max() * want.max() > 2 * bound.max()
    assert_within(d_first, want, bound, "d_initial_state")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("b,t,h,dk,dv", [(1, 100, 1, 128, 64), (1, 300, 2, 64, 64), (1, 2100, 1, 128, 64), (2, 700, 80, 64, 24)])
@pytest.mark.parametrize("log_decay", [-1e-3, -2.0 ** -12])
def test_with_decay(b, t, h, dk, dv, log_decay, dtype):
    """The state after the last token, from one token at most two groups before it."""
    values = 1 + (torch.arange(dk, device="cuda") % 128) / 128.0
    decay = torch.full((h,), log_decay, device="cuda")
    teeth = 0.0
    for ago in (0, 1, 50, 99, 180):
        if ago >= t:
            continue
        k = torch.zeros((b, t, h, dk), device="cuda", dtype=dtype)
        k[:, t - 1 - ago] = values.to(dtype)
        v = torch.zeros((b, t, h, dv), device="cuda", dtype=dtype)
        v[:, t - 1 - ago] = 1.0
        last = api.linear_attention(k, k, v, decay, output_final_state=True)[1]
        f = np.exp(f64(decay)[0] * ago)
        want = np.broadcast_to(f64(values)[:, None] * f, (b, h, dk, dv))
        bound = UNIT * (3 * 4 + 2 * ago * abs(log_decay) * 1.4427 + 6 + 2) * want
        teeth = max(teeth, off_in_two_terms(f64(values), f).max() * want.max() / bound.max())
        assert_within(last, want, bound, "final state")
    assert teeth > 1.5
