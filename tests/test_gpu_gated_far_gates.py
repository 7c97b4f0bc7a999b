"""Gates far from zero in every type: 32-bit states and the outputs of both, prompts and single tokens, to the bounds that each type has.

The bounds are those of tests/gated_reference.py, with what 16-bit sequences leave out added: exp(-|g|) is off by up to 1.23 |g| u besides (u = 2^-24: the product
|g| log2(e) is rounded by u of itself, the constant by 0.23 u, both times ln 2), taken as 1.3 |g| u, so that 20 + 1.3 |g| stands in the place of 20:
    E_t = f (E_{t-1} + u (4 + (20 + 1.3 |g|) rest) A_{t-1}) + (20 + 1.3 |g|) u |b_t| + 2 u A_t
"""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests import gated_reference as ref
from tests.lm_reference import assert_within, f64

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
u = ref.u


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def forward(x, g, kind, first, wide):
    """(t, d): h, last state, and the bounds of both in 32 bits."""
    f, rest, i, _, _ = ref.gates(g, kind)
    b, lost = i * x, ref.LOST[kind] * np.abs(x)
    many = 20.0 + (1.3 * np.abs(g) if wide else 0.0)
    h, e, a = first.copy(), np.zeros_like(first), np.abs(first)
    hs, es = np.zeros_like(b), np.zeros_like(b)
    for k in range(len(b)):
        e = f[k] * (e + u * (4.0 + many[k] * rest[k] if wide else u * (4.0 + 20.0 * rest[k])) * a) + (many[k] if wide else 20.0) * u * np.abs(b[k]) + ref.F * a + lost[k]
        h = f[k] * h + b[k]
        a = f[k] * a + np.abs(b[k])
        e = e + 2.0 * u * a
        hs[k], es[k] = h, e
    return hs, es, h, e + 1e-37


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["complement", "one", "root"])
@pytest.mark.parametrize("t,d", [(40, 64), (130, 33), (300, 2)])
def test_gates_of_30_to_80(t, d, kind, dtype):
    g = torch.Generator(device="cuda").manual_seed(t + d)
    kind_of = TYPES[dtype]
    x = torch.randn((1, t, d), generator=g, device="cuda").to(kind_of)
    gate = 30.0 + 50.0 * torch.rand((1, t, d), generator=g, device="cuda")
    sign = torch.randint(0, 2, (1, t, d), generator=g, device="cuda") * 2 - 1
    sign[..., 0], sign[..., 1] = 1, -1                        # a channel that only remembers, one that only forgets
    gate = (gate * sign).to(kind_of)
    for first in (torch.zeros((1, d), device="cuda"), torch.randn((1, d), generator=g, device="cuda")):
        wide = dtype != "f32"
        hs, es, h, e = forward(f64(x[0]), f64(gate[0]), kind, f64(first[0]), wide)
        y, last = api.gated_recurrence(x, gate, first, output_final_state=True, input_gate=kind)
        assert_within(y[0], hs, ref.rounded(hs, es, kind_of), "y")
        assert_within(last[0], h, e, "state")
        # token by token: the bound without what is left out
        pool = first.clone()
        for k in range(t):
            api.gated_recurrence_step(x[:, k], gate[:, k], pool, input_gate=kind)
        _, _, h, e = forward(f64(x[0]), f64(gate[0]), kind, f64(first[0]), False)
        assert_within(pool[0], h, e, "state of the steps")
