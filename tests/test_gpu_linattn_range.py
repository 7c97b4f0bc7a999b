"""Linear attention over the range of its types: scores, keys, states, gradients and decays that are large, small or not numbers.

The bounds are those of lm_reference.py without its allowance for scores and keys that fall below float16's smallest step: scores,
states and keys are brought to the type's range by powers of two that put the largest of a token (scores) or of a group (the
others) near 2^14, so that a step of 2^-24 is 2^-38 of that largest, and half of it is lost at most.  What remains is the step of
the outputs themselves, 2^-24, and, with S and X the largest score and state there can be,
    2^-38 (128 S max |v| + dk max |q| X)."""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.lm_reference import U, assert_within, f64, mix, transpose
from tests.test_gpu_linattn import draw

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]
# walks run whole (64 and 128 wide), in parts of a cluster, and cut over blocks
SHAPES = [(1, 300, 2, 64, 64), (2, 300, 2, 128, 128), (1, 2100, 1, 128, 72), (2, 300, 80, 16, 24)]
each = lambda f: pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])(pytest.mark.parametrize("shape", SHAPES, ids=str)(f))  # noqa: E731


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert api.linear_attention_status() == 0


def bounded(dtype, q, k, v, decay, lead, init, in_scale, out_scale):
    o, x = mix(q, k, v, decay, lead, init, in_scale, out_scale)
    ao, ax = mix(*(np.abs(y) for y in (q, k, v)), decay, lead, None if init is None else np.abs(init), abs(in_scale), abs(out_scale))
    u, (t, dk) = U[dtype], (q.shape[1], q.shape[3])
    big_q, big_k, big_v = (np.abs(y).max() for y in (q, k, v))
    score = dk * big_q * big_k * abs(in_scale * out_scale)
    state = t * big_k * big_v * abs(in_scale) + (0.0 if init is None else np.abs(init).max())
    small = 2.0 ** -24 + 2.0 ** -38 * (128 * score * big_v + dk * big_q * state * abs(out_scale)) if dtype == torch.float16 else 0.0
    return o, u * np.abs(o) + (1.02 * u + 1e-5) * ao + small + 1e-30, x, (2.0 ** -16 + 1e-5) * ax + 1e-30


def check_outputs(q, k, v, decay, scale, s0, o, last):
    want, eo, x, ex = bounded(q.dtype, f64(q), f64(k), f64(v), f64(decay), 1, None if s0 is None else f64(s0), 1.0, scale)
    assert np.abs(want).max() < 6e4                                  # the outputs themselves are inside float16
    assert_within(o, want, eo, "o")
    if last is not None:
        assert_within(last, x, ex, "final state")


def check_gradients(q, k, v, decay, scale, s0, d_o, d_last, got):
    dtype, none = q.dtype, lambda x: None if x is None else f64(x)
    q, k, v, d_o, decay, s0, d_last = f64(q), f64(k), f64(v), f64(d_o), f64(decay), none(s0), none(d_last)
    dq, eq, _, _ = bounded(dtype, d_o, v, k, decay, 1, transpose(s0), 1.0, scale)
    dv, ev, d0, e0 = bounded(dtype, k, q, d_o, decay, 0, d_last, scale, 1.0)
    dk, ek, _, _ = bounded(dtype, v, d_o, q, decay, 0, transpose(d_last), scale, 1.0)
    assert max(np.abs(x).max() for x in (dq, dk, dv)) < 6e4
    for name, x, want, e in zip(("dq", "dk", "dv", "d_initial_state"), got, (dq, dk, dv, d0), (eq, ek, ev, e0)):
        if x is not None:
            assert_within(x, want, e, name)


@each
def test_scores_above_the_type(shape, dtype):
    """Products of a hundred features leave float16, what they weigh does not."""
    b, t, h, dk, dv = shape
    _, _, v, _, decay, _, _ = draw(5 + t, b, t, h, dk, dv, dtype)
    q, k = ((60 + 60 * torch.rand((b, t, h, dk), device="cuda")).to(dtype) for _ in range(2))
    v = (v.float() * 1e-3).to(dtype)
    decay.fill_(-0.05)
    scale = 1.0 if dk < 100 else dk ** -0.5
    assert (q.float() * k.float()).sum(-1).max() * scale > 65504
    o, last = api.linear_attention(q, k, v, decay, scale=scale, output_final_state=True)
    check_outputs(q, k, v, decay, scale, None, o, last)


@pytest.mark.parametrize("size", [1e-5, 1e-6])
@each
def test_small_gradients(shape, dtype, size):
    """Gradients of outputs as a mean over many tokens leaves them, times large keys and values."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, _, _ = draw(6 + t, b, t, h, dk, dv, dtype)
    q, k = ((x.float() * 100).to(dtype) for x in (q, k))
    d_o = (d_o.float() * size).to(dtype)
    check_gradients(q, k, v, decay, dk ** -0.5, None, d_o, None, api.linear_attention_backward(d_o, q, k, v, decay))


@each
def test_gradients_of_large_scores(shape, dtype):
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, s0, d_last = draw(4 + t, b, t, h, dk, dv, dtype, True)
    q, k = ((x.float() * 1e-3).to(dtype) for x in (q, k))
    v, d_o = ((60 + 60 * torch.rand((b, t, h, dv), device="cuda")).to(dtype) for _ in range(2))
    decay.fill_(-0.05)
    assert (v.float() * d_o.float()).sum(-1).max() > 65504
    check_gradients(q, k, v, decay, 1.0, s0, d_o, d_last, api.linear_attention_backward(d_o, q, k, v, decay, 1.0, s0, d_final_state=d_last))


@each
def test_tokens_of_very_different_size(shape, dtype):
    """Queries over thirty binary orders of magnitude in one group: every token has a power of two of its own."""
    b, t, h, dk, dv = shape
    q, k, v, _, decay, _, _ = draw(7 + t, b, t, h, dk, dv, dtype)
    q = (q.float() * torch.exp2(-12.0 * torch.rand((b, t, h, 1), device="cuda"))).to(dtype)
    q[:, ::7] *= 1000
    k, v = (k.float() * 50).to(dtype), (v.float() * 1e-3).to(dtype)
    o, last = api.linear_attention(q, k, v, decay, scale=1.0, output_final_state=True)
    check_outputs(q, k, v, decay, 1.0, None, o, last)


@pytest.mark.parametrize("size", [1e9, 1e15])
@each
def test_groups_without_keys_keep_a_large_state(shape, dtype, size):
    """Masked tokens: keys of zero, whole groups of them, with states far above them in either direction.  (Gradients of 1e15
    would not be inside float16.)"""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, s0, d_last = draw(9 + t, b, t, h, dk, dv, dtype, True)
    decay.fill_(-1e-3)
    s0, d_last = s0 * size, d_last * size
    for x in (q, k, d_o):
        x[:, 128:256] = 0
    for keys in (k, torch.zeros_like(k)):
        o, last = api.linear_attention(q, keys, v, decay, scale=1 / size, initial_state=s0, output_final_state=True)
        check_outputs(q, keys, v, decay, 1 / size, s0, o, last)
    if size == 1e9:
        k, v = ((x.float() * 1e-6).to(dtype) for x in (k, v))
        got = api.linear_attention_backward(d_o, q, k, v, decay, 1 / size, s0, d_final_state=d_last)
        check_gradients(q, k, v, decay, 1 / size, s0, d_o, d_last, got)


@each
def test_keys_of_every_size(shape, dtype):
    """Groups of large, ordinary, tiny and no keys, one after another: the power of two that goes with a group changes by more than a
    factor of float32's smallest number, and back."""
    b, t, h, dk, dv = shape
    q, k, v, _, decay, s0, _ = draw(10 + t, b, t, h, dk, dv, dtype, True)
    decay.fill_(-1e-4)
    size = torch.ones(t, device="cuda")
    for i in range(0, t, 128):
        size[i:i + 128] = (1.0, 1e-6, 0.0, 1e3)[i // 128 % 4]
    k = (k.float() * size[None, :, None, None]).to(dtype)
    for scale in (1e-3, 2.0 ** -60):
        q2 = (q.float() * (1.0 if scale == 1e-3 else 1e4)).to(dtype)
        o, last = api.linear_attention(q2, k, v, decay, scale=scale, initial_state=s0, output_final_state=True)
        check_outputs(q2, k, v, decay, scale, s0, o, last)
    d_o, d_last = v, torch.zeros_like(s0)                            # (here queries and scale are the keys of two of the walks)
    got = api.linear_attention_backward(d_o, k, q, v, decay, 2.0 ** -50, None, d_final_state=d_last)
    check_gradients(k, q, v, decay, 2.0 ** -50, None, d_o, d_last, got)


@each
def test_a_decay_that_is_no_number(shape, dtype):
    """A model that has gone wrong shows it, in prompts and gradients as in single tokens; other heads keep their bits."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, s0, d_last = draw(8 + t, b, t, max(h, 2), dk, dv, dtype, True)

    def all_of(decay, s0=s0, d_last=d_last):
        o, last = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
        dq, dk, dv, d_first = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last)
        state = torch.zeros_like(last) if s0 is None else s0.clone()
        step = api.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state)
        return [o.transpose(1, 2), last, dq.transpose(1, 2), dk.transpose(1, 2), dv.transpose(1, 2), state, step] + ([] if d_first is None else [d_first])

    for states in ((s0, d_last), (None, None)):
        want = all_of(decay, *states)
        for head in (0, q.shape[2] - 1):
            bad = decay.clone()
            bad[head] = float("nan")
            others = torch.arange(len(decay), device="cuda") != head
            for x, w in zip(all_of(bad, *states), want):
                assert torch.isnan(x[:, head]).all()
                assert torch.equal(x[:, others], w[:, others])
