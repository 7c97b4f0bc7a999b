"""Linear attention with a decay for each head: outputs, states and gradients against the 64-bit definition and against
differences of it, over lengths, widths, layouts, decays and types; single tokens; streams and graphs."""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.lm_reference import assert_within, bounded_mix, f64, gradients, mix

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert api.linear_attention_status() == 0


def draw(seed, b, t, h, dk, dv, dtype, states=False, tail=()):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    q, k = (torch.nn.functional.silu(n(b, t, h, dk)).to(dtype) for _ in range(2))
    v, d_o = (n(b, t, h, dv).to(dtype) for _ in range(2))
    decay = -torch.exp2(-8.0 * (torch.arange(h, device="cuda") + 1.0) / h)
    s0, d_last = (n(b, h, dk, dv) if states else None for _ in range(2))
    return q, k, v, d_o, decay, s0, d_last


def check_forward(q, k, v, decay, scale, s0, o, last):
    want, eo, x, ex = bounded_mix(q.dtype, f64(q), f64(k), f64(v), f64(decay), 1, None if s0 is None else f64(s0), 1.0, scale)
    assert_within(o, want, eo, "o")
    if last is not None:
        assert_within(last, x, ex, "final state")


def check_backward(q, k, v, decay, scale, s0, d_o, d_last, got):
    none = lambda x: None if x is None else f64(x)  # noqa: E731
    want = gradients(q.dtype, f64(q), f64(k), f64(v), f64(decay), scale, none(s0), f64(d_o), none(d_last))
    for name, x, (w, e) in zip(("dq", "dk", "dv", "d_initial_state"), got, want):
        if x is not None:
            assert_within(x, w, e, name)


SHAPES = [  # b, t, h, dk, dv
    (1, 1, 1, 64, 64), (2, 2, 3, 128, 128), (1, 127, 2, 64, 64), (2, 128, 2, 128, 128), (1, 129, 3, 64, 128),
    (1, 257, 2, 128, 64), (2, 640, 2, 128, 128), (1, 700, 4, 64, 64), (1, 200, 2, 40, 72), (3, 131, 1, 8, 128),
    (1, 150, 2, 20, 36), (1, 140, 2, 1, 1), (1, 300, 1, 96, 120), (1, 2100, 1, 128, 128), (1, 1500, 2, 64, 64),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("states", [False, True], ids=["plain", "states"])
def test_against_the_definition(shape, dtype, states):
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, s0, d_last = draw(t + dk, b, t, h, dk, dv, dtype, states)
    scale = dk ** -0.5
    o, last = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
    assert o.is_contiguous() and o.dtype == dtype
    check_forward(q, k, v, decay, scale, s0, o, last)
    check_backward(q, k, v, decay, scale, s0, d_o, d_last, api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last))
    assert torch.equal(o, api.linear_attention(q, k, v, decay, initial_state=s0)[0])        # the same bits again, without the state


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 2040, 2, 24, 40), (1, 2040, 1, 128, 72), (1, 3200, 3, 32, 32), (1, 4300, 16, 16, 24), (2, 1300, 11, 16, 16)], ids=str)
def test_walks_split_over_blocks(shape, dtype):
    """Few heads of many tokens: parts of a walk start from the states of the parts before them, in either direction."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, s0, d_last = draw(t + h, b, t, h, dk, dv, dtype, True)
    decay[0] = -1e-3
    scale = dk ** -0.5
    o, last = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
    check_forward(q, k, v, decay, scale, s0, o, last)
    check_backward(q, k, v, decay, scale, s0, d_o, d_last, api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last))


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
def test_decays_at_their_ends(dtype):
    """No decay, a decay of a few tokens, one that underflows inside a group of tokens, and no memory at all."""
    q, k, v, d_o, decay, s0, d_last = draw(5, 1, 300, 5, 64, 64, dtype, True)
    decay.copy_(torch.tensor([0.0, -0.5, -20.0, float("-inf"), -1e-4]))
    o, last = api.linear_attention(q, k, v, decay, scale=0.3, initial_state=s0, output_final_state=True)
    check_forward(q, k, v, decay, 0.3, s0, o, last)
    check_backward(q, k, v, decay, 0.3, s0, d_o, d_last, api.linear_attention_backward(d_o, q, k, v, decay, 0.3, s0, d_final_state=d_last))


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
def test_large_states(dtype):
    """Without decay the state outgrows float16's range; the outputs, scaled down, do not."""
    b, t, h, d = 1, 1500, 1, 64
    g = torch.Generator(device="cuda").manual_seed(9)
    q = (torch.rand((b, t, h, d), generator=g, device="cuda") * 0.1).to(dtype)
    k = (torch.rand((b, t, h, d), generator=g, device="cuda") * 20).to(dtype)
    v = (torch.rand((b, t, h, d), generator=g, device="cuda") * 20).to(dtype)
    decay = torch.zeros(h, device="cuda")
    o, last = api.linear_attention(q, k, v, decay, scale=1e-3, output_final_state=True)
    assert last.max() > 1e5
    check_forward(q, k, v, decay, 1e-3, None, o, last)


@pytest.mark.parametrize("t,d", [(140, 64), (300, 128)])
def test_gradients_against_differences(t, d):
    """The loss is linear in each of q, k, v and the first state alone: a difference of the 64-bit definition is exact."""
    q, k, v, d_o, decay, s0, d_last = draw(31 + t, 1, t, 2, d, d, torch.float16, True)
    scale = d ** -0.5
    got = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last)
    x = [f64(y) for y in (q, k, v, s0)]
    bounds = [e for _, e in gradients(q.dtype, *x[:3], f64(decay), scale, x[3], f64(d_o), f64(d_last))]

    def loss(q, k, v, s0):
        o, last = mix(q, k, v, f64(decay), 1, s0, 1.0, scale)
        return (o * f64(d_o)).sum() + (last * f64(d_last)).sum()

    rng = np.random.default_rng(t)
    for which, name in enumerate(("dq", "dk", "dv", "d_initial_state")):
        for _ in range(6):
            at = tuple(int(rng.integers(n)) for n in x[which].shape)
            hi, lo = ([y.copy() for y in x] for _ in range(2))
            hi[which][at] += 0.5
            lo[which][at] -= 0.5
            want = loss(*hi) - loss(*lo)
            assert abs(f64(got[which])[at] - want) <= bounds[which][at] + 1e-9 * abs(want), (name, at)


def test_autograd_gives_the_same_gradients():
    q, k, v, d_o, decay, s0, d_last = draw(41, 2, 200, 2, 64, 64, torch.bfloat16, True)
    want = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last)
    leaves = [x.clone().requires_grad_() for x in (q, k, v, s0)]
    o, last = api.linear_attention(*leaves[:3], decay, initial_state=leaves[3], output_final_state=True)
    torch.autograd.backward([o, last], [d_o, d_last])
    for x, w in zip(leaves, want):
        assert torch.equal(x.grad, w)
    # one head of keys shared by all: its gradient is the sum over the heads
    one = k[:, :, :1].clone().requires_grad_()
    api.linear_attention(q, one.expand_as(k), v, decay)[0].backward(d_o)
    parts = api.linear_attention_backward(d_o, q, one.detach().expand_as(k), v, decay)[1]
    assert_within(one.grad, f64(parts.float().sum(2, keepdim=True)), 2.0 ** -8 * np.abs(f64(parts)).sum(2, keepdims=True) * 2 + 1e-30, "shared key")
    # a loss that only uses the sum of the outputs hands in a gradient of strides 0
    q2 = q.clone().requires_grad_()
    api.linear_attention(q2, k, v, decay)[0].sum().backward()
    assert torch.equal(q2.grad, api.linear_attention_backward(torch.ones_like(v), q, k, v, decay)[0])


@pytest.mark.parametrize("t", [100, 300])
def test_layouts(t):
    """Heads before tokens, one buffer for all three, a head repeated by a stride of 0, rows off 16-byte boundaries: the
    same bits as from dense arrays."""
    q, k, v, d_o, decay, _, _ = draw(51, 2, t, 3, 64, 64, torch.bfloat16)
    want, grads = api.linear_attention(q, k, v, decay)[0], api.linear_attention_backward(d_o, q, k, v, decay)

    def same(q, k, v, d_o, want=want, grads=grads):
        assert torch.equal(api.linear_attention(q, k, v, decay)[0], want)
        for x, w in zip(api.linear_attention_backward(d_o, q, k, v, decay)[:3], grads):
            assert torch.equal(x, w)

    by_head = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, d_o)]
    same(*by_head)
    joined = torch.cat([q, k, v], -1)
    same(joined[..., :64], joined[..., 64:128], joined[..., 128:], d_o)
    shifted = torch.empty(q.numel() + 1, dtype=q.dtype, device="cuda")[1:].view(q.shape).copy_(q)
    same(shifted, k, v, d_o)
    wide = torch.zeros(*q.shape[:3], 67, dtype=q.dtype, device="cuda")
    wide[..., :64] = k
    same(q, wide[..., :64], v, d_o)
    shared = q[:, :, :1].expand_as(q)
    same(shared, k, v, d_o, api.linear_attention(shared.contiguous(), k, v, decay)[0], api.linear_attention_backward(d_o, shared.contiguous(), k, v, decay))
    first = k[:1].expand_as(k)
    same(q, first, v, d_o, api.linear_attention(q, first.contiguous(), v, decay)[0], api.linear_attention_backward(d_o, q, first.contiguous(), v, decay))


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 96)])
def test_packed(dtype, dk, dv):
    """Sequences of every kind of length, each as if it were alone; an empty one keeps its state; what one sequence holds -
    not even a NaN - never reaches another."""
    lens = [0, 1, 128, 37, 0, 129, 300, 1, 255]
    off = np.concatenate([[0], np.cumsum(lens)])
    q, k, v, d_o, decay, _, _ = draw(61, 1, int(off[-1]), 2, dk, dv, dtype)
    q, k, v, d_o = (x[0] for x in (q, k, v, d_o))
    g = torch.Generator(device="cuda").manual_seed(1)
    s0, d_last = (torch.randn((len(lens), 2, dk, dv), generator=g, device="cuda") for _ in range(2))
    offsets = torch.from_numpy(off).cuda()
    bad = [3, 7]                                   # sequences that hold nothing finite
    for i in bad:
        for x in (q, k, v, d_o):
            x[off[i]:off[i + 1]] = float("nan")
            x[off[i]:off[i] + 1] = float("inf")
    o, last = api.linear_attention(q, k, v, decay, initial_state=s0, offsets=offsets, output_final_state=True)
    grads = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, offsets=offsets, d_final_state=d_last)
    for i in range(len(lens)):
        if i in bad:
            continue
        part = lambda x: x[off[i]:off[i + 1]][None]  # noqa: E731
        check_forward(part(q), part(k), part(v), decay, dk ** -0.5, s0[i:i + 1], part(o), last[i:i + 1])
        check_backward(part(q), part(k), part(v), decay, dk ** -0.5, s0[i:i + 1], part(d_o), d_last[i:i + 1],
                       [part(x) for x in grads[:3]] + [grads[3][i:i + 1]])


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("shape", [(2, 300, 80, 16, 24), (1, 700, 150, 32, 16), (1, 520, 60, 24, 72), (5, 130, 31, 8, 128), (1, 100, 149, 16, 16)], ids=str)
@pytest.mark.parametrize("states", [False, True], ids=["plain", "states"])
def test_more_walks_than_multiprocessors(shape, dtype, states):
    """Walks are cut where a multiprocessor's share of them ends, and the state is handed over; states in place as well."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, s0, d_last = draw(t + h, b, t, h, dk, dv, dtype, states)
    decay[: h // 2] = -1e-3 * (1 + torch.arange(h // 2, device="cuda"))
    scale = dk ** -0.5
    o, last = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
    check_forward(q, k, v, decay, scale, s0, o, last)
    check_backward(q, k, v, decay, scale, s0, d_o, d_last, api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last))
    assert torch.equal(o, api.linear_attention(q, k, v, decay, initial_state=s0)[0])


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_packed_and_more_walks_than_multiprocessors(dtype, seed):
    """One walk over many blocks, whole blocks of empty sequences, several short walks to a block; more than 32 sequences."""
    rng = np.random.default_rng(seed)
    h, dk, dv = 5, 24, 16
    lens = [int(n) for n in rng.choice([0, 1, 3, 40, 128, 129, 300], 45)]
    lens[[0, 22, 44][seed]] = 2500
    lens[5:9] = [0] * 4
    off = np.concatenate([[0], np.cumsum(lens)])
    q, k, v, d_o, decay, _, _ = draw(71 + seed, 1, int(off[-1]), h, dk, dv, dtype)
    q, k, v, d_o = (x[0] for x in (q, k, v, d_o))
    decay[0] = -1e-3
    g = torch.Generator(device="cuda").manual_seed(seed)
    s0, d_last = (torch.randn((len(lens), h, dk, dv), generator=g, device="cuda") for _ in range(2))
    offsets = torch.from_numpy(off).cuda()
    o, last = api.linear_attention(q, k, v, decay, initial_state=s0, offsets=offsets, output_final_state=True)
    grads = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, offsets=offsets, d_final_state=d_last)
    for i in range(len(lens)):
        part = lambda x: x[off[i]:off[i + 1]][None]  # noqa: E731
        check_forward(part(q), part(k), part(v), decay, dk ** -0.5, s0[i:i + 1], part(o), last[i:i + 1])
        check_backward(part(q), part(k), part(v), decay, dk ** -0.5, s0[i:i + 1], part(d_o), d_last[i:i + 1],
                       [part(x) for x in grads[:3]] + [grads[3][i:i + 1]])


def test_cut_walks_on_two_streams_and_in_a_graph():
    q, k, v, _, decay, s0, _ = draw(91, 2, 700, 80, 32, 64, torch.bfloat16, True)
    want = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
    torch.cuda.synchronize()
    sides, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for _ in range(5):
        for side in sides:                              # each call has scratch memory of its own
            with torch.cuda.stream(side):
                got.append(api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got.append(api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for one in got for a, b in zip(one, want))


def test_scratch_sizes_and_refusals():
    """Scratch memory is asked for where many walks leave a last wave short of blocks, and has to be as large as asked for."""
    from paper_2411_17887_b200 import binding as B

    def args(b, t, h, **more):
        at = lambda i: (i << 28, t * h * 64, h * 64, 64)  # noqa: E731
        return B.tcu_linattn_args(B.TCU_BF16, b, t, h, 64, 64, 1.0, 9 << 28, at(1), at(2), at(3), at(4), d_o=at(5), d_q=at(6), d_k=at(7), d_v=at(8), **more)

    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert B.tcu_linattn_scratch_bytes(args(1, 4096, sms), 0) == 0                        # one wave, full
    assert B.tcu_linattn_scratch_bytes(args(1, 4096, sms + 9, d_offsets=10 << 28), 0) == 0
    size = B.tcu_linattn_scratch_bytes(args(1, 4096, sms + 9), 0)
    assert size >= sms * (64 * 64 * 4 + 4)
    assert B.tcu_linattn_scratch_bytes(args(1, 4096, sms // 3 + 3), 1) == size
    buf = torch.empty(256, dtype=torch.uint8, device="cuda").zero_()
    for where, n in ((11 << 28, size - 1), ((11 << 28) + 16, size)):
        assert B.tcu_linattn_forward(args(1, 4096, sms + 9, d_scratch=where, scratch_bytes=n), buf, 256) == B.TCU_ERR_WORKSPACE


def test_empty_calls():
    decay = torch.zeros(2, device="cuda")
    empty = torch.empty((0, 5, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert api.linear_attention(empty, empty, empty, decay)[0].shape == empty.shape
    none = torch.empty((3, 0, 2, 64), dtype=torch.bfloat16, device="cuda")
    s0 = torch.randn((3, 2, 64, 64), device="cuda")
    o, last = api.linear_attention(none, none, none, decay, initial_state=s0, output_final_state=True)
    assert o.shape == none.shape and torch.equal(last, s0)
    assert torch.equal(api.linear_attention_backward(none, none, none, none, decay, initial_state=s0, d_final_state=s0)[3], s0)


def test_prompt_in_parts_with_the_state_in_place():
    """A prompt taken in two calls, the second continuing from the state of the first."""
    q, k, v, _, decay, _, _ = draw(71, 2, 500, 2, 128, 128, torch.bfloat16)
    _, middle = api.linear_attention(q[:, :333], k[:, :333], v[:, :333], decay, output_final_state=True)
    o, last = api.linear_attention(q[:, 333:], k[:, 333:], v[:, 333:], decay, initial_state=middle, output_final_state=True)
    want, eo, x, ex = bounded_mix(q.dtype, f64(q), f64(k), f64(v), f64(decay), 1, None, 1.0, 128 ** -0.5)
    assert_within(o, want[:, 333:], eo[:, 333:], "o")
    assert_within(last, x, 2 * ex, "final state")


# ---- single tokens: everything in 32 bits, so the bounds are those of 32-bit sums of dk terms and one rounding
@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("b,h,dk,dv", [(1, 1, 64, 64), (3, 2, 128, 128), (5, 3, 40, 72), (2, 2, 20, 36), (2, 1, 7, 5), (4, 1, 128, 1), (1, 2, 1, 128)])
def test_single_tokens(b, h, dk, dv, dtype):
    q, k, v, _, decay, _, _ = draw(81 + dv, b, 1, h, dk, dv, dtype)
    q, k, v = q[:, 0], k[:, 0], v[:, 0]
    pool = torch.randn((b + 2, h, dk, dv), device="cuda")
    slots = torch.randperm(b + 2, device="cuda")[:b].to(torch.int32)
    before, state = f64(pool), pool.clone()
    o = api.linear_attention_step(q, k, v, decay, state, scale=0.4, slots=slots)
    want = before.copy()
    at = slots.cpu().numpy()
    a = np.exp(f64(decay))[None, :, None, None]
    want[at] = a * before[at] + f64(k)[..., :, None] * f64(v)[..., None, :]
    size = np.abs(a * before[at]) + np.abs(f64(k)[..., :, None] * f64(v)[..., None, :])
    bound = np.zeros_like(want)
    bound[at] = 4 * 2.0 ** -24 * size
    assert_within(state, want, bound, "state")
    total = 0.4 * np.einsum("bhk,bhkv->bhv", f64(q), want[at])
    asum = 0.4 * np.einsum("bhk,bhkv->bhv", np.abs(f64(q)), size)
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    assert_within(o, total, u * np.abs(total) + (dk + 8) * 2.0 ** -24 * asum + (2.0 ** -25 if dtype == torch.float16 else 0.0) + 1e-30, "o")


def test_single_tokens_skip_and_stride():
    """Entries outside the pool are skipped; strided inputs; without slots sequence b has entry b."""
    b, h, d = 4, 2, 64
    q, k, v, _, decay, _, _ = draw(91, b, 1, h, d, d, torch.bfloat16)
    joined = torch.cat([q, k, v], -1)[:, 0]
    q, k, v = (joined[..., i * d:(i + 1) * d] for i in range(3))
    state = torch.randn((b, h, d, d), device="cuda")
    want = state.clone()
    ow = api.linear_attention_step(q.contiguous(), k.contiguous(), v.contiguous(), decay, want)
    got = state.clone()
    assert torch.equal(api.linear_attention_step(q, k, v, decay, got), ow) and torch.equal(got, want)
    got = state.clone()
    slots = torch.tensor([0, -1, 2, b], dtype=torch.int32, device="cuda")
    o = api.linear_attention_step(q, k, v, decay, got, slots=slots)
    for i, ok in enumerate([True, False, True, False]):
        assert torch.equal(got[i], want[i] if ok else state[i])
        assert torch.equal(o[i], ow[i] if ok else torch.zeros_like(o[i]))


def test_tokens_one_by_one_match_the_prompt():
    b, t, h, d = 2, 150, 2, 64
    q, k, v, _, decay, _, _ = draw(101, b, t, h, d, d, torch.bfloat16)
    o, last = api.linear_attention(q, k, v, decay, output_final_state=True)
    state = torch.zeros((b, h, d, d), device="cuda")
    steps = torch.stack([api.linear_attention_step(q[:, i], k[:, i], v[:, i], decay, state) for i in range(t)], 1)
    want, eo, x, ex = bounded_mix(q.dtype, f64(q), f64(k), f64(v), f64(decay), 1, None, 1.0, d ** -0.5)
    assert_within(steps, want, eo, "steps")
    assert_within(o, want, eo, "prompt")
    assert_within(state, x, ex, "state of the steps")
    assert_within(last, x, ex, "state of the prompt")


def test_side_stream_and_graph():
    q, k, v, d_o, decay, s0, d_last = draw(111, 1, 300, 2, 128, 128, torch.bfloat16, True)
    want = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
    grads = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = q * 0
        torch.cuda._sleep(2_000_000)
        late += q                                   # ready only after the wait: a call on another stream would read zeros
        got = api.linear_attention(late, k, v, decay, initial_state=s0, output_final_state=True)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    state = torch.zeros((1, 2, 128, 128), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, last = api.linear_attention(q, k, v, decay, initial_state=s0, output_final_state=True)
        back = api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0, d_final_state=d_last)
        api.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(last, want[1])
    for x, w in zip(back, grads):
        assert torch.equal(x, w)
    again = torch.zeros_like(state)
    for _ in range(2):
        api.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, again)
    assert torch.equal(state, again)
