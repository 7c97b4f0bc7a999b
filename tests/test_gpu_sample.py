"""Sampling: tokens equal to the definition's in 64 bits, log probabilities to 32, over vocabularies, types, settings, ties, masked tokens, strides."""
import math

import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.lm_reference import f64
from tests.sample_reference import token_of

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def draw(rows, v, dtype, seed=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((rows, v), generator=g, device="cuda") * spread).to(dtype), torch.rand(rows, generator=g, device="cuda")


def check(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    tokens, log_probs = api.sample(logits, u, temperature, top_k, top_p, min_p, output_log_prob=True)
    assert tokens.dtype == torch.int64 and log_probs.dtype == torch.float32
    rows = logits.shape[0]
    settings = [f64(s) if isinstance(s, torch.Tensor) else np.full(rows, float(s)) for s in (temperature, top_k, top_p, min_p)]
    x, at = f64(logits), f64(u)
    for r in range(rows):
        token, log_prob = token_of(x[r], at[r], *(s[r] for s in settings))
        assert int(tokens[r]) == token, (r, int(tokens[r]), token, [s[r] for s in settings])
        got = float(log_probs[r])
        # rounded to 32 bits once; sums are 64 bits
        assert got == log_prob or abs(got - log_prob) <= 2.0 ** -24 * abs(log_prob) + 1e-10, (r, got, log_prob)
    assert torch.equal(tokens, api.sample(logits, u, temperature, top_k, top_p, min_p))


RULES = {"whole": {}, "warm": dict(temperature=1.7), "cold": dict(temperature=0.1), "greedy": dict(temperature=0.0), "k": dict(top_k=40), "k1": dict(top_k=1), "p": dict(top_p=0.9),
         "p_small": dict(top_p=0.05), "min_p": dict(min_p=0.03), "k_p": dict(top_k=100, top_p=0.8, temperature=0.9), "k_m": dict(top_k=20, min_p=0.1), "p_m": dict(top_p=0.95, min_p=0.01),
         "all": dict(top_k=300, top_p=0.97, min_p=0.005, temperature=1.3), "p0": dict(top_p=0.0), "m2": dict(min_p=2.0), "k_big": dict(top_k=10 ** 9)}


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("rows,v", [(3, 1), (5, 2), (40, 33), (20, 1000), (6, 4097), (200, 5003), (3, 50001)])
def test_rules(rows, v, rule, dtype):
    check(*draw(rows, v, dtype, rows + v), **RULES[rule])


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,v", [(2, 131071), (1, 262144), (3, 262143), (300, 16385), (149, 2049)])
def test_large(rows, v, dtype):
    logits, u = draw(rows, v, dtype, v)
    for rule in ("whole", "p", "all"):
        check(logits, u, **RULES[rule])


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("spread", [0.0, 1e-3, 30.0, 3000.0])
def test_flat_and_steep(spread, dtype):
    """All logits alike, nearly alike, and far apart: the whole of the row in one bin of the first histogram, or nearly all in the last."""
    logits, u = draw(8, 3001, dtype, 5, spread)
    for rule in RULES:
        check(logits, u, **RULES[rule])
    check(logits, u, top_k=2500, top_p=0.999)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
def test_ties(dtype):
    """Few different logits: top_k and top_p end within tokens that are equal, of which the lower ones are kept."""
    logits, u = draw(60, 4000, dtype, 6)
    logits = logits.round()
    for rule in ("k", "p", "k_p", "all", "min_p", "greedy", "p_small"):
        check(logits, u, **RULES[rule])
    check(logits, u, top_k=1500, top_p=0.5)
    check(torch.where(logits > 0, 0.0, -0.0).to(dtype), u, top_k=77)                     # a zero is a zero
    # equal weights: every border is exact
    flat = torch.zeros((5, 1000), device="cuda", dtype=dtype)
    at = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24], device="cuda")
    assert api.sample(flat, at).tolist() == [0, 250, 500, 750, 999]
    assert api.sample(flat, at, top_p=0.5).tolist() == [0, 125, 250, 375, 499]
    assert api.sample(flat, at, top_k=8).tolist() == [0, 2, 4, 6, 7]
    assert api.sample(flat, at, top_k=8, top_p=0.5).tolist() == [0, 1, 2, 3, 3]


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
def test_settings_of_each_row(dtype):
    logits, u = draw(120, 2500, dtype, 7)
    g = torch.Generator(device="cuda").manual_seed(1)
    some = lambda: torch.rand(120, generator=g, device="cuda")  # noqa: E731
    temperature = torch.where(some() < 0.2, 0.0, 0.5 + some())
    top_k = torch.where(some() < 0.5, torch.randint(-1, 300, (120,), generator=g, device="cuda"), 0).to(torch.int32)
    top_p = torch.where(some() < 0.5, some(), 1.0)
    min_p = torch.where(some() < 0.5, 0.2 * some(), 0.0)
    check(logits, u, temperature, top_k, top_p, min_p)
    check(logits, u.double(), temperature, 50, top_p)
    check(logits, u, 0.8, top_k, 1.0, min_p)
    nan = torch.full((120,), float("nan"), device="cuda")
    assert torch.equal(api.sample(logits, u, 1.0, 0, nan, nan), api.sample(logits, u))     # no number, no limit
    assert torch.equal(api.sample(logits, u, nan), logits.float().argmax(1))
    assert torch.equal(api.sample(logits, u, -torch.ones_like(nan)), logits.float().argmax(1))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
def test_masked_tokens(dtype):
    logits, u = draw(50, 3000, dtype, 8)
    g = torch.Generator(device="cuda").manual_seed(2)
    logits[torch.rand(logits.shape, generator=g, device="cuda") < 0.7] = -math.inf
    logits[3] = -math.inf
    logits[4, 1:] = -math.inf
    logits[5, :-1] = -math.inf
    logits[6] = torch.finfo(dtype).min                                                    # masked by the lowest value: all alike
    logits[7, 100:] = torch.finfo(dtype).min
    logits[8, ::3] = math.nan
    logits[9] = math.nan
    logits[10, 1000:] = math.nan
    logits[11, [5, 700, 2999]] = math.inf
    logits[12, 17] = math.inf
    logits[12, 18:] = math.nan
    for rule in RULES:
        check(logits, u, **RULES[rule])
    assert api.sample(logits, u)[[3, 9]].tolist() == [-1, -1]


def test_random_numbers_at_their_ends():
    logits, _ = draw(6, 700, torch.float32, 9)
    logits[:, -3:] = -math.inf
    logits[:, 0] = -200.0                                                                 # a weight of 1e-88
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, -1.0, math.nan], device="cuda")
    tokens = api.sample(logits, u).tolist()
    assert tokens == [0, 696, 696, 696, 0, 0]
    assert api.sample(logits, u.double(), top_k=1).tolist() == logits.argmax(1).tolist()


def test_temperatures_at_their_ends():
    """So hot that all tokens are alike, so cold that only those with the largest logit are left; infinite ones from memory."""
    logits, u = draw(20, 900, torch.float32, 11)
    logits[:, ::7] = -math.inf
    logits[:, 5] = logits[:, 700] = logits.amax(1) + 1.0
    allowed = (logits > -math.inf).nonzero()[:, 1].view(20, -1)
    for hot in (torch.full((20,), math.inf, device="cuda"), 1e299, torch.full((20,), 3e38, device="cuda")):
        for limits in ({}, dict(top_k=allowed.shape[1])):
            tokens = api.sample(logits, u, hot, **limits)
            at = torch.floor(u.double() * allowed.shape[1]).long()
            assert torch.equal(tokens, allowed.gather(1, at[:, None])[:, 0])
        assert torch.isin(api.sample(logits, u, hot, top_p=0.5), allowed).all()
    for cold in (1e-320, 1e-300, torch.full((20,), 1e-45, device="cuda"), 1e-20):
        for limits in ({}, dict(top_k=100), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=700, top_p=0.99)):
            tokens = api.sample(logits, u, cold, **limits)
            assert torch.equal(tokens, torch.where(u < 0.5, 5, 700)), (cold, limits)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("limits", [dict(top_k=150), dict(top_k=400), dict(top_k=3000), dict(top_k=3000, top_p=0.7), dict(top_p=0.995), dict(top_k=2000, min_p=1e-4),
                                    dict(min_p=1e-5, top_p=0.99)], ids=str)
def test_many_kept(limits, dtype):
    """More tokens than are listed: histograms, with few and with many tokens in the bin that they name."""
    for rows, v, spread in ((6, 30011, 1.0), (160, 9000, 2.0), (3, 200001, 0.5)):
        logits, u = draw(rows, v, dtype, v, spread)
        check(logits, u, 1.1, **limits)
    check(logits.round(), u, 1.1, **limits)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
def test_strides(dtype):
    wide, u = draw(20, 2100, dtype, 10)
    for logits in (wide[:, :2001], wide[:, 1:2000], wide[:, 3:1502], wide[::2, 7:2100], wide[:1, 5:905].expand(20, 900), wide[:, :300].t().contiguous().t(), wide[:, :1]):
        check(logits, u[:logits.shape[0]], top_p=0.9)
        check(logits, u[:logits.shape[0]])


def test_no_rows_and_refusals():
    assert api.sample(torch.empty((0, 10), device="cuda"), torch.empty(0, device="cuda")).shape == (0,)
    logits, u = draw(3, 10, torch.float32)
    with pytest.raises(RuntimeError, match="no_grad"):
        api.sample(logits.clone().requires_grad_(), u)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            api.sample(torch.autograd.forward_ad.make_dual(logits, logits), u)
    with pytest.raises(RuntimeError):
        api.sample(torch.zeros((1, (1 << 18) + 1), device="cuda"), u[:1])


def test_graph_and_streams():
    sets = [draw(70, 9001, torch.bfloat16, s) for s in range(3)]
    call = lambda logits, u: api.sample(logits, u, 0.8, 60, 0.9, 0.001, output_log_prob=True)  # noqa: E731
    want = [call(*s) for s in sets]
    held = [z.clone() for z in sets[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = call(*held)
    for k in (1, 2, 0):
        for z, new in zip(held, sets[k]):
            z.copy_(new)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[k]))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for stream, s in zip(streams, sets):
            with torch.cuda.stream(stream):
                got.append(call(*s))
    torch.cuda.synchronize()
    for k, outs in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(outs, want[k % 3]))
