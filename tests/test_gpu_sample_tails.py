"""Sampling where top_p ends far below the largest logit, among more tokens than are listed: the token is the definition's unless u or top_p lies within
1e-11 of the border between two, however light the tokens are."""
import math
from decimal import ROUND_CEILING, Decimal, localcontext

import numpy as np
import pytest
import torch

BORDER = 1e-11           # u and top_p are further than this from every border that they are compared with
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def one_peak(n, logit, top_p, peak):
    """One logit of 0 at place `peak`, n of `logit`: how many of the equal ones top_p keeps, and (u, token) for places among them, with fifty digits."""
    with localcontext() as context:
        context.prec = 50
        w, p = Decimal(logit).exp(), Decimal(top_p)
        border = (p * (1 + n * w) - 1) / w
        kept = int(border.to_integral_value(ROUND_CEILING))
        assert 0 < kept < n and min(kept - border, border - (kept - 1)) * w / (1 + n * w) > BORDER
        total, drawn = 1 + kept * w, []
        for j in (0, kept // 3, kept // 2, kept - 40, kept - 2, kept - 1):
            # the middle of tie j, in the order of tokens
            u = float(((j + Decimal("0.5")) * w + (1 if j >= peak else 0)) / total)
            drawn.append((u, j + (1 if j >= peak else 0), float(w.ln() - total.ln())))
            assert w / 2 / total - abs(Decimal(u) * total - ((j + Decimal("0.5")) * w + (1 if j >= peak else 0))) / total > BORDER
    return kept, drawn


# (equal tokens, their logit, top_p or the part of them that is kept, place of the peak)
PEAKS = [(262143, -18.42068, 0.9997385, 0), (262143, -16.118, 0.9974453, 0), (131071, -21.3, 0.99999, 0), (200000, -22.251, 0.99998, 0), (262143, -13.8, None, 100000),
         (262143, -18.4, None, 262143), (262143, -20.7, None, 5), (150001, -19.5, None, 0), (600, -15.0, None, 600), (1025, -9.0, None, 3)]


def peak_case(n, logit, top_p, peak, dtype):
    logit = float(torch.tensor(logit).to(dtype))
    if top_p is None:                                        # the middle of a tie
        w = math.exp(logit)
        top_p = (1.0 + (int(0.87 * n) - 0.5) * w) / (1.0 + n * w)
    return logit, top_p, one_peak(n, logit, top_p, peak)


# (a top_p that is given goes with a logit of 32 bits)
TYPED = [(case, dtype) for case in PEAKS for dtype in DTYPES if case[2] is None or dtype == "f32"]


@pytest.mark.parametrize("case,dtype", TYPED, ids=str)
def test_cases_lie_off_the_borders(case, dtype):
    peak_case(*case, DTYPES[dtype])


@pytest.mark.parametrize("seed", range(4))
def test_tails_lie_off_the_borders(seed):
    tail_case(seed)


@pytest.mark.gpu
@pytest.mark.parametrize("case,dtype", TYPED, ids=str)
def test_one_peak_above_equal_tokens(case, dtype):
    n, _, _, peak = case
    logit, top_p, (_, drawn) = peak_case(*case, DTYPES[dtype])
    row = torch.full((n + 1,), logit, device="cuda", dtype=DTYPES[dtype])
    row[peak] = 0.0
    u = torch.tensor([u for u, _, _ in drawn], device="cuda", dtype=torch.float64)
    from paper_2411_17887_b200 import api
    for rows in (row[None].expand(len(u), -1), row[None].expand(len(u), -1).contiguous()):
        tokens, log_probs = api.sample(rows, u, top_p=top_p, output_log_prob=True)
        assert tokens.tolist() == [token for _, token, _ in drawn]
        for got, (_, _, want) in zip(log_probs.tolist(), drawn):
            assert abs(got - want) <= 2.0 ** -24 * abs(want) + 1e-10              # rounded to 32 bits once; sums of 64 bits


def tail_case(seed):
    """A few large logits above a tail of different light ones: the row, top_p, and (u, token)."""
    rng = np.random.default_rng(seed)
    v = (30001, 100003, 262144, 131072)[seed]
    x = (-17.0 + (0.002, 0.05, 0.3, 0.001)[seed] * rng.standard_normal(v)).astype(np.float32)
    x[rng.integers(0, v, 3)] = (0.0, -0.5, -1.25)
    wide = np.longdouble
    order = np.lexsort((np.arange(v), -x))
    w = np.exp(x.astype(wide) - wide(x.max()))
    upto = np.cumsum(w[order])
    kept = int((0.3, 0.6, 0.9, 0.99)[seed] * v)
    top_p = float((upto[kept - 1] - w[order[kept - 1]] / 2) / upto[-1])
    assert min(upto[kept - 1] / upto[-1] - top_p, top_p - upto[kept - 2] / upto[-1]) > BORDER
    tokens = np.sort(order[:kept])
    upto = np.cumsum(w[tokens])
    drawn = []
    for j in (1, kept // 2, kept - 100, kept - 1):
        u = float((upto[j] - w[tokens[j]] / 2) / upto[-1])
        assert min(upto[j] / upto[-1] - u, u - upto[j - 1] / upto[-1]) > BORDER
        drawn.append((u, int(tokens[j])))
    return x, top_p, drawn


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(4))
def test_light_tails(seed):
    x, top_p, drawn = tail_case(seed)
    from paper_2411_17887_b200 import api
    rows = torch.from_numpy(x).cuda()[None].expand(len(drawn), -1)
    u = torch.tensor([u for u, _ in drawn], device="cuda", dtype=torch.float64)
    assert api.sample(rows, u, top_p=top_p).tolist() == [token for _, token in drawn]
    # the same weights, at another temperature
    assert api.sample(rows * 2.0, u, temperature=2.0, top_p=top_p).tolist() == [token for _, token in drawn]
