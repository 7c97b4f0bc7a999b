"""Cases for timing further language-model operators of this library and for checking their outputs: the gated linear recurrence
(prompts, training, single tokens), layer norm with its gradients, and sampling of tokens from logits.

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes the inputs of one, `run()` computes it -
with the library's operators where `own` is true, otherwise in elementary torch operations - `work()` says what it cannot do
without, and `exact()` evaluates the definition in 64 bits.

Recurrence, for every channel of a sequence on its own, with f = sigmoid(gate):
    h_t = f_t h_{t-1} + i_t x_t          i = 1 - f ("complement"), 1 ("one") or sqrt(1 - f^2) ("root")
Gradients, with D_t the gradient with respect to h_t:
    D_t = dy_t + f_{t+1} D_{t+1}    dx_t = i_t D_t    dgate_t = D_t (h_{t-1} f_t' + x_t i_t')
Layer norm: y = weight (x - mean) / sqrt(variance + eps) + bias over the last axis.
Sampling, for each row of logits with largest value m: weights w = exp((logit - m) / temperature).  In the order of falling
logits, the lower token first among equals, the tokens kept are the first top_k of them, as far as w >= min_p, and of these the
fewest whose weights add up to top_p times the weight of them all.  The token drawn is the first in the order of tokens up to and with which
the kept weights add up to more than u times their sum; the log of its probability is that of its weight over the sum.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # a short question to a small model: launch latency is all of it
        {"name": "recurrence_short", "op": "prompt", "dtype": "bf16", "b": 1, "t": 37, "d": 1024, "state": False, "input": "complement"},
        # one long document that continues a conversation (a state is handed in): a long axis, an odd length
        {"name": "recurrence_long", "op": "prompt", "dtype": "bf16", "b": 1, "t": 16383, "d": 2048, "state": True, "input": "root"},
        # a serving batch of 24 prompts of very different lengths (an empty one and a single token among them), packed, odd rows
        {"name": "recurrence_ragged", "op": "ragged", "dtype": "f16", "b": 24, "t": 16001, "d": 1501, "lens": 7, "input": "complement"},
        # a training step of a small model on short, odd sequences, cut out of longer ones (states and their gradients travel)
        {"name": "recurrence_train_short", "op": "train", "dtype": "f16", "b": 2, "t": 257, "d": 510, "state": True, "input": "one"},
        # a training step of an ordinary layer
        {"name": "recurrence_train", "op": "train", "dtype": "bf16", "b": 8, "t": 4096, "d": 2048, "state": False, "input": "complement"},
        # a full serving batch, one token each, states scattered over a pool
        {"name": "recurrence_token", "op": "token", "dtype": "bf16", "b": 192, "d": 4096, "pool": 200, "input": "complement"},
        # the rows of one decoding step
        {"name": "norm_step", "op": "norm", "dtype": "bf16", "n": 16, "d": 1024, "param": "f32"},
        # a training step of a small model with rows of an odd width
        {"name": "norm_train_small", "op": "norm_train", "dtype": "f16", "n": 1021, "d": 501, "param": "f16"},
        # a training step of an ordinary layer, an odd number of rows
        {"name": "norm_train", "op": "norm_train", "dtype": "bf16", "n": 32749, "d": 2048, "param": "f32"},
        # one user's next token
        {"name": "sample_one", "op": "sample", "dtype": "bf16", "n": 1, "v": 32000, "rule": "top_k", "banned": False},
        # a serving batch, every user with settings of their own, some tokens banned
        {"name": "sample_batch", "op": "sample", "dtype": "f32", "n": 192, "v": 50001, "rule": "mixed", "banned": True},
        # rollouts for training: temperature alone, from the whole of a large vocabulary
        {"name": "sample_whole", "op": "sample", "dtype": "bf16", "n": 256, "v": 128000, "rule": "temperature", "banned": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "ragged", "train", "train", "token", "norm", "norm_train", "norm_train", "sample", "sample", "sample"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if op in ("prompt", "ragged", "train"):
        d = _log_int(rng, 1, 4096)
        if rng.random() < 0.5:
            d += -d % 64
        b = _log_int(rng, 2, 40) if op == "ragged" else _log_int(rng, 1, 32)
        most = (1 << (25 if dtype == "f32" else 26)) // d                         # tokens: below the largest listed case
        t = _log_int(rng, 1, max(1, min(16384, most // (1 if op == "ragged" else b))))
        kind = rng.choice(["complement", "complement", "one", "root"])
        if op == "ragged":
            return {"op": op, "dtype": dtype, "b": b, "t": max(t, 16), "d": d, "lens": rng.randint(0, 1 << 20), "input": kind}
        return {"op": op, "dtype": dtype, "b": b, "t": t, "d": d, "state": rng.random() < 0.5, "input": kind}
    if op == "token":
        b = _log_int(rng, 1, 192)
        return {"op": op, "dtype": dtype, "b": b, "d": _log_int(rng, 1, 4096), "pool": b + rng.randint(0, 8), "input": rng.choice(["complement", "one", "root"])}
    if op in ("norm", "norm_train"):
        d = _log_int(rng, 16, 8192)
        if rng.random() < 0.5:
            d += -d % 64
        return {"op": op, "dtype": dtype, "n": _log_int(rng, 1, min(65536, (1 << (25 if dtype == "f32" else 26)) // d)), "d": d, "param": rng.choice(["f32", dtype])}
    v = _log_int(rng, 100, 131072)
    return {"op": op, "dtype": dtype, "n": _log_int(rng, 1, min(256, (1 << (24 if dtype == "f32" else 25)) // v)), "v": v,
            "rule": rng.choice(["greedy", "temperature", "top_k", "top_p", "min_p", "mixed", "mixed"]), "banned": rng.random() < 0.3}


def _lengths(case):
    """The lengths of a ragged case: over the range of their logarithm, one empty and one of a single token among them."""
    rng, b, left = random.Random(case["lens"]), case["b"], case["t"]
    weights = [math.exp(rng.uniform(0.0, 5.0)) for _ in range(b)]
    lens = [max(0, int(left * w / sum(weights))) for w in weights]
    if b > 2:
        lens[1], lens[2] = 0, 1
    lens[0] += left - sum(lens)
    return lens


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, op = TYPES[case["dtype"]], case["op"]
    s = {"op": op}

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if op in ("norm", "norm_train"):
        n, d, pt = case["n"], case["d"], TYPES[case["param"]]
        # a residual stream: a few channels far larger than the rest, rows off zero
        s["x"] = (normal(n, d) * torch.exp(0.7 * normal(d)) + 0.3 * normal(n, 1)).to(dt)
        s["weight"], s["bias"] = (1.0 + 0.2 * normal(d)).to(pt), (0.1 * normal(d)).to(pt)
        if op == "norm_train":
            s["d_y"] = (0.1 * normal(n, d)).to(dt)
        return s
    if op == "sample":
        n, v = case["n"], case["v"]
        peaks = torch.relu(normal(n, v) - 2.5) * 5.0                              # a few tokens well above the rest
        s["logits"] = (2.0 * normal(n, v) + peaks + normal(n, 1)).to(dt)
        if case["banned"]:
            s["logits"].masked_fill_(torch.rand((n, v), generator=g, device="cuda") < 0.1, -math.inf)
        s["u"] = torch.rand(n, generator=g, device="cuda")
        rule = case["rule"]
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = 0.8, 0, 1.0, 0.0
        if rule == "greedy":
            s["temperature"] = 0.0
        elif rule == "top_k":
            s["top_k"], s["top_p"] = 50, 0.95
        elif rule == "top_p":
            s["top_p"] = 0.9
        elif rule == "min_p":
            s["min_p"] = 0.02
        elif rule == "mixed":       # each row its own: greedy ones, ones without a rule, ones with all three
            pick = torch.randint(0, 6, (n,), generator=g, device="cuda")
            s["temperature"] = torch.where(pick == 0, 0.0, 0.6 + 0.6 * torch.rand(n, generator=g, device="cuda"))
            s["top_k"] = torch.where((pick == 1) | (pick == 5), torch.randint(1, 200, (n,), generator=g, device="cuda"), 0).to(torch.int32)
            s["top_p"] = torch.where((pick == 2) | (pick == 5), 0.5 + 0.49 * torch.rand(n, generator=g, device="cuda"), 1.0)
            s["min_p"] = torch.where((pick == 3) | (pick == 5), 0.1 * torch.rand(n, generator=g, device="cuda"), 0.0)
        return s
    b, d = case["b"], case["d"]
    s["input"] = case["input"]
    lead = {"ragged": (case.get("t"),), "token": (b,)}.get(op, (b, case.get("t")))
    s["x"] = normal(*lead, d).to(dt)
    # gates: channels that remember from a few tokens to hundreds
    s["gate"] = (4.0 * torch.rand(d, generator=g, device="cuda") + 1.0 + normal(*lead, d)).to(dt)
    if op == "ragged":
        lens = _lengths(case)
        s["offsets"] = torch.tensor([0] + lens, device="cuda").cumsum(0)
        s["longest"] = max(lens)
    if op == "token":
        s["state"] = normal(case["pool"], d)
        s["slots"] = torch.randperm(case["pool"], generator=g, device="cuda")[:b].to(torch.int32)
    if op in ("prompt", "train"):
        s["s0"] = normal(b, d) if case["state"] else None
    if op == "train":
        s["d_y"] = (0.1 * normal(*lead, d)).to(dt)
        s["d_last"] = 0.1 * normal(b, d) if case["state"] else None
    return s


# ------------------------------------------------------------------------------------------------------ plain form
def _gates(gate, kind):
    """f, i, and the derivatives of both by the gate."""
    f, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    df = f * rest
    if kind == "complement":
        return f, rest, df, -df
    if kind == "one":
        return f, torch.ones_like(f), df, torch.zeros_like(f)
    i = torch.sqrt(rest * (1.0 + f))
    return f, i, df, -f * f * torch.sqrt(rest / (1.0 + f))


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along axis 1 by doubling: log2(t) passes over both arrays."""
    step, t = 1, a.shape[1]
    while step < t:
        b = torch.cat([b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def _first(b, a, s0):
    """b with what the state before the first token adds to it."""
    return b if s0 is None else torch.cat([(b[:, 0] + a[:, 0] * s0)[:, None], b[:, 1:]], 1)


def _plain_sample(s):
    logits = s["logits"].double()
    n, v = logits.shape

    def each(value):
        return value.double()[:, None] if isinstance(value, torch.Tensor) else torch.full((n, 1), float(value), device=logits.device, dtype=torch.float64)

    temperature, top_k, top_p, min_p = (each(s[name]) for name in ("temperature", "top_k", "top_p", "min_p"))
    falling, order = torch.sort(logits, dim=1, descending=True, stable=True)
    w = torch.exp((falling - falling[:, :1]) / torch.where(temperature > 0, temperature, 1.0))
    rank = torch.arange(v, device=logits.device)
    top_k = torch.where(temperature > 0, top_k, 1.0)
    kept = ((top_k <= 0) | (rank < top_k)) & ((w >= min_p) | (rank == 0))
    w = torch.where(kept, w, 0.0)
    before = torch.cumsum(w, 1) - w
    kept &= (top_p >= 1.0) | (before < top_p * w.sum(1, keepdim=True)) | (rank == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(kept, w, 0.0))
    upto = torch.cumsum(w, 1)
    token = (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1)
    return token, torch.log(w.gather(1, token[:, None])[:, 0] / upto[:, -1]).float()


def _plain(s):
    op = s["op"]
    if op == "sample":
        return _plain_sample(s)
    if op in ("norm", "norm_train"):
        dt, x, weight = s["x"].dtype, s["x"].float(), s["weight"].float()
        centred = x - x.mean(1, keepdim=True)
        r = torch.rsqrt(centred.square().mean(1, keepdim=True) + 1e-5)
        unit = centred * r
        y = (unit * weight + s["bias"].float()).to(dt)
        if op == "norm":
            return y
        d_y = s["d_y"].float()
        d_unit = d_y * weight
        d_x = r * (d_unit - d_unit.mean(1, keepdim=True) - unit * (d_unit * unit).mean(1, keepdim=True))
        return y, d_x.to(dt), (d_y * unit).sum(0).to(s["weight"].dtype), d_y.sum(0).to(s["weight"].dtype)
    dt, x = s["x"].dtype, s["x"].float()
    f, i, df, di = _gates(s["gate"].float(), s["input"])
    if op == "token":
        pool, at = s["state"], s["slots"].long()
        new = f * pool[at] + i * x
        pool[at] = new
        return new.to(dt), pool
    if op == "ragged":
        off = s["offsets"]
        lens = off[1:] - off[:-1]
        at = torch.arange(s["longest"], device="cuda")
        valid = (at < lens[:, None])[..., None]
        take = (off[:-1, None] + at).clamp(max=x.shape[0] - 1)
        h = _scan(torch.where(valid, f[take], 1.0), torch.where(valid, (i * x)[take], 0.0))
        token = torch.arange(x.shape[0], device="cuda")
        row = (token[:, None] >= off[1:]).sum(1)
        return h[row, token - off[row]].to(dt), h[:, -1]
    s0 = s["s0"]
    h = _scan(f, _first(i * x, f, s0))
    if op == "prompt":
        return h.to(dt), h[:, -1]
    first = torch.zeros_like(h[:, :1]) if s0 is None else s0[:, None]
    before = torch.cat([first, h[:, :-1]], 1)
    d_y = s["d_y"].float().flip(1)
    later = torch.cat([torch.zeros_like(f[:, :1]), f.flip(1)[:, :-1]], 1)
    grad = _scan(later, d_y if s["d_last"] is None else torch.cat([d_y[:, :1] + s["d_last"][:, None], d_y[:, 1:]], 1)).flip(1)
    d_x, d_gate = i * grad, grad * (before * df + x * di)
    has = s0 is not None
    return h.to(dt), h[:, -1] if has else None, d_x.to(dt), d_gate.to(dt), f[:, 0] * grad[:, 0] if has else None


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2411_17887_b200 import api
    op = s["op"]
    if op == "sample":
        return api.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], output_log_prob=True)
    if op == "norm":
        return api.layer_norm(s["x"], s["weight"], s["bias"])
    if op == "norm_train":
        return (api.layer_norm(s["x"], s["weight"], s["bias"]), *api.layer_norm_backward(s["d_y"], s["x"], s["weight"]))
    x, gate, kind = s["x"], s["gate"], s["input"]
    if op == "token":
        return api.gated_recurrence_step(x, gate, s["state"], slots=s["slots"], input_gate=kind), s["state"]
    if op == "ragged":
        return api.gated_recurrence(x, gate, offsets=s["offsets"], output_final_state=True, input_gate=kind)
    if op == "prompt":
        return api.gated_recurrence(x, gate, initial_state=s["s0"], output_final_state=True, input_gate=kind)
    has = s["s0"] is not None
    y, last, marks = api.gated_recurrence(x, gate, initial_state=s["s0"], output_final_state=has, input_gate=kind, output_marks=True)
    d_x, d_gate, d_s0 = api.gated_recurrence_backward(s["d_y"], x, gate, initial_state=s["s0"], d_final_state=s["d_last"], input_gate=kind, marks=marks)
    return y, last, d_x, d_gate, d_s0


# ------------------------------------------------------------------------------------------------------ floors
def work(case):
    e, op = BYTES[case["dtype"]], case["op"]
    if op == "sample":
        n, v = case["n"], case["v"]
        return {"bytes": n * v * e + 16 * n, "flops": 4 * n * v}
    if op in ("norm", "norm_train"):
        n, d, p = case["n"], case["d"], BYTES[case["param"]]
        if op == "norm":
            return {"bytes": 2 * n * d * e + 2 * d * p, "flops": 8 * n * d}
        return {"bytes": 4 * n * d * e + 4 * d * p, "flops": 24 * n * d}       # x, dy read, y, dx written
    d = case["d"]
    if op == "token":
        return {"bytes": case["b"] * d * (8 + 3 * e) + 4 * case["b"], "flops": 8 * case["b"] * d}
    n = (1 if op == "ragged" else case["b"]) * case["t"] * d
    state = case["b"] * d * 4
    if op == "train":                                                           # x, gate, dy read, y, dx, dgate written
        return {"bytes": 6 * n * e + (4 * state if case["state"] else 0), "flops": 24 * n}
    return {"bytes": 3 * n * e + state * (2 if op == "prompt" and case["state"] else 1), "flops": 8 * n}


# ------------------------------------------------------------------------------------------------------ 64 bits
def _exact_row(logits, u, temperature, top_k, top_p, min_p):
    """The token of one row, and the log of its probability, by their definition, on the host."""
    order = np.lexsort((np.arange(logits.size), -logits))
    if not temperature > 0:
        return int(order[0]), 0.0
    w = np.exp((logits[order] - logits[order[0]]) / temperature)
    m = logits.size if top_k <= 0 else min(int(top_k), logits.size)
    m = max(1, min(m, int(np.searchsorted(-w, -min_p, side="right"))))
    if top_p < 1.0:
        upto = np.cumsum(w[:m])
        m = min(m, int(np.searchsorted(upto, top_p * upto[-1], side="left")) + 1)
    kept = np.sort(order[:m])
    upto = np.cumsum(np.exp((logits[kept] - logits[order[0]]) / temperature))
    token = int(kept[min(np.searchsorted(upto, u * upto[-1], side="right"), m - 1)])
    return token, (logits[token] - logits[order[0]]) / temperature - math.log(math.fsum(np.exp((logits[kept] - logits[order[0]]) / temperature)))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "sample":
        logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
        rules = [np.broadcast_to(s[name].double().cpu().numpy() if isinstance(s[name], torch.Tensor) else float(s[name]), u.shape)
                 for name in ("temperature", "top_k", "top_p", "min_p")]
        tokens, log_probs = zip(*(_exact_row(row, u[k], *(r[k] for r in rules)) for k, row in enumerate(logits)))
        return torch.tensor(tokens, device="cuda"), torch.tensor(log_probs, device="cuda", dtype=torch.float64)
    if op in ("norm", "norm_train"):
        x, weight, bias = s["x"].double(), s["weight"].double(), s["bias"].double()
        variance, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        deviation = torch.sqrt(variance + 1e-5)
        y = weight * (x - mean) / deviation + bias
        if op == "norm":
            return y
        d_y, d = s["d_y"].double(), case["d"]
        inner = weight * d_y
        along = (inner * (x - mean)).sum(1, keepdim=True) / (deviation ** 2 * d)
        d_x = (inner - inner.sum(1, keepdim=True) / d - (x - mean) * along) / deviation
        return y, d_x, torch.einsum("nd,nd->d", d_y, (x - mean) / deviation), d_y.sum(0)
    x, gate, kind = s["x"].double(), s["gate"].double(), s["input"]
    f = 1.0 / (1.0 + torch.exp(-gate))
    rest = 1.0 / (1.0 + torch.exp(gate))
    i = {"complement": rest, "one": torch.ones_like(f), "root": torch.sqrt(rest * (1.0 + f))}[kind]
    if op == "token":
        at, pool = s["slots"].long(), s["state"].double()
        pool[at] = f * pool[at] + i * x
        return pool[at], pool
    if op == "ragged":
        outs, lasts, at = [], [], 0
        for n in _lengths(case):
            h = torch.zeros(case["d"], device="cuda", dtype=torch.float64)
            for t in range(at, at + n):
                h = f[t] * h + i[t] * x[t]
                outs.append(h)
            lasts.append(h)
            at += n
        return torch.stack(outs), torch.stack(lasts)
    b, t, d = x.shape
    h = torch.zeros(b, d, device="cuda", dtype=torch.float64) if s["s0"] is None else s["s0"].double()
    first, outs, add = h, torch.empty_like(x), i * x
    for k in range(t):
        h = torch.addcmul(add[:, k], f[:, k], h)
        outs[:, k] = h
    if op == "prompt":
        return outs, h
    has = s["s0"] is not None
    flow = s["d_last"].double() if has else torch.zeros_like(first)
    grads, d_y = torch.empty_like(x), s["d_y"].double()
    for k in range(t - 1, -1, -1):
        grads[:, k] = d_y[:, k] + flow
        flow = f[:, k] * grads[:, k]
    before = torch.cat([first[:, None], outs[:, :-1]], 1)
    slope = {"complement": -f * rest, "one": torch.zeros_like(f), "root": -f * f * rest / torch.clamp(i, min=1e-300)}[kind]
    return outs, h if has else None, i * grads, grads * (before * f * rest + x * slope), flow if has else None
