"""Cases for timing the language-model operators of this library and for checking their outputs: linear attention with a
constant decay for each head (prompts, training, single tokens) and the token embedding (lookup, table gradient).

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes the inputs of one, `run()` computes it -
with the library's operators where `own` is true, otherwise in elementary torch operations in 32 bits - `work()` says what it
cannot do without, and `exact()` evaluates the definition in 64 bits.

Linear attention, per sequence and head, with a = exp(log_decay[head]) and a state S of dk x dv:
    S_t = a S_{t-1} + k_t v_t^T          o_t = scale * S_t^T q_t
Gradients, with D_t the gradient with respect to S_t:
    D_t = scale * q_t do_t^T + a D_{t+1}    dq_t = scale * S_t do_t    dk_t = D_t v_t    dv_t = D_t^T k_t
Embedding: out[n] = scale * table[ids[n]]; table gradient: row v is scale * (sum of d_out[n] over the n with ids[n] = v).
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
CHUNK = 128       # tokens a chunk in the plain form


def listed():
    return [
        # a short question to a small model: launch latency is all of it
        {"name": "prompt_short", "op": "prompt", "dtype": "bf16", "b": 1, "t": 37, "h": 4, "dk": 64, "dv": 64, "state": False},
        # one long document that continues a conversation (a state is handed in): few heads, a long axis, an odd length
        {"name": "prompt_long", "op": "prompt", "dtype": "bf16", "b": 1, "t": 8191, "h": 16, "dk": 128, "dv": 128, "state": True},
        # a serving batch of 24 prompts of very different lengths (an empty one and a single token among them), packed
        {"name": "prompts_ragged", "op": "ragged", "dtype": "f16", "b": 24, "t": 16001, "h": 12, "dk": 96, "dv": 128, "lens": 7},
        # the largest prompt batch: many heads and sequences, bound by memory
        {"name": "prompt_batch", "op": "prompt", "dtype": "bf16", "b": 8, "t": 4096, "h": 32, "dk": 128, "dv": 128, "state": False},
        # a training step of a small model on short, odd sequences, cut out of longer ones (states and their gradients travel)
        {"name": "train_short", "op": "train", "dtype": "f16", "b": 2, "t": 257, "h": 6, "dk": 64, "dv": 64, "state": True},
        # a training step of an ordinary layer
        {"name": "train_layer", "op": "train", "dtype": "bf16", "b": 4, "t": 4096, "h": 16, "dk": 128, "dv": 128, "state": False},
        # one user, one token
        {"name": "token_one", "op": "token", "dtype": "bf16", "b": 1, "h": 16, "dk": 128, "dv": 128, "pool": 4},
        # a full serving batch, one token each, states scattered over a pool
        {"name": "token_batch", "op": "token", "dtype": "bf16", "b": 192, "h": 16, "dk": 128, "dv": 128, "pool": 200},
        # the tokens of one decoding step
        {"name": "lookup_step", "op": "lookup", "dtype": "bf16", "n": 16, "v": 32000, "d": 1024},
        # the tokens of a training batch, an odd number of them
        {"name": "lookup_batch", "op": "lookup", "dtype": "bf16", "n": 32749, "v": 50000, "d": 2048},
        # table gradient of a small model with rows of an odd width
        {"name": "table_grad_small", "op": "table_grad", "dtype": "f16", "n": 1021, "v": 4099, "d": 500},
        # table gradient of a training batch: a few tokens make up much of it, most rows get nothing
        {"name": "table_grad_batch", "op": "table_grad", "dtype": "bf16", "n": 65536, "v": 50000, "d": 1024},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["prompt", "ragged", "train", "train", "token", "lookup", "table_grad", "table_grad"])
    dtype = rng.choice(["bf16", "f16"])
    if op in ("prompt", "ragged", "train"):
        h = _log_int(rng, 1, 32)
        dk = 8 * rng.randint(2, 16)
        dv = rng.choice([dk, dk, 8 * rng.randint(2, 16)])
        b = _log_int(rng, 1, 8) if op != "ragged" else _log_int(rng, 2, 40)
        most = (1 << 28) // (h * (dk + dv) * (4 if op == "train" else 1))          # elements: below the largest listed case
        t = _log_int(rng, 1, max(1, min(8192, most // (b if op != "ragged" else 1))))
        if op == "ragged":
            return {"op": op, "dtype": dtype, "b": b, "t": max(t, 16), "h": h, "dk": dk, "dv": dv, "lens": rng.randint(0, 1 << 20)}
        return {"op": op, "dtype": dtype, "b": b, "t": t, "h": h, "dk": dk, "dv": dv, "state": rng.random() < 0.5}
    if op == "token":
        b, h = _log_int(rng, 1, 192), _log_int(rng, 1, 16)
        dk = 8 * rng.randint(2, 16)
        return {"op": op, "dtype": dtype, "b": b, "h": h, "dk": dk, "dv": rng.choice([dk, 8 * rng.randint(2, 16)]), "pool": b + rng.randint(0, 8)}
    dtype = rng.choice(["bf16", "f16", "f32"])
    v, d = _log_int(rng, 100, 50000), _log_int(rng, 16, 2048)
    most = (1 << 26) // d
    return {"op": op, "dtype": dtype, "n": _log_int(rng, 1, min(65536, most)), "v": min(v, 2 * most), "d": d}


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
    dt = TYPES[case["dtype"]]
    s = {"op": case["op"]}

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if case["op"] in ("lookup", "table_grad"):
        n, v, d = case["n"], case["v"], case["d"]
        cdf = torch.cumsum(1.0 / (torch.arange(v, device="cuda", dtype=torch.float64) + 3.0), 0)      # the usual law of token counts
        at = torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * cdf[-1]
        s.update(ids=torch.searchsorted(cdf, at).clamp_(max=v - 1), rows=v, scale=math.sqrt(d))
        if case["op"] == "lookup":
            s["table"] = (normal(v, d) / math.sqrt(d)).to(dt)
        else:
            s["d_out"] = (normal(n, d) * 1e-2).to(dt)
        return s
    b, h, dk, dv = case["b"], case["h"], case["dk"], case["dv"]
    lead = {"ragged": (case.get("t"),), "token": (b,)}.get(case["op"], (b, case.get("t")))
    s["q"] = torch.nn.functional.silu(normal(*lead, h, dk)).to(dt)
    s["k"] = torch.nn.functional.silu(normal(*lead, h, dk)).to(dt)
    s["v"] = normal(*lead, h, dv).to(dt)
    s["log_decay"] = -torch.exp2(-8.0 * (torch.arange(h, device="cuda") + 1.0) / h)     # from a few tokens of memory to hundreds
    s["scale"] = dk ** -0.5
    if case["op"] == "ragged":
        lens = _lengths(case)
        s["offsets"] = torch.tensor([0] + lens, device="cuda").cumsum(0)
        s["longest"] = max(lens)
    if case["op"] == "token":
        s["state"] = normal(case["pool"], h, dk, dv)
        s["slots"] = torch.randperm(case["pool"], generator=g, device="cuda")[:b].to(torch.int32)
    if case["op"] in ("prompt", "train"):
        s["s0"] = normal(b, h, dk, dv) if case["state"] else None
    if case["op"] == "train":
        s["d_o"] = normal(*lead, h, dv).to(dt)
        s["d_state"] = normal(b, h, dk, dv) if case["state"] else None
    return s


# ------------------------------------------------------------------------------------------------------ plain form
def _mix(q, k, v, g, s0, lead):
    """o_i = sum over j <= i of a^(i-j) (q_i . k_j) v_j + a^(i+lead) s0^T q_i, in chunks: (b, t, h, d) in 32 bits."""
    b, t, h, _ = q.shape
    n = -(-t // CHUNK)
    q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, 0, 0, n * CHUNK - t)).transpose(1, 2).reshape(b, h, n, CHUNK, -1) for x in (q, k, v))
    i = torch.arange(CHUNK, device=q.device, dtype=torch.float32)
    c = torch.arange(n, device=q.device, dtype=torch.float32)
    g1, g2 = g[:, None], g[:, None, None]
    near = torch.where(i[:, None] >= i, torch.exp(g2 * (i[:, None] - i).clamp(min=0)), 0.0)
    o = (q @ k.transpose(-1, -2) * near[:, None]) @ v
    kv = (k * torch.exp(g1 * (CHUNK - 1 - i))[:, None, :, None]).transpose(-1, -2) @ v
    before = torch.where(c[:, None] > c, torch.exp(g2 * CHUNK * (c[:, None] - c - 1).clamp(min=0)), 0.0)
    s = (before @ kv.flatten(3)).view(kv.shape)             # the state before each chunk, without s0
    o = o + (q * torch.exp(g1 * (i + 1))[:, None, :, None]) @ s
    o = o.reshape(b, h, n * CHUNK, -1)[:, :, :t]
    if s0 is not None:
        at = torch.arange(t, device=q.device, dtype=torch.float32)
        o = o + (q.reshape(b, h, n * CHUNK, -1)[:, :, :t] * torch.exp(g1 * (at + lead))[:, :, None]) @ s0
    return o.transpose(1, 2)


def _last_state(k, v, g, s0, lens, tail=0):
    """sum over t < len of a^(len-1-t+tail) k_t v_t^T + a^len s0"""
    at = torch.arange(k.shape[1], device=k.device)
    left = (lens[:, None] - 1 - at).float()[:, :, None]
    w = torch.where(left >= 0, torch.exp(g * (left.clamp(min=0) + tail)), 0.0)
    s = (k * w[..., None]).permute(0, 2, 3, 1) @ v.transpose(1, 2)
    return s if s0 is None else s + torch.exp(g * lens[:, None])[..., None, None] * s0


def _plain(s):
    op = s["op"]
    if op == "lookup":
        return (s["table"][s["ids"]].float() * s["scale"]).to(s["table"].dtype)
    if op == "table_grad":
        return torch.zeros(s["rows"], s["d_out"].shape[1], device="cuda").index_add_(0, s["ids"], s["d_out"].float()) * s["scale"]
    dt = s["q"].dtype
    q, k, v, g = s["q"].float(), s["k"].float(), s["v"].float(), s["log_decay"]
    if op == "token":
        pool, at = s["state"], s["slots"].long()
        new = torch.exp(g)[:, None, None] * pool[at] + k[..., :, None] * v[..., None, :]
        pool[at] = new
        return (q[..., None, :] @ new).squeeze(-2).mul(s["scale"]).to(dt), pool
    if op == "ragged":
        off = s["offsets"]
        lens = off[1:] - off[:-1]
        at = torch.arange(s["longest"], device="cuda")
        valid = (at < lens[:, None])[..., None, None]
        take = (off[:-1, None] + at).clamp(max=q.shape[0] - 1)
        q, k, v = (torch.where(valid, x[take], 0.0) for x in (q, k, v))
        o = _mix(q * s["scale"], k, v, g, None, 1)
        token = torch.arange(s["q"].shape[0], device="cuda")
        row = (token[:, None] >= off[1:]).sum(1)
        return o[row, token - off[row]].to(dt), _last_state(k, v, g, None, lens)
    lens = torch.full((q.shape[0],), q.shape[1], device="cuda")
    o = _mix(q * s["scale"], k, v, g, s["s0"], 1).to(dt)
    last = _last_state(k, v, g, s["s0"], lens)
    if op == "prompt":
        return o, last
    d_o, d_s, s0 = s["d_o"].float(), s["d_state"], s["s0"]
    flip = lambda x: x.flip(1)  # noqa: E731
    turn = lambda x: None if x is None else x.transpose(-1, -2)  # noqa: E731
    qs = flip(q * s["scale"])
    dq = _mix(d_o * s["scale"], v, k, g, turn(s0), 1)
    dk = flip(_mix(flip(v), flip(d_o * s["scale"]), flip(q), g, turn(d_s), 0))
    dv = flip(_mix(flip(k), qs, flip(d_o), g, d_s, 0))
    d_s0 = None if s0 is None else _last_state(qs, flip(d_o), g, d_s, lens, 1)
    return o, last if s0 is not None else None, dq.to(dt), dk.to(dt), dv.to(dt), d_s0


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2411_17887_b200 import api
    op = s["op"]
    if op == "lookup":
        return api.embedding(s["ids"], s["table"], scale=s["scale"])
    if op == "table_grad":
        return api.embedding_backward(s["d_out"], s["ids"], s["rows"], scale=s["scale"])
    q, k, v, g = s["q"], s["k"], s["v"], s["log_decay"]
    if op == "token":
        return api.linear_attention_step(q, k, v, g, s["state"], scale=s["scale"], slots=s["slots"]), s["state"]
    if op == "ragged":
        return api.linear_attention(q, k, v, g, scale=s["scale"], offsets=s["offsets"], output_final_state=True)
    if op == "prompt":
        return api.linear_attention(q, k, v, g, scale=s["scale"], initial_state=s["s0"], output_final_state=True)
    o, last = api.linear_attention(q, k, v, g, scale=s["scale"], initial_state=s["s0"], output_final_state=s["s0"] is not None)
    dq, dk, dv, d_s0 = api.linear_attention_backward(s["d_o"], q, k, v, g, scale=s["scale"], initial_state=s["s0"], d_final_state=s["d_state"])
    return o, last, dq, dk, dv, d_s0


# ------------------------------------------------------------------------------------------------------ floors
def _rows_met(n, v):
    """How many different rows n tokens meet, in the mean."""
    p = 1.0 / (np.arange(v) + 3.0)
    return float(np.sum(-np.expm1(n * np.log1p(-p / p.sum()))))


def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "lookup":
        n, d = case["n"], case["d"]
        return {"bytes": n * 8 + (n + _rows_met(n, case["v"])) * d * e, "flops": n * d}
    if case["op"] == "table_grad":
        n, d = case["n"], case["d"]
        return {"bytes": n * 8 + n * d * e + case["v"] * d * 4, "flops": n * d + _rows_met(n, case["v"]) * d}
    b, h, dk, dv = case["b"], case["h"], case["dk"], case["dv"]
    state = b * h * dk * dv * 4
    if case["op"] == "token":
        return {"bytes": 2 * state + b * h * 2 * (dk + dv) * e + 4 * b, "flops": 5 * b * h * dk * dv}
    tokens = (case["t"] if case["op"] == "ragged" else b * case["t"]) * h
    rows = tokens * (dk + dv) * e          # q and o, or k and v: each pair once
    if case["op"] == "ragged":
        return {"bytes": 2 * rows + state, "flops": 4 * tokens * dk * dv}
    if case["op"] == "prompt":
        return {"bytes": 2 * rows + state * (2 if case["state"] else 1), "flops": 4 * tokens * dk * dv}
    # forward: q, k, v -> o; backward: q, k, v, do -> dq, dk, dv. The state is formed once more going back.
    back = 2 * rows + rows + tokens * dk * e
    return {"bytes": 2 * rows + back + (5 * state if case["state"] else 0), "flops": 14 * tokens * dk * dv}


# ------------------------------------------------------------------------------------------------------ 64 bits
def _walk(q, k, v, a, scale, state, outputs):
    """The definition, token by token, over the first axis of (t, rows, d): every o_t, and the last state."""
    for t in range(q.shape[0]):
        state = a * state + k[t, :, :, None] * v[t, :, None, :]
        outputs.append(scale * torch.matmul(q[t, :, None, :], state).squeeze(1))
    return state


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "lookup":
        return s["table"].double()[s["ids"]] * s["scale"]
    if op == "table_grad":
        order = torch.sort(s["ids"], stable=True)
        total = torch.zeros(case["n"] + 1, case["d"], device="cuda", dtype=torch.float64)
        torch.cumsum(s["d_out"].double()[order.indices], 0, out=total[1:])
        row = torch.arange(case["v"], device="cuda")
        lo, hi = (torch.searchsorted(order.values, row, right=r) for r in (False, True))
        return (total[hi] - total[lo]) * s["scale"]
    h, dk, dv, scale = case["h"], case["dk"], case["dv"], s["scale"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    decay = torch.exp(s["log_decay"].double())
    if op == "token":
        at, pool = s["slots"].long(), s["state"].double()
        pool[at] = decay[:, None, None] * pool[at] + torch.einsum("bhk,bhv->bhkv", k, v)
        return scale * torch.einsum("bhk,bhkv->bhv", q, pool[at]), pool
    if op == "ragged":
        outs, states, at = [], [], 0
        for n in _lengths(case):
            got = []
            states.append(_walk(q[at:at + n], k[at:at + n], v[at:at + n], decay[:, None, None], scale,
                                torch.zeros(h, dk, dv, device="cuda", dtype=torch.float64), got))
            outs += got
            at += n
        return torch.stack(outs), torch.stack(states)
    b, t = case["b"], case["t"]
    rows = lambda x, d: x.transpose(0, 1).reshape(t, b * h, d)  # noqa: E731
    back = lambda xs, d: torch.stack(xs).view(t, b, h, d).transpose(0, 1)  # noqa: E731
    a = decay.repeat(b)[:, None, None]
    q, k, v = rows(q, dk), rows(k, dk), rows(v, dv)
    zero = torch.zeros(b * h, dk, dv, device="cuda", dtype=torch.float64)
    first = zero if s["s0"] is None else s["s0"].double().view(b * h, dk, dv)
    outs = []
    last = _walk(q, k, v, a, scale, first, outs)
    if op == "prompt":
        return back(outs, dv), last.view(b, h, dk, dv)
    d_o = rows(s["d_o"].double(), dv)
    dq, dk_, dv_, state = [], [], [], first
    for i in range(t):
        state = a * state + k[i, :, :, None] * v[i, :, None, :]
        dq.append(scale * torch.matmul(state, d_o[i, :, :, None]).squeeze(2))
    grad = zero if s["d_state"] is None else s["d_state"].double().view(b * h, dk, dv)
    for i in range(t - 1, -1, -1):
        grad = grad + scale * q[i, :, :, None] * d_o[i, :, None, :]
        dk_.append(torch.matmul(grad, v[i, :, :, None]).squeeze(2))
        dv_.append(torch.matmul(k[i, :, None, :], grad).squeeze(1))
        grad = a * grad
    has = s["s0"] is not None
    return (back(outs, dv), last.view(b, h, dk, dv) if has else None, back(dq, dk), back(dk_[::-1], dk), back(dv_[::-1], dv),
            grad.view(b, h, dk, dv) if has else None)
