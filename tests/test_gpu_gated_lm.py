"""The example model with gated layers: embedding, linear attention, layer norm, gated recurrence and sampling as they are used together."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("linear_lm", Path(__file__).resolve().parents[1] / "examples" / "linear_lm.py")
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def model_of(lm, seed):
    torch.manual_seed(seed)
    return lm.LinearLM(vocabulary=90, width=72, heads=2, d_head=24, layers=4, gated=True).cuda()


def test_training_and_serving(lm):
    model = model_of(lm, 1)
    successor = torch.randperm(90, device="cuda")
    lm.train(model, successor, steps=5, batch=4, tokens=150)
    prompts = [lm.sequences(successor, 1, n)[0] for n in (0, 129, 40, 300, 1)]
    tokens, seen = lm.serve(model, prompts, new_tokens=12)
    # Each layer's output and what is added to it is rounded to bfloat16 (2^-8) a few times on either way: four layers stay inside 2^-3 of the
    # largest logit.
    for prompt, chosen, logits in zip(prompts, tokens, seen):
        whole, _ = model(torch.cat([prompt, chosen])[None])
        want = whole[0, len(prompt) - 1:-1].float()
        assert (logits.float() - want).abs().max() <= 2.0 ** -3 * want.abs().max()
    assert lm.api.linear_attention_status() == 0


def test_tokens_that_are_drawn(lm):
    model = model_of(lm, 2)
    prompts = [torch.randint(90, (n,), device="cuda") for n in (3, 70, 200)]
    # one candidate: the likeliest token, every time
    drawn, seen = lm.serve(model, prompts, 8, temperature=0.7, top_k=1)
    assert torch.equal(drawn, seen.float().argmax(-1))
    # seven candidates: none but these
    drawn, seen = lm.serve(model, prompts, 30, temperature=1.0, top_k=7, top_p=0.99)
    seventh = seen.float().sort(-1, descending=True).values[..., 6]
    assert (seen.float().gather(-1, drawn[..., None])[..., 0] >= seventh).all()


def test_gradients_reach_every_parameter(lm):
    model = model_of(lm, 3)
    ids = torch.randint(90, (3, 140), device="cuda")
    logits, _ = model(ids)
    logits.float().logsumexp(-1).sum().backward()
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.abs().sum() > 0, name


def test_gradients_are_those_of_plain_operators(lm, monkeypatch):
    """The same model with both new operators in elementary torch in 32 bits."""
    model = model_of(lm, 4)
    ids = torch.randint(90, (2, 100), device="cuda")

    def gradients():
        model.zero_grad()
        logits, _ = model(ids)
        logits.float().logsumexp(-1).sum().backward()
        return {name: p.grad.float().clone() for name, p in model.named_parameters()}

    def plain_norm(x, weight, bias, eps=1e-5):
        v = x.float() - x.float().mean(-1, keepdim=True)
        return (v * torch.rsqrt(v.square().mean(-1, keepdim=True) + eps) * weight + bias).to(x.dtype)

    def plain_recurrence(x, gate, initial_state=None, offsets=None, output_final_state=False, input_gate="root"):
        f = torch.sigmoid(gate.float())
        b, h, out = torch.sqrt(1.0 - f * f) * x.float(), torch.zeros_like(x[:, 0], dtype=torch.float32), []
        for t in range(x.shape[1]):
            h = f[:, t] * h + b[:, t]
            out.append(h)
        return torch.stack(out, 1).to(x.dtype), h

    got = gradients()
    monkeypatch.setattr(lm.api, "layer_norm", plain_norm)
    monkeypatch.setattr(lm.api, "gated_recurrence", plain_recurrence)
    want = gradients()
    # both round every layer's values to bfloat16 (2^-8), at the same places: what differs is which way some of them are rounded
    for name in got:
        assert (got[name] - want[name]).norm() <= 2.0 ** -5 * want[name].norm(), name
