"""The example model on the operators: it learns, and tokens taken one at a time go on from packed prompts as a whole pass does."""
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


def test_training_and_serving(lm):
    torch.manual_seed(1)
    model = lm.LinearLM(vocabulary=90, width=64, heads=2, d_head=24).cuda()
    successor = torch.randperm(90, device="cuda")
    losses = lm.train(model, successor, steps=60, batch=8, tokens=150)
    assert losses[-1] < 0.5 * losses[0]

    prompts = [lm.sequences(successor, 1, n)[0] for n in (0, 129, 40, 300, 1)]
    tokens, seen = lm.serve(model, prompts, new_tokens=12)
    # Each layer's output and what is added to it is rounded to bfloat16 (2^-8) a few times on either way: two layers stay
    # well inside 2^-4 of the largest logit.
    for prompt, chosen, logits in zip(prompts, tokens, seen):
        whole, _ = model(torch.cat([prompt, chosen])[None])
        want = whole[0, len(prompt) - 1:-1].float()
        assert (logits.float() - want).abs().max() <= 2.0 ** -4 * want.abs().max()
    assert lm.api.linear_attention_status() == 0


def test_gradients_reach_every_parameter(lm):
    torch.manual_seed(2)
    model = lm.LinearLM(vocabulary=50, width=32, heads=3, d_head=16).cuda()
    ids = torch.randint(50, (3, 140), device="cuda")
    logits, _ = model(ids)
    logits.float().logsumexp(-1).sum().backward()
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.abs().sum() > 0, name
