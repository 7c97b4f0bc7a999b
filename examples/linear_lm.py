#!/usr/bin/env python3
"""A small language model on the library's operators, trained and then served.

    python examples/linear_lm.py [--steps 160]

Token embedding (its table also gives the logits), layers of linear attention with a decay for each head, torch for the
projections between them.  Training runs lookup, attention and the gradients of both; serving takes prompts of different
lengths packed one behind the other, keeps their states in a pool, and goes on one token at a time.  The sequences follow a
fixed permutation of the vocabulary, so that the model can learn every next token.
"""
from __future__ import annotations

import argparse
import math
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

from paper_2411_17887_b200 import api  # noqa: E402


class Layer(torch.nn.Module):
    def __init__(self, width: int, heads: int, d_head: int):
        super().__init__()
        self.heads, self.d_head = heads, d_head
        self.into = torch.nn.Parameter(torch.randn(width, 3 * heads * d_head) * width ** -0.5)
        self.back = torch.nn.Parameter(torch.randn(heads * d_head, width) * (heads * d_head) ** -0.5)
        # heads that remember from two tokens to hundreds
        self.register_buffer("log_decay", -torch.exp2(-8.0 * (torch.arange(heads) + 1.0) / heads))

    def qkv(self, x: torch.Tensor):
        x = x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5).to(x.dtype)
        q, k, v = (x @ self.into.to(x.dtype)).unflatten(-1, (3 * self.heads, self.d_head)).split(self.heads, -2)      # views, one beside another
        return torch.nn.functional.silu(q), torch.nn.functional.silu(k), v

    def out(self, x: torch.Tensor, o: torch.Tensor) -> torch.Tensor:
        return x + o.flatten(-2) @ self.back.to(x.dtype)


class LinearLM(torch.nn.Module):
    def __init__(self, vocabulary: int = 500, width: int = 128, heads: int = 4, d_head: int = 32, layers: int = 2):
        super().__init__()
        self.width = width
        self.table = torch.nn.Parameter(torch.randn(vocabulary, width) * width ** -0.5)
        self.layers = torch.nn.ModuleList(Layer(width, heads, d_head) for _ in range(layers))

    def embed(self, ids: torch.Tensor):
        table = self.table.to(torch.bfloat16)
        return table, api.embedding(ids, table, scale=math.sqrt(self.width))

    def forward(self, ids: torch.Tensor, offsets: torch.Tensor | None = None, keep_states: bool = False):
        """Logits of all tokens - ids (batch, tokens), or packed (tokens,) with offsets - and the layers' states after the last."""
        table, x = self.embed(ids)
        states = []
        for layer in self.layers:
            o, last = api.linear_attention(*layer.qkv(x), layer.log_decay, offsets=offsets, output_final_state=keep_states)
            x = layer.out(x, o)
            states.append(last)
        return x @ table.T, states

    @torch.no_grad()
    def step(self, ids: torch.Tensor, pools, slots: torch.Tensor) -> torch.Tensor:
        """Logits after one more token of each sequence; sequence b has entry slots[b] of every layer's pool of states."""
        table, x = self.embed(ids)
        for layer, pool in zip(self.layers, pools):
            x = layer.out(x, api.linear_attention_step(*layer.qkv(x), layer.log_decay, pool, slots=slots))
        return x @ table.T


def sequences(successor: torch.Tensor, batch: int, tokens: int) -> torch.Tensor:
    at = [torch.randint(len(successor), (batch,), device=successor.device)]
    for _ in range(tokens):
        at.append(successor[at[-1]])
    return torch.stack(at, 1)


def train(model: LinearLM, successor: torch.Tensor, steps: int, batch: int = 32, tokens: int = 160) -> list[float]:
    rule = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for _ in range(steps):
        ids = sequences(successor, batch, tokens)
        logits, _ = model(ids[:, :-1])
        loss = torch.nn.functional.cross_entropy(logits.float().flatten(0, 1), ids[:, 1:].flatten())
        rule.zero_grad()
        loss.backward()
        rule.step()
        losses.append(float(loss.detach()))
    return losses


@torch.no_grad()
def serve(model: LinearLM, prompts: list[torch.Tensor], new_tokens: int, entries: int | None = None):
    """The tokens that follow each prompt, and the logits that they were chosen by."""
    device = prompts[0].device
    offsets = torch.tensor([0] + [len(p) for p in prompts], device=device).cumsum(0)
    logits, states = model(torch.cat(prompts), offsets=offsets, keep_states=True)
    entries = entries or len(prompts) + 3
    slots = torch.randperm(entries, device=device)[: len(prompts)].to(torch.int32)
    pools = []
    for state in states:
        pool = state.new_zeros((entries, *state.shape[1:]))
        pool[slots.long()] = state
        pools.append(pool)
    logits = logits[offsets[1:] - 1]
    chosen, seen = [], []
    for _ in range(new_tokens):
        seen.append(logits)
        chosen.append(logits.argmax(-1))
        logits = model.step(chosen[-1], pools, slots)
    return torch.stack(chosen, 1), torch.stack(seen, 1)


def main() -> None:
    args = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    args.add_argument("--steps", type=int, default=160)
    args = args.parse_args()
    torch.manual_seed(0)
    model = LinearLM().cuda()
    successor = torch.randperm(500, device="cuda")
    losses = train(model, successor, args.steps)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {args.steps} steps")
    prompts = [sequences(successor, 1, n)[0] for n in (0, 6, 130, 40)]
    tokens, _ = serve(model, prompts, 20)
    before = torch.cat([torch.stack([p[-1] for p in prompts])[:, None], tokens[:, :-1]], 1)
    print(f"{len(prompts)} prompts, 20 tokens each: {int((tokens == successor[before]).sum())} of {tokens.numel()} follow the permutation")
    if api.linear_attention_status():
        raise SystemExit("a linear-attention call gave up a wait")


if __name__ == "__main__":
    main()
