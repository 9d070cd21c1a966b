"""A small decoder trained with compressed activations: AsiLinear layers, and around them the language-model operators of
paper_2505_05086_amd.lm.

    embedding          token lookup with scaling; its gradient by sorted tokens
    qk_norm_rotate     norms of queries and keys for each head with the position rotation
    token_logprobs_grad  the loss and its gradient in the logits in one pass, the gradient in the logits' place
    AdamW              one launch for all tensors, states in 8 bits, the gradients' norm clipped on the way
    token_logprobs     at the end, the next token and its alternatives, one token at a time over a cache of keys and values

    python examples/finetune_lm.py [--steps 150] [--state-bits 8]

The data is synthetic: every token is followed by the one that a fixed permutation gives.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch
import torch.nn as nn
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_05086_amd as asi  # noqa: E402


class Block(nn.Module):
    def __init__(self, dim: int, heads: int, k_heads: int, ff: int, ranks):
        super().__init__()
        self.heads, self.k_heads, self.head_dim = heads, k_heads, dim // heads
        self.norm1, self.norm2 = nn.RMSNorm(dim), nn.RMSNorm(dim)
        self.qkv = asi.AsiLinear(dim, (heads + 2 * k_heads) * self.head_dim, bias=False, ranks=ranks, seed=1)
        self.out = asi.AsiLinear(dim, dim, bias=False, ranks=ranks, seed=2)
        self.up = asi.AsiLinear(dim, 2 * ff, bias=False, ranks=ranks, seed=3)
        self.down = asi.AsiLinear(ff, dim, bias=False, ranks=ranks, seed=4)
        self.q_gain, self.k_gain = nn.Parameter(torch.ones(self.head_dim)), nn.Parameter(torch.ones(self.head_dim))

    def forward(self, x, cos, sin, positions, cache=None):
        q, k, v = self.qkv(self.norm1(x)).split([n * self.head_dim for n in (self.heads, self.k_heads, self.k_heads)], -1)
        heads = lambda t: t.unflatten(-1, (-1, self.head_dim))  # noqa: E731
        q, k = asi.qk_norm_rotate(heads(q), heads(k), self.q_gain, self.k_gain, cos, sin, positions, heads_first=True)
        v = heads(v).transpose(1, 2)
        if cache is not None:
            if cache:
                k, v = torch.cat((cache[0], k), 2), torch.cat((cache[1], v), 2)
            cache[:] = k, v
        each = self.heads // self.k_heads
        y = F.scaled_dot_product_attention(q, k.repeat_interleave(each, 1), v.repeat_interleave(each, 1), is_causal=q.shape[2] > 1)
        x = x + self.out(y.transpose(1, 2).flatten(2))
        gate, up = self.up(self.norm2(x)).chunk(2, -1)
        return x + self.down(F.silu(gate) * up)


class Decoder(nn.Module):
    """The output layer shares the embedding's table."""

    def __init__(self, vocab: int, dim: int = 128, layers: int = 2, heads: int = 4, k_heads: int = 2, ff: int = 256, length: int = 512,
                 ranks=(8, 16, 32)):
        super().__init__()
        self.table = nn.Parameter(torch.randn(vocab, dim) * dim ** -0.5)
        self.blocks = nn.ModuleList(Block(dim, heads, k_heads, ff, ranks) for _ in range(layers))
        self.norm = nn.RMSNorm(dim)
        cos, sin = asi.rotary_table(length, dim // heads, device="cpu")
        self.register_buffer("cos", cos)
        self.register_buffer("sin", sin)

    def forward(self, tokens, start: int = 0, caches=None):
        positions = torch.arange(start, start + tokens.shape[1], device=tokens.device)
        x = asi.embedding(tokens, self.table, scale=math.sqrt(self.table.shape[1]))
        for n, block in enumerate(self.blocks):
            x = block(x, self.cos, self.sin, positions, None if caches is None else caches[n])
        return self.norm(x) @ self.table.t()


def train_step(model, optimizer, tokens, clip: float = 1.0) -> torch.Tensor:
    """One step on (batch, length) tokens, each position's target the next token.  Nothing waits for the GPU."""
    logits = model(tokens)
    targets = torch.cat((tokens[:, 1:], torch.full_like(tokens[:, :1], asi.lm.IGNORE_INDEX)), 1)
    weights = torch.full(targets.shape, -1.0 / targets[:, 1:].numel(), device=tokens.device)
    with torch.no_grad():
        r = asi.token_logprobs_grad(logits, targets, weights, out=logits)
        loss = (r.logprob * weights).sum()
    optimizer.zero_grad(set_to_none=True)
    # the products behind the logits need the table and their inputs, not the logits: their gradient may take their place
    logits.backward(r.grad)
    norm = torch.linalg.vector_norm(torch.stack([p.grad.norm() for p in model.parameters()]))
    optimizer.step(grad_scale=(clip / norm).clamp(max=1.0).reshape(1))
    return loss


@torch.no_grad()
def generate(model, tokens, count: int, top: int = 3):
    """`count` tokens after (batch, length) tokens, the likeliest each time, and their alternatives' log probabilities."""
    caches = [[] for _ in model.blocks]
    logits, found, scores = model(tokens, 0, caches)[:, -1].contiguous(), [], []
    for n in range(count):
        r = asi.token_logprobs(logits, top=top)
        found.append(r.top_index[:, :1])
        scores.append(r.top_logprob)
        if n + 1 < count:
            logits = model(found[-1], tokens.shape[1] + n, caches)[:, -1]
    return torch.cat(found, 1), torch.stack(scores, 1)


def main(steps: int = 150, state_bits: int = 8, vocab: int = 997, batch: int = 8, length: int = 64, device: str = "cuda", quiet: bool = False):
    torch.manual_seed(0)
    follows = torch.randperm(vocab, device=device)
    model = Decoder(vocab).to(device)
    decayed = [p for p in model.parameters() if p.dim() > 1]
    optimizer = asi.AdamW([{"params": decayed}, {"params": [p for p in model.parameters() if p.dim() < 2], "weight_decay": 0.0}], lr=3e-3,
                          weight_decay=0.01, state_bits=state_bits)
    losses = []
    for step in range(steps):
        tokens = [torch.randint(0, vocab, (batch,), device=device)]
        for _ in range(length - 1):
            tokens.append(follows[tokens[-1]])
        losses.append(train_step(model, optimizer, torch.stack(tokens, 1)))
        if not quiet and step % 25 == 24:
            print(f"step {step + 1}: loss {float(losses[-1]):.4f}", flush=True)
    model.eval()
    prompt = torch.stack((follows[:batch], follows[follows[:batch]]), 1)
    tokens, scores = generate(model, prompt, 8)
    want = [follows[prompt[:, -1]]]
    for _ in range(7):
        want.append(follows[want[-1]])
    share = float((tokens == torch.stack(want, 1)).float().mean())
    if not quiet:
        print(f"{100 * share:.0f} % of the generated tokens follow the rule; log probabilities of the alternatives {scores[0, 0].tolist()}")
    return [float(x) for x in losses], share


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    main(a.steps, a.state_bits)
