"""The operators together, as examples/finetune_lm.py uses them: a training run, and one step's gradients against the
same network in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "finetune_lm.py")
    spec = importlib.util.spec_from_file_location("finetune_lm", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_run_learns(bits):
    losses, share = _example().main(steps=120, state_bits=bits, quiet=True)
    assert losses[0] > math.log(997)                     # no better than a guess: the shared table first predicts the token itself
    assert losses[-1] < 0.5 * math.log(997)
    assert share > 0.5


def _plain(model, tokens, weights):
    """The network's loss in 64 bits by elementary operations, as a function of the model's own parameters."""
    p = {k: v.detach().double().requires_grad_(True) for k, v in model.named_parameters()}

    def rms(x, w):
        return x / (x.square().mean(-1, keepdim=True) + torch.finfo(torch.float32).eps).sqrt() * w

    x = p["table"][tokens] * math.sqrt(model.table.shape[1])
    b, t = tokens.shape
    for n, block in enumerate(model.blocks):
        w = lambda name: p[f"blocks.{n}.{name}"]  # noqa: E731,B023
        h, hk, d = block.heads, block.k_heads, block.head_dim
        qkv = rms(x, w("norm1.weight")) @ w("qkv.weight").t()
        q, k, v = (y.unflatten(-1, (-1, d)).transpose(1, 2) for y in qkv.split([h * d, hk * d, hk * d], -1))

        def turned(y, gain):
            y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain
            c, s = model.cos[:t].double(), model.sin[:t].double()
            lo, hi = y[..., :d // 2], y[..., d // 2:]
            return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)

        q, k = turned(q, w("q_gain")), turned(k, w("k_gain"))
        k, v = k.repeat_interleave(h // hk, 1), v.repeat_interleave(h // hk, 1)
        a = q @ k.transpose(2, 3).contiguous() / math.sqrt(d)
        a = a.masked_fill(torch.ones(t, t, dtype=torch.bool, device=a.device).triu(1), -math.inf).softmax(-1)
        x = x + (a @ v).transpose(1, 2).flatten(2) @ w("out.weight").t()
        gate, up = (rms(x, w("norm2.weight")) @ w("up.weight").t()).chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ w("down.weight").t()
    logits = rms(x, p["norm.weight"]) @ p["table"].t()
    targets = torch.cat((tokens[:, 1:], tokens[:, :1]), 1)
    logp = torch.log_softmax(logits, -1).gather(-1, targets[..., None])[..., 0]
    loss = (logp * weights)[:, :-1].sum()
    loss.backward()
    return loss.detach(), p


def test_one_step_against_64_bits():
    m = _example()
    torch.manual_seed(1)
    model = m.Decoder(499, ranks=(4, 16, 24)).cuda()
    with torch.no_grad():
        for b in model.blocks:
            b.q_gain.uniform_(0.5, 1.5)
            b.k_gain.uniform_(0.5, 1.5)
    tokens = torch.randint(0, 499, (4, 33), device="cuda")

    class Keep:                                  # in the optimiser's place: what would be applied
        def zero_grad(self, set_to_none):
            for p in model.parameters():
                p.grad = None

        def step(self, grad_scale):
            self.scale = float(grad_scale)

    keep = Keep()
    loss = m.train_step(model, keep, tokens)
    want, p = _plain(model, tokens, -1.0 / (4 * 32))
    assert abs(float(loss) - float(want)) < 1e-4 * abs(float(want))
    # the weight gradients of the compressed layers are the method's approximation; everything else is exact up to fp32: a chain of about
    # ten products of up to 256 terms, each within 256 * 2^-24 of its norm
    for name, q in model.named_parameters():
        if any(part in name for part in ("qkv", "out", "up", "down")):
            continue
        off = (q.grad.double() - p[name].grad).norm() / p[name].grad.norm()
        assert off < 10 * 256 * 2.0 ** -24, (name, float(off))
    assert 0 < keep.scale <= 1
