"""The operators that keep no logits and no mask together, as examples/finetune_lm.py uses them: a training run with dropout, and one
step's gradients against the same network with the masks drawn in numpy."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2505_05086_amd as asi
from test_gpu_lm_dropout import kept

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "finetune_lm.py")
    spec = importlib.util.spec_from_file_location("finetune_lm", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_a_training_run_with_dropout():
    losses, share = _example().main(steps=30, quiet=True, dropout=0.1)
    assert len(losses) == 30 and all(math.isfinite(x) for x in losses) and 0 <= share <= 1


def _mask(shape, p, seed, offset):
    n = math.prod(shape)
    return torch.from_numpy(kept(0, n, p, seed, offset)).cuda().view(shape).double() * (65536 / (65536 - round(p * 65536)))


def test_one_step_with_dropout_against_64_bits():
    m = _example()
    torch.manual_seed(2)
    p = 0.2
    model = m.Decoder(499, ranks=(4, 16, 24), dropout=p).cuda()
    model.seed.fill_(77)
    tokens = torch.randint(0, 499, (4, 33), device="cuda")
    targets = torch.cat((tokens[:, 1:], torch.full_like(tokens[:, :1], -100)), 1)
    loss = -asi.linear_logprobs(model.hidden(tokens), model.table, targets).logprob.sum() / (4 * 32)
    loss.backward()
    w = {k: v.detach().double().requires_grad_(True) for k, v in model.named_parameters()}

    def rms(x, gain, eps=torch.finfo(torch.float32).eps):
        return x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain

    t, layers = tokens.shape[1], len(model.blocks)
    x = w["table"][tokens] * math.sqrt(model.table.shape[1])
    x = x * _mask(x.shape, p, 77, 2 * layers)
    for n, block in enumerate(model.blocks):
        of = lambda name: w[f"blocks.{n}.{name}"]  # noqa: E731,B023
        h, hk, d = block.heads, block.k_heads, block.head_dim
        qkv = rms(x, of("norm1.weight")) @ of("qkv.weight").t()
        q, k, v = (y.unflatten(-1, (-1, d)).transpose(1, 2) for y in qkv.split([h * d, hk * d, hk * d], -1))

        def turned(y, gain):
            y = rms(y, gain, 1e-6)
            c, s = model.cos[:t].double(), model.sin[:t].double()
            lo, hi = y[..., :d // 2], y[..., d // 2:]  # noqa: B023
            return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)

        q, k = turned(q, of("q_gain")), turned(k, of("k_gain"))
        k, v = k.repeat_interleave(h // hk, 1), v.repeat_interleave(h // hk, 1)
        a = (q @ k.transpose(2, 3).contiguous() / math.sqrt(d)).masked_fill(torch.ones(t, t, dtype=torch.bool, device="cuda").triu(1), -math.inf).softmax(-1)
        x = x + (a @ v).transpose(1, 2).flatten(2) @ of("out.weight").t() * _mask(x.shape, p, 77, 2 * n)
        gate, up = (rms(x, of("norm2.weight")) @ of("up.weight").t()).chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ of("down.weight").t() * _mask(x.shape, p, 77, 2 * n + 1)
    logp = torch.log_softmax(rms(x, w["norm.weight"]) @ w["table"].t(), -1)
    want = -logp[:, :-1].gather(-1, tokens[:, 1:, None]).sum() / (4 * 32)
    want.backward()
    # a chain of about ten products of up to 499 terms, each within 499 * 2^-24 of its norm; the compressed layers' weight gradients are the
    # method's approximation
    assert abs(float(loss) - float(want)) < 1e-4 * float(want)
    for name, q in model.named_parameters():
        if any(part in name for part in ("qkv", "out", "up", "down")):
            continue
        off = (q.grad.double() - w[name].grad).norm() / w[name].grad.norm()
        assert off < 10 * 499 * 2.0 ** -24, (name, float(off))
