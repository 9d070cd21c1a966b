"""The operators of a language model's fine-tuning step that stand beside the compressed layers, as work to be measured.

Kinds of a case:
  score   log probabilities of given tokens with entropy and the top alternatives: scoring, sampling, evaluation
  loss    the same log probabilities and entropy with the gradient of their weighted sum, in one call: a training step's loss
  embed   embedding lookup with scaling
  embed-grad  the table's gradient from the gradient of the looked-up rows
  rotate  norms of queries and keys for each head with the position rotation
  rotate-grad  its backward pass: gradients of queries, keys and the two gains
  adamw   one optimiser step over all tensors of a model, states in 32 or in 8 bits

`run` computes each in its plain form (elementary torch operations in 32 bits), or, where `own` is set, through the
framework's operators.  `exact` states each once more in 64 bits.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
IGNORE = -100
BLOCK = 256                      # elements that share a scale where states are held in 8 bits
LR, BETAS, EPS, DECAY, STEP = 1e-3, (0.9, 0.999), 1e-8, 0.1, 100


# ---- the cases --------------------------------------------------------------------------------------------
def _score(name, rows, vocab, dtype="bf16", top=0, pad=0, scale=1.0, targets=True):
    case = dict(kind="score", rows=rows, vocab=vocab, dtype=dtype, top=top, pad=pad, scale=scale, targets=targets)
    return dict(case, name=name) if name else case


def _loss(name, rows, vocab, dtype="bf16", pad=0, entropy=False, scale=1.0):
    case = dict(kind="loss", rows=rows, vocab=vocab, dtype=dtype, pad=pad, entropy=entropy, scale=scale)
    return dict(case, name=name) if name else case


def _embed(name, tokens, vocab, dim, dtype="bf16", grad=False, grad_dtype="f32", accumulate=False):
    case = dict(kind="embed-grad" if grad else "embed", tokens=tokens, vocab=vocab, dim=dim, dtype=dtype,
                grad_dtype=grad_dtype, accumulate=accumulate)
    return dict(case, name=name) if name else case


def _rotate(name, batch, tokens, q_heads, k_heads, head_dim, rot_dim=0, dtype="bf16", interleaved=False, heads_first=True,
            grad=False):
    case = dict(kind="rotate-grad" if grad else "rotate", batch=batch, tokens=tokens, q_heads=q_heads, k_heads=k_heads,
                head_dim=head_dim, rot_dim=rot_dim or head_dim, dtype=dtype, interleaved=interleaved, heads_first=heads_first)
    return dict(case, name=name) if name else case


def _adamw(name, layers, hidden, ff, vocab=0, dtype="f32", grad_dtype="f32", master=False, bits=32):
    case = dict(kind="adamw", layers=layers, hidden=hidden, ff=ff, vocab=vocab, dtype=dtype, grad_dtype=grad_dtype,
                master=master, bits=bits)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the next token of eight sequences, with the alternatives a sampler looks at: latency counts
        _score("score-next-token", 8, 32000, top=20, targets=False, scale=1.25),
        # scoring a prompt: an odd number of positions, a vocabulary that leaves no row but the first aligned
        _score("score-prompt", 1023, 50001, dtype="f32", top=5),
        # the loss of 8 x 512 tokens and its gradient, a third of the positions without a target
        _loss("loss-step", 4096, 32000),
        # the first thing a training step does: 8 x 512 tokens looked up in a 2048-wide table
        _embed("embed-step", 4096, 32000, 2048),
        # the gradient of that lookup, the whole table written
        _embed("embed-grad-step", 4096, 32000, 2048, grad=True),
        # long documents, added to the gradient that an output layer with the same table has left: few tokens make up most of them
        _embed("embed-grad-add", 32767, 50001, 1000, grad=True, accumulate=True),
        # one token of eight sequences in a decoder: grouped heads, latency counts
        _rotate("rotate-next-token", 8, 1, 32, 4, 64),
        # 8 x 512 tokens of the 2048-wide decoder block, heads first for the attention that follows
        _rotate("rotate-step", 8, 512, 32, 4, 64),
        # long sequences through the backward pass, in 32 bits, with three quarters of each head rotated in neighbouring pairs
        _rotate("rotate-grad-long", 3, 4001, 16, 8, 128, 96, dtype="f32", interleaved=True, heads_first=False, grad=True),
        # a model small enough to be trained on a device: many tensors, few elements
        _adamw("adamw-small", 8, 256, 704, vocab=4096),
        # two decoder blocks in bf16 with 32-bit copies, states in 8 bits
        _adamw("adamw-8bit", 2, 2048, 5632, dtype="bf16", grad_dtype="bf16", master=True, bits=8),
        # a larger part of such a model in 32 bits throughout
        _adamw("adamw-large", 6, 2048, 5632),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges."""
    kind = rng.choice(["score", "loss", "embed", "embed-grad", "rotate", "rotate-grad", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("score", "loss"):
        while True:
            rows, vocab, pad = _log(rng, 1 if kind == "score" else 16, 8192), _log(rng, 500, 200000), rng.choice([0, 0, 8, 13])
            if rows * (vocab + pad) <= 1.3e8:
                break
        scale = rng.choice([1.0, 0.7, 1.25])
        if kind == "score":
            return _score("", rows, vocab, dtype, rng.choice([0, 1, 5, 20, 32]), pad, scale, rng.random() < 0.8)
        return _loss("", rows, vocab, dtype, pad, rng.random() < 0.5, scale)
    if kind in ("embed", "embed-grad"):
        tokens, vocab, dim = _log(rng, 1 if kind == "embed" else 16, 65536), _log(rng, 1000, 130000), _log(rng, 64, 4096)
        while max(tokens, vocab) * dim > 1.4e8:
            tokens, vocab, dim = max(1, tokens // 2), vocab // 2, dim
        accumulate = kind == "embed-grad" and rng.random() < 0.4
        return _embed("", tokens, vocab, dim, dtype, kind == "embed-grad", "f32" if accumulate else rng.choice(["f32", "bf16"]), accumulate)
    if kind in ("rotate", "rotate-grad"):
        head_dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 160, 256])
        k_heads = rng.choice([1, 2, 4, 8])
        q_heads = k_heads * rng.choice([1, 2, 4, 7])
        rot_dim = rng.choice([head_dim, head_dim, head_dim // 2])
        while True:
            batch, tokens = _log(rng, 1, 64), _log(rng, 1, 8192)
            if batch * tokens * (q_heads + k_heads) * head_dim <= 5e7:
                break
        return _rotate("", batch, tokens, q_heads, k_heads, head_dim, rot_dim, dtype, rng.random() < 0.3, rng.random() < 0.5,
                       kind == "rotate-grad")
    while True:
        layers, hidden, ff, vocab = rng.randint(1, 24), _log(rng, 64, 2048), _log(rng, 128, 6000), rng.choice([0, 1000, 4096, 32000])
        if layers * hidden * (4 * hidden + 3 * ff) + vocab * hidden <= 2.5e8:
            break
    master = dtype == "bf16" and rng.random() < 0.6
    return _adamw("", layers, hidden, ff, vocab, dtype, rng.choice([dtype, "f32"]), master, rng.choice([32, 8]))


def _sizes(case):
    """Elements of each tensor: a decoder's projections, feed-forward matrices and gains, and its table."""
    h, f = case["hidden"], case["ff"]
    block = [h * h] * 4 + [h * f] * 3 + [h] * 2
    return block * case["layers"] + ([case["vocab"] * h] if case["vocab"] else []) + [h]


def _distinct(tokens, vocab):
    """Expected number of different tokens where token v has the share log((v + 2) / (v + 1)) / log(vocab + 1)."""
    v = np.arange(vocab, dtype=np.float64)
    p = np.log((v + 2) / (v + 1)) / math.log(vocab + 1)
    return float(-np.expm1(tokens * np.log1p(-p)).sum())


def work(case):
    kind = case["kind"]
    es = BYTES[case["dtype"]]
    if kind == "score":
        t, v = case["rows"], case["vocab"]
        return {"bytes": t * (v * es + 4 + (12 if case["targets"] else 0) + 12 * case["top"]), "flops": 6 * t * v}
    if kind == "loss":
        t, v = case["rows"], case["vocab"]
        return {"bytes": t * (2 * v * es + 20 + (4 if case["entropy"] else 0)), "flops": 10 * t * v}
    if kind == "embed":
        t, d = case["tokens"], case["dim"]
        return {"bytes": t * 8 + _distinct(t, case["vocab"]) * d * es + t * d * es, "flops": t * d}
    if kind == "embed-grad":
        t, d, gs = case["tokens"], case["dim"], BYTES[case["grad_dtype"]]
        written = 2 * _distinct(t, case["vocab"]) if case["accumulate"] else case["vocab"]
        return {"bytes": t * 8 + t * d * es + written * d * gs, "flops": 2 * t * d}
    if kind in ("rotate", "rotate-grad"):
        n = case["batch"] * case["tokens"]
        x = n * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        back = kind == "rotate-grad"
        return {"bytes": x * es * (3 if back else 2) + n * (8 + 4 * case["rot_dim"]), "flops": x * (20 if back else 9)}
    n = sum(_sizes(case))
    param = (8 + es if case["master"] else 2 * es) + BYTES[case["grad_dtype"]]
    return {"bytes": n * (param + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)), "flops": 16 * n}


# ---- inputs -----------------------------------------------------------------------------------------------
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _tokens(g, n, vocab):
    """Token ids whose frequencies fall like natural text's (the r-th most frequent about as 1/r), ids in no order."""
    dev = g.device
    rank = torch.exp(torch.rand(n, generator=g, device=dev) * math.log(vocab + 1)).sub_(1).long().clamp_(0, vocab - 1)
    return torch.randperm(vocab, generator=g, device=dev)[rank]


def _inputs(case, seed):
    dev = _device()
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s = SimpleNamespace(case=case, g=g)
    dtype = DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    kind = case["kind"]
    if kind in ("score", "loss"):
        t, v = case["rows"], case["vocab"]
        full = torch.empty(t, v + case["pad"], dtype=dtype, device=dev).normal_(0.0, 2.5, generator=g)
        s.logits = full[:, :v]
        s.targets = torch.randint(0, v, (t,), generator=g, device=dev)
        likely = torch.arange(t, device=dev) % 2 == 0                 # a trained model's target is often likely
        s.logits[torch.arange(t, device=dev)[likely], s.targets[likely]] = 12.0
        s.logits[:, torch.randint(0, v, (max(1, v // 100),), generator=g, device=dev)] = float("-inf")   # tokens that may not come
        s.logits[torch.arange(t, device=dev), s.targets] = s.logits[torch.arange(t, device=dev), s.targets].clamp_min(-8.0)
        if kind == "loss":
            without = torch.rand(t, generator=g, device=dev) < 1 / 3
            s.targets[without] = IGNORE
            s.a = torch.where(without, 0.0, -1.0 / t * (0.5 + torch.rand(t, generator=g, device=dev)))
            s.b = torch.rand(t, generator=g, device=dev) * (-0.01 / t) if case["entropy"] else None
        elif not case["targets"]:
            s.targets = None
    elif kind in ("embed", "embed-grad"):
        n, v, d = case["tokens"], case["vocab"], case["dim"]
        s.tokens = _tokens(g, n, v)
        s.scale = math.sqrt(d)
        if kind == "embed":
            s.table = torch.empty(v, d, dtype=dtype, device=dev).normal_(0.0, d ** -0.5, generator=g)
        else:
            s.grad_out = randn(n, d).to(dtype)
            s.grad = randn(v, d) if case["accumulate"] else None
    elif kind in ("rotate", "rotate-grad"):
        b, t, hq, hk, dh, rot = (case[k] for k in ("batch", "tokens", "q_heads", "k_heads", "head_dim", "rot_dim"))
        qkv = (randn(b, t, (hq + 2 * hk) * dh) * 1.5).to(dtype)       # one projection's output; the values stay where they are
        s.q = qkv[..., :hq * dh].view(b, t, hq, dh)
        s.k = qkv[..., hq * dh:(hq + hk) * dh].view(b, t, hk, dh)
        s.q_gain, s.k_gain = ((1.0 + 0.2 * randn(dh)).to(dtype) for _ in range(2))
        length = 16384
        freq = 10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        angle = torch.arange(length, device=dev, dtype=torch.float64)[:, None] * freq
        s.cos, s.sin = angle.cos().float(), angle.sin().float()
        first = torch.randint(0, length - t + 1, (b, 1), generator=g, device=dev)
        s.positions = first + torch.arange(t, device=dev)
        if kind == "rotate-grad":
            shape = (lambda h: (b, h, t, dh)) if case["heads_first"] else (lambda h: (b, t, h, dh))
            s.grad_q, s.grad_k = randn(*shape(hq)).to(dtype), randn(*shape(hk)).to(dtype)
    else:
        sizes = _sizes(case)
        starts = np.concatenate([[0], np.cumsum([-(-n // BLOCK) * BLOCK for n in sizes])])
        total = int(starts[-1])
        s.starts, s.sizes = starts[:-1], sizes
        # one buffer of each sort holds the tensors of the model, each from a multiple of 256 elements on; what lies between them is zero
        s.inside = torch.zeros(total, dtype=torch.bool, device=dev)
        for at, n in zip(s.starts, sizes):
            s.inside[at:at + n] = True
        value = (randn(total) * 0.02).masked_fill_(~s.inside, 0)
        s.param = value.to(dtype)
        s.master = value if case["master"] else None
        s.grad = (randn(total) * torch.exp(randn(total)) * 1e-3).masked_fill_(~s.inside, 0).to(DTYPES[case["grad_dtype"]])
        s.clip = torch.full((1,), 0.75, device=dev)
        avg = (randn(total) * 3e-4).masked_fill_(~s.inside, 0)
        sq = (torch.exp(randn(total) - 13.5)).masked_fill_(~s.inside, 0)
        if case["bits"] == 32:
            s.avg, s.sq = avg, sq
        else:
            s.avg, s.avg_scale = _to_8bit(avg)
            s.sq, s.sq_scale = _to_8bit(sq.sqrt_())
    return s


def _views(flat, s, per=1):
    return [flat[at // per:at // per + -(-n // per)] for at, n in zip(s.starts.tolist(), s.sizes)]


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "adamw" and own:
        from paper_2505_05086_amd import AdamW
        params = [torch.nn.Parameter(p) for p in _views(s.param, s)]
        grads = _views(s.grad, s)
        s.optimizer = AdamW(params, lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, state_bits=case["bits"], master=case["master"])
        kept = {"exp_avg": (s.avg, 1), "exp_avg_sq" if case["bits"] == 32 else "exp_avg_sqrt": (s.sq, 1)}
        if case["bits"] == 8:
            kept.update(exp_avg_scale=(s.avg_scale, BLOCK), exp_avg_sqrt_scale=(s.sq_scale, BLOCK))
        if case["master"]:
            kept["master"] = (s.master, 1)
        views = {k: _views(t, s, per) for k, (t, per) in kept.items()}
        s.grads = None if s.grad.dtype == s.param.dtype else grads     # a parameter's own gradient has its type
        for i, p in enumerate(params):
            if s.grads is None:
                p.grad = grads[i]
            s.optimizer.state[p].update({k: v[i] for k, v in views.items()})
        s.optimizer.param_groups[0]["step"] = STEP - 1
    return s


# ---- plain forms ------------------------------------------------------------------------------------------
def _stats(x, scale):
    z = x.float() * scale
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    s = e.sum(-1, keepdim=True)
    return z, e / s, (top + torch.log(s))


def _entropy(z, p, lse):
    return -(torch.where(p > 0, z - lse, 0.0) * p).sum(-1)


def _plain_score(s):
    c = s.case
    z, p, lse = _stats(s.logits, c["scale"])
    out = {"entropy": _entropy(z, p, lse)}
    if s.targets is not None:
        out["logprob"] = (z.gather(1, s.targets[:, None]) - lse)[:, 0]
    if c["top"]:
        # equal values by their index: a key that holds both, the value's bits in an order of whole numbers above the index
        bits = s.logits.float().add(0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (order << 32) + (c["vocab"] - torch.arange(c["vocab"], device=z.device))
        best = key.topk(min(c["top"], c["vocab"]), dim=-1).values
        out["top_index"] = c["vocab"] - (best & 0xFFFFFFFF)
        out["top_logprob"] = z.gather(1, out["top_index"]) - lse
    return out


def _plain_loss(s):
    c = s.case
    z, p, lse = _stats(s.logits, c["scale"])
    given = s.targets != IGNORE
    at = torch.where(given, s.targets, 0)[:, None]
    out = {"logprob": torch.where(given, (z.gather(1, at) - lse)[:, 0], 0.0)}
    a = torch.where(given, s.a, 0.0)[:, None]
    d = -p * a
    d.scatter_add_(1, at, a)
    if s.b is not None:
        out["entropy"] = _entropy(z, p, lse)
        d -= s.b[:, None] * p * (torch.where(p > 0, z - lse, 0.0) + out["entropy"][:, None])
    out["grad"] = (d * c["scale"]).to(s.logits.dtype)
    return out


def _plain_embed(s):
    return (s.table[s.tokens].float() * s.scale).to(s.table.dtype)


def _plain_embed_grad(s):
    c = s.case
    grad = s.grad if c["accumulate"] else torch.zeros(c["vocab"], c["dim"], device=s.tokens.device)
    grad.index_add_(0, s.tokens, s.grad_out.float() * s.scale)
    return grad.to(DTYPES[c["grad_dtype"]])


def _turn(n, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    a, b = (n[..., 0:rot:2], n[..., 1:rot:2]) if interleaved else (n[..., :rot // 2], n[..., rot // 2:rot])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((ya, yb), -1).flatten(-2) if interleaved else torch.cat((ya, yb), -1)
    return torch.cat((y, n[..., rot:]), -1)


def _plain_rotate(s):
    c = s.case
    cos, sin = s.cos[s.positions][:, :, None], s.sin[s.positions][:, :, None]

    def one(x, gain):
        x = x.float()
        n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain.float()
        y = _turn(n, cos, sin, c["interleaved"]).to(gain.dtype)
        return y.transpose(1, 2).contiguous() if c["heads_first"] else y

    return {"q": one(s.q, s.q_gain), "k": one(s.k, s.k_gain)}


def _plain_rotate_grad(s):
    c = s.case
    cos, sin = s.cos[s.positions][:, :, None], s.sin[s.positions][:, :, None]

    def one(x, gain, dy):
        dy = (dy.transpose(1, 2) if c["heads_first"] else dy).float()
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        dn = _turn(dy, cos, -sin, c["interleaved"])
        xr = x * r
        wd = dn * gain.float()
        dx = r * (wd - xr * (wd * xr).mean(-1, keepdim=True))
        return dx.to(gain.dtype), (dn * xr).sum((0, 1, 2))

    (dq, dqg), (dk, dkg) = one(s.q, s.q_gain, s.grad_q), one(s.k, s.k_gain, s.grad_k)
    return {"q": dq, "k": dk, "q_gain": dqg, "k_gain": dkg}


_SMALL = 2.0 ** -126             # below it a scale has no reciprocal in 32 bits: its block is held as zeros


def _to_8bit(x):
    """Blocks of 256 values as 8-bit floats (4 bits of exponent, 3 of mantissa) and a 32-bit scale that takes the largest to 448."""
    blocks = x.view(-1, BLOCK)
    scale = blocks.abs().amax(-1) * (1.0 / 448.0)
    inverse = torch.where(scale >= _SMALL, scale.reciprocal(), 0.0)
    scale = torch.where(scale >= _SMALL, scale, 0.0)
    return (blocks * inverse[:, None]).to(torch.float8_e4m3fn).flatten(), scale


def _from_8bit(code, scale):
    return (code.float().view(-1, BLOCK) * scale[:, None]).flatten()


def _plain_adamw(s):
    c = s.case
    b1, b2 = BETAS
    step = STEP
    g = s.grad.float() * s.clip
    avg, root = (s.avg, None) if c["bits"] == 32 else (_from_8bit(s.avg, s.avg_scale), _from_8bit(s.sq, s.sq_scale))
    sq = s.sq if root is None else root * root
    avg = avg * b1 + g * (1 - b1)
    sq = sq * b2 + (g * g) * (1 - b2)
    root = sq.sqrt()
    update = avg / (root * (1.0 / math.sqrt(1 - b2 ** step)) + EPS)
    p = s.param.float() if s.master is None else s.master
    p = p * (1 - LR * DECAY) - update * (LR / (1 - b1 ** step))
    out = {"param": s.param.copy_(p)}
    if s.master is not None:
        out["master"] = s.master.copy_(p)
    if c["bits"] == 32:
        return dict(out, avg=s.avg.copy_(avg), sq=s.sq.copy_(sq))
    s.avg, s.avg_scale = _to_8bit(avg)
    code, s.sq_scale = _to_8bit(root)
    # a positive root is never held as zero: the next step divides by it
    least = torch.full_like(root, 2.0 ** -9).to(torch.float8_e4m3fn)
    held = (root > 0) & (s.sq_scale.repeat_interleave(BLOCK) > 0)
    s.sq = torch.where(held & (code.float() == 0), least.view(torch.uint8), code.view(torch.uint8)).view(torch.float8_e4m3fn)
    return dict(out, avg=s.avg, avg_scale=s.avg_scale, sqrt=s.sq, sqrt_scale=s.sq_scale)


PLAIN = {"score": _plain_score, "loss": _plain_loss, "embed": _plain_embed, "embed-grad": _plain_embed_grad,
         "rotate": _plain_rotate, "rotate-grad": _plain_rotate_grad, "adamw": _plain_adamw}


# ---- the framework's operators ----------------------------------------------------------------------------
def _own(s):
    import paper_2505_05086_amd as asi
    c = s.case
    kind = c["kind"]
    if kind == "score":
        r = asi.token_logprobs(s.logits, s.targets, top=min(c["top"], c["vocab"]), scale=c["scale"])
        out = {"entropy": r.entropy}
        if s.targets is not None:
            out["logprob"] = r.logprob
        if c["top"]:
            out.update(top_index=r.top_index, top_logprob=r.top_logprob)
        return out
    if kind == "loss":
        r = asi.token_logprobs_grad(s.logits, s.targets, s.a, s.b, scale=c["scale"], ignore_index=IGNORE)
        out = {"logprob": r.logprob, "grad": r.grad}
        return out if s.b is None else dict(out, entropy=r.entropy)
    if kind == "embed":
        return asi.embedding(s.tokens, s.table, scale=s.scale)
    if kind == "embed-grad":
        return asi.embedding_grad(s.tokens, s.grad_out, c["vocab"], scale=s.scale, dtype=DTYPES[c["grad_dtype"]], out=s.grad,
                                  accumulate=c["accumulate"])
    if kind == "rotate":
        q, k = asi.qk_norm_rotate(s.q, s.k, s.q_gain, s.k_gain, s.cos, s.sin, s.positions, eps=1e-6,
                                  interleaved=c["interleaved"], heads_first=c["heads_first"])
        return {"q": q, "k": k}
    if kind == "rotate-grad":
        dq, dk, dqg, dkg = asi.qk_norm_rotate_grad(s.q, s.k, s.q_gain, s.k_gain, s.cos, s.sin, s.grad_q, s.grad_k, s.positions,
                                                   eps=1e-6, interleaved=c["interleaved"], heads_first=c["heads_first"])
        return {"q": dq, "k": dk, "q_gain": dqg, "k_gain": dkg}
    s.optimizer.param_groups[0]["step"] = STEP - 1
    s.optimizer.step(grad_scale=s.clip, grads=s.grads)
    out = {"param": s.param}
    if s.master is not None:
        out["master"] = s.master
    if c["bits"] == 32:
        return dict(out, avg=s.avg, sq=s.sq)
    return dict(out, avg=s.avg, avg_scale=s.avg_scale, sqrt=s.sq, sqrt_scale=s.sq_scale)


def run(state):
    return _own(state) if own else PLAIN[state.case["kind"]](state)


# ---- 64 bits ----------------------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("score", "loss"):
        return _exact_logits(s)
    if kind == "embed":
        return s.table.index_select(0, s.tokens).double().mul(s.scale)
    if kind == "embed-grad":
        total = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device=s.tokens.device)
        rows = s.grad_out.double()
        for part in torch.arange(len(s.tokens), device=rows.device).split(4096):
            total.index_put_((s.tokens[part],), rows[part], accumulate=True)
        total *= s.scale
        return total if s.grad is None else total + s.grad.double()
    if kind in ("rotate", "rotate-grad"):
        return _exact_rotate(s)
    return _exact_adamw(s)


def _exact_logits(s):
    """Row by row in parts, by the definitions p = exp(z) / sum exp(z) and -sum p log p."""
    c = s.case
    keep = {}
    for part in torch.arange(c["rows"], device=s.logits.device).split(max(1, 20_000_000 // c["vocab"])):
        x = s.logits[part].double()
        logp = torch.log_softmax(x * c["scale"], -1)
        entropy = torch.special.entr(logp.exp()).sum(-1)
        row = {}
        if c["kind"] == "score" or c["entropy"]:
            row["entropy"] = entropy
        if s.targets is not None:
            y = s.targets[part]
            row["logprob"] = torch.where(y >= 0, logp.gather(1, y.clamp_min(0)[:, None])[:, 0], 0.0)
        if c["kind"] == "score" and c["top"]:
            order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :c["top"]]
            row.update(top_index=order, top_logprob=logp.gather(1, order))
        if c["kind"] == "loss":
            hot = torch.zeros_like(x)
            hot[torch.arange(len(y), device=x.device), y.clamp_min(0)] = (y >= 0).double()
            p = logp.exp()
            a = (s.a[part].double() * (y >= 0))[:, None]
            d = a * (hot - p)
            if s.b is not None:
                d += s.b[part].double()[:, None] * (torch.special.entr(p) - p * entropy[:, None])
            row["grad"] = d * c["scale"]
        for k, v in row.items():
            keep.setdefault(k, []).append(v)
    return {k: torch.cat(v) for k, v in keep.items()}


def _exact_rotate(s):
    """Each pair as a complex number, turned by multiplication."""
    c = s.case
    rot = c["rot_dim"]
    phase = torch.complex(s.cos[s.positions].double(), s.sin[s.positions].double())[:, :, None]

    def turn(n, phase):
        head = n[..., :rot].unflatten(-1, (-1, 2) if c["interleaved"] else (2, -1))
        axis = -1 if c["interleaved"] else -2
        z = torch.complex(head.select(axis, 0).contiguous(), head.select(axis, 1).contiguous()) * phase
        return torch.cat((torch.stack((z.real, z.imag), axis).flatten(-2), n[..., rot:]), -1)

    def unit(x):
        x = x.double()
        return x, (x.square().sum(-1, keepdim=True) / c["head_dim"] + 1e-6).sqrt()

    out = {}
    for name, x, gain in (("q", s.q, s.q_gain), ("k", s.k, s.k_gain)):
        x, size = unit(x)
        if c["kind"] == "rotate":
            y = turn(x / size * gain.double(), phase)
            out[name] = y.transpose(1, 2) if c["heads_first"] else y
        else:
            dy = (s.grad_q if name == "q" else s.grad_k).double()
            dn = turn(dy.transpose(1, 2) if c["heads_first"] else dy, phase.conj())
            u = x / size
            out[name + "_gain"] = (dn * u).flatten(0, 2).sum(0)
            w = dn * gain.double()
            out[name] = (w - u * ((u * w).sum(-1, keepdim=True) / c["head_dim"])) / size
    return out


def _exact_adamw(s):
    c = s.case
    b1, b2 = BETAS
    wide = lambda code, scale: code.double().view(-1, BLOCK).mul(scale.double()[:, None]).flatten()  # noqa: E731
    g = s.grad.double() * s.clip.double()
    m, v = (s.avg.double(), s.sq.double()) if c["bits"] == 32 else (wide(s.avg, s.avg_scale), wide(s.sq, s.sq_scale).square())
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g.square()
    mean, var = m / (1 - b1 ** STEP), v / (1 - b2 ** STEP)
    p = (s.param if s.master is None else s.master).double()
    p = p - LR * DECAY * p - LR * mean / (var.sqrt() + EPS)
    out = {"param": p}
    if s.master is not None:
        out["master"] = p
    if c["bits"] == 32:
        return dict(out, avg=m, sq=v)
    for name, x in (("avg", m), ("sqrt", v.sqrt())):
        size = x.view(-1, BLOCK).abs().amax(-1) / 448
        part = x.view(-1, BLOCK) / torch.where(size > 0, size, 1.0)[:, None]
        # to the nearest of the values that 4 bits of exponent and 3 of mantissa have, the even one of two that are as near
        step = torch.exp2(torch.floor(torch.log2(part.abs().clamp_min(2.0 ** -6))) - 3)
        held = torch.round(part / step) * step
        if name == "sqrt":
            held = torch.where((part > 0) & (held == 0), 2.0 ** -9, held)
        out.update({name: held.flatten(), name + "_scale": size})
    return out
