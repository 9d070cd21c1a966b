"""The language-model operators (include/asi_lm.h) against their definitions in 64 bits.

U = 2^-24 is half an fp32 ulp.  Bounds are a count of roundings times U times the magnitudes that are added up, and
2^-8 of the value (half the spacing of bf16's 7 mantissa bits) where a result is rounded to bf16; each is derived where it stands.
"""
import copy
import math

import numpy as np
import pytest
import torch

import paper_2505_05086_amd as asi

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _close(got, want, bound, what):
    """|got - want| <= bound entry by entry; where `want` is not finite the two are equal."""
    got, want = got.double(), want.double()
    bound = torch.as_tensor(bound, dtype=torch.float64, device=got.device).expand_as(want)
    assert got.shape == want.shape, what
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    assert torch.equal(got[odd].nan_to_num(7.0), want[odd].nan_to_num(7.0)), f"{what}: infinities"
    off = ((got - want).abs() - bound)[~odd]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{what}: {float(off.max()):.3g} over its bound"


def _round(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


# ---- token log probabilities ------------------------------------------------------------------------------
def _logits(rows, vocab, dtype, seed, pad=0, shift=0, spread=3.0):
    """Rows `pad` elements apart from each other's end, the first one `shift` elements into its storage."""
    flat = torch.empty(rows * (vocab + pad) + shift, device="cuda").normal_(0, spread, generator=_gen(seed)).to(dtype)
    return flat[shift:].as_strided((rows, vocab), (vocab + pad, 1))


def _definition(x, targets, scale, ignore):
    """logprob, entropy, p, log p of every row in 64 bits; rows of nothing but -infinity as the header says."""
    z = x.double() * scale
    empty = (x == -INF).all(-1)
    logp = torch.log_softmax(torch.where(empty[:, None], 0.0, z), -1)
    p = logp.exp()
    entropy = torch.special.entr(p).sum(-1)
    entropy[empty], p[empty], logp[empty] = 0.0, 0.0, -INF
    logprob = None
    if targets is not None:
        fine = (targets >= 0) & (targets < x.shape[1])
        logprob = logp.gather(1, torch.where(fine, targets, 0)[:, None])[:, 0]
        logprob = torch.where(fine, logprob, NAN)
        logprob[targets == ignore] = 0.0
    return logprob, entropy, p, logp


def _order(x, top):
    """Indices of the largest, equal ones by ascending index, NaN before everything."""
    key = torch.where(torch.isnan(x), INF, x.double())
    key = torch.stack((torch.isnan(x).double(), key), -1).cpu().numpy()
    return torch.from_numpy(np.stack([np.lexsort((np.arange(len(k)), -k[:, 1], -k[:, 0]))[:top] for k in key])).to(x.device)


def _value_bound(x, scale):
    # a difference, its product and the logarithm's: 8 roundings of the largest |z|; a sum of up to 2^11 terms a thread, of which
    # no more than 128 in a row change its last bit, and its joining
    finite = torch.where(torch.isfinite(x), x, 0).double().abs().amax(-1) * scale
    return U * (8 * finite + 256)


SIZES = [(1, 1), (3, 2), (5, 7), (2, 63), (4, 64), (3, 65), (7, 257), (2, 1000), (3, 4095), (2, 4096), (3, 8193), (2, 32000), (3, 50001), (1, 131075),
         (1, 200000), (2, 40000), (2, 80000), (2100, 3001), (300, 17001), (70, 66000)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_token_logprobs(size, dtype):
    rows, vocab = size
    for k, (pad, shift, scale) in enumerate([(0, 0, 1.0), (8, 0, 0.7), (3, 1, 1.3)]):
        x = _logits(rows, vocab, DTYPES[dtype], 100 * vocab + k, pad, shift)
        targets = torch.randint(0, vocab, (rows,), generator=_gen(k), device="cuda")
        targets[0] = vocab - 1
        if rows > 1:
            targets[1] = -100
        top = min(vocab, (0, 1, 20)[k])
        r = asi.token_logprobs(x, targets, top=top, scale=scale)
        logprob, entropy, _, logp = _definition(x, targets, scale, -100)
        bound = _value_bound(x, scale)
        _close(r.logprob, logprob, bound, "logprob")
        # entropy = log s - scale w / s: w's terms are as many roundings of magnitudes of up to |z|
        _close(r.entropy, entropy, bound + U * 256 * entropy.clamp_min(1.0), "entropy")
        if top:
            index = _order(x, top)
            assert torch.equal(r.top_index, index)
            _close(r.top_logprob, logp.gather(1, index), bound[:, None], "top_logprob")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("vocab,top", [(1, 1), (5, 5), (40, 40), (300, 64), (1500, 33), (5000, 64), (32000, 20), (40001, 7)])
def test_top_alternatives_with_equal_logits(vocab, top, dtype):
    g = _gen(vocab)
    rows = [torch.randint(-3, 3, (vocab,), generator=g, device="cuda").float(),              # few values, many of each
            torch.zeros(vocab, device="cuda"),                                               # all equal
            torch.where(torch.rand(vocab, generator=g, device="cuda") < 0.5, 0.0, -0.0),     # zeros of both signs are equal
            torch.full((vocab,), -INF, device="cuda"),                                       # fewer than `top` that may come
            torch.arange(vocab, device="cuda").float() / 64,                                 # ascending
            torch.randn(vocab, generator=g, device="cuda")]
    rows[3][vocab // 2] = 1.0
    rows[5][torch.rand(vocab, generator=g, device="cuda") < 0.1] = torch.finfo(torch.bfloat16).min
    x = torch.stack(rows).to(DTYPES[dtype])
    r = asi.token_logprobs(x, top=top)
    index = _order(x, top)
    assert torch.equal(r.top_index, index)
    _close(r.top_logprob, _definition(x, None, 1.0, -100)[3].gather(1, index), _value_bound(torch.where(x > -1e30, x, 0), 1.0)[:, None], "top")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("vocab", [9, 1000, 33333])
def test_logits_that_are_not_finite(vocab, dtype):
    x = _logits(6, vocab, DTYPES[dtype], vocab)
    x[0] = -INF                                          # an empty row
    x[1, 1:] = -INF                                      # one token may come
    x[2, vocab // 2] = NAN
    x[3, vocab - 1] = INF
    x[4] = torch.finfo(DTYPES[dtype]).min                # masked by the type's lowest value, all of them
    x[5, ::2] = torch.finfo(DTYPES[dtype]).min
    targets = torch.tensor([3, 0, 1, 2, vocab - 1, 1], device="cuda")
    a, b = torch.full((6,), -0.5, device="cuda"), torch.full((6,), 0.25, device="cuda")
    r = asi.token_logprobs(x, targets, top=3)
    d = asi.token_logprobs_grad(x, targets, a, b)
    for got in (r, d):
        assert got.logprob.tolist()[0] == -INF and got.entropy[0] == 0
        assert abs(float(got.logprob[1])) == 0 and abs(float(got.entropy[1])) == 0
        assert torch.isnan(got.logprob[2:4]).all() and torch.isnan(got.entropy[2:4]).all()
        assert abs(float(got.logprob[4]) + math.log(vocab)) < 300 * U
        assert abs(float(got.entropy[4]) - math.log(vocab)) < 300 * U
        assert torch.isfinite(got.logprob[5]) and torch.isfinite(got.entropy[5])
    assert torch.equal(r.top_index[0], torch.arange(3, device="cuda")) and (r.top_logprob[0] == -INF).all()
    assert r.top_index[1].tolist() == [0, 1, 2] and r.top_logprob[1].tolist() == [0.0, -INF, -INF]
    assert r.top_index[2, 0] == vocab // 2 and torch.isnan(r.top_logprob[2:4]).all() and r.top_index[3, 0] == vocab - 1
    assert r.top_index[4].tolist() == [0, 1, 2]
    grad = d.grad.float()
    assert (grad[0] == 0).all() and (grad[1] == 0).all()
    assert torch.isnan(grad[2:4]).all()
    assert torch.isfinite(grad[4:]).all()
    assert (grad[5, ::2] == 0).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_token_logprobs_grad(size, dtype):
    rows, vocab = size
    for k, (pad, shift, scale) in enumerate([(0, 0, 1.0), (8, 0, 0.7), (3, 1, 1.3)]):
        x = _logits(rows, vocab, DTYPES[dtype], 100 * vocab + k, pad, shift)
        targets = torch.randint(0, vocab, (rows,), generator=_gen(k), device="cuda")
        a = torch.randn(rows, generator=_gen(9 + k), device="cuda")
        b = torch.randn(rows, generator=_gen(19 + k), device="cuda") if k != 1 else None
        targets[0] = 0
        if rows > 1:
            targets[1] = -100
        r = asi.token_logprobs_grad(x, targets, a, b, scale=scale)
        logprob, entropy, p, logp = _definition(x, targets, scale, -100)
        bound = _value_bound(x, scale)
        _close(r.logprob, logprob, bound, "logprob")
        _close(r.entropy, entropy, bound + U * 256 * entropy.clamp_min(1.0), "entropy")
        wa = torch.where(targets == -100, 0.0, a.double())[:, None]
        wb = (torch.zeros_like(a) if b is None else b).double()[:, None]
        hot = torch.zeros_like(p)
        hot[torch.arange(rows), targets.clamp_min(0)] = (targets >= 0).double()
        logp = logp.clamp_min(-1e4)
        want = scale * (wa * (hot - p) - wb * p * (logp + entropy[:, None]))
        # p's relative error is that of exp(log p): the values' bound and the quotient's roundings; log p + entropy is off by the two
        # values' bounds
        size_of = p * (wa.abs() + wb.abs() * (logp.abs() + entropy[:, None] + 1))
        err = scale * ((2 * bound[:, None] + 16 * U) * size_of + U * 256 * wb.abs() * p * entropy[:, None].clamp_min(1.0) + 4 * U * hot * wa.abs())
        _close(r.grad, want, err + _round(x.dtype) * want.abs() * 1.01 + 1e-38, "grad")
        # in place: the same bits
        mine = x.clone(memory_format=torch.preserve_format) if pad == 0 and shift == 0 else _logits(rows, vocab, x.dtype, 100 * vocab + k, pad, shift)
        again = asi.token_logprobs_grad(mine, targets, a, b, scale=scale, out=mine)
        assert again.grad.data_ptr() == mine.data_ptr() and torch.equal(mine, r.grad)
        # a result whose rows lie otherwise
        other = torch.empty(rows * (vocab + 5) + 3, dtype=x.dtype, device="cuda")[3:].as_strided((rows, vocab), (vocab + 5, 1))
        assert torch.equal(asi.token_logprobs_grad(x, targets, a, b, scale=scale, out=other).grad, r.grad)


@pytest.mark.parametrize("vocab", [700, 20000, 150000])
def test_alternatives_beside_many_infinities(vocab):
    x = _logits(2, vocab, torch.float32, vocab)
    x[:, torch.randperm(vocab, generator=_gen(1), device="cuda")[:vocab // 3]] = INF
    x[1, torch.randperm(vocab, generator=_gen(2), device="cuda")[:5]] = NAN
    r = asi.token_logprobs(x, top=20)
    assert torch.equal(r.top_index, _order(x, 20)) and torch.isnan(r.top_logprob).all()


def test_targets_out_of_range_give_nan():
    x = _logits(4, 1000, torch.float32, 3)
    targets = torch.tensor([-1, 1000, 999, -100], device="cuda")
    a = torch.ones(4, device="cuda")
    r, d = asi.token_logprobs(x, targets), asi.token_logprobs_grad(x, targets, a)
    for lp in (r.logprob, d.logprob):
        assert torch.isnan(lp[:2]).all() and torch.isfinite(lp[2]) and lp[3] == 0
    assert torch.isnan(d.grad[:2]).all() and torch.isfinite(d.grad[2]).all() and (d.grad[3] == 0).all()
    assert torch.isfinite(r.entropy).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_token_logprobs_through_autograd_and_against_differences(dtype):
    rows, vocab, eps = 6, 777, 2.0 ** -6
    x = _logits(rows, vocab, DTYPES[dtype], 5)
    targets = torch.randint(0, vocab, (2, 3), generator=_gen(1), device="cuda")
    targets[1, 1] = -100
    x = x.view(2, 3, vocab).requires_grad_(True)
    a, b = torch.randn(2, 3, generator=_gen(2), device="cuda"), torch.randn(2, 3, generator=_gen(3), device="cuda")
    r = asi.token_logprobs(x, targets, top=4, scale=0.9)
    assert not r.top_logprob.requires_grad and not r.top_index.requires_grad
    ((r.logprob * a).sum() + (r.entropy * b).sum()).backward()
    direct = asi.token_logprobs_grad(x.detach(), targets, a, b, scale=0.9)
    assert torch.equal(x.grad, direct.grad)
    x2 = x.detach().clone().requires_grad_(True)
    (asi.token_logprobs(x2, targets, scale=0.9).logprob * a).sum().backward()
    assert torch.equal(x2.grad, asi.token_logprobs_grad(x.detach(), targets, a, None, scale=0.9).grad)
    # central differences of the kernel's own values along directions of entries +-1: the third derivatives of log s and of its
    # entropy in such a direction are below 2 and 2 (log vocab + 3) of the weights, the values off by their bounds
    base = x.detach().float()
    for k in range(3):
        v = torch.randint(0, 2, base.shape, generator=_gen(30 + k), device="cuda").float() * 2 - 1
        f = []
        for s in (eps, -eps):
            q = asi.token_logprobs(base + s * v, targets, scale=0.9)
            f.append(float((q.logprob.double() * a).sum() + (q.entropy.double() * b).sum()))
        slope = (f[0] - f[1]) / (2 * eps)
        along = float((x.grad.double() * v).sum())
        weight = float(a.abs().sum() * 2 + b.abs().sum() * 2 * (math.log(vocab) + 3))
        values = U * (8 * 20 + 512) * float(a.abs().sum() + 8 * b.abs().sum())
        sizes = float((x.grad.double().abs()).sum()) * 2 * _round(x.dtype)
        # base + eps v is rounded too: U of |x| up to 16 for each entry, seen through the gradient
        moved = 16 * U / eps * float(x.grad.double().abs().sum())
        assert abs(slope - along) <= eps ** 2 / 6 * weight + values / eps + sizes + moved


def test_second_derivatives_are_refused():
    x = _logits(2, 50, torch.float32, 1).requires_grad_(True)
    grad, = torch.autograd.grad(asi.token_logprobs(x).entropy.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()


def test_no_rows_and_no_targets():
    x = torch.empty(0, 100, device="cuda")
    r = asi.token_logprobs(x, torch.empty(0, dtype=torch.int64, device="cuda"), top=3)
    assert r.logprob.shape == (0,) and r.top_index.shape == (0, 3)
    assert asi.token_logprobs_grad(x, None, None).grad.shape == (0, 100)
    x = _logits(3, 50, torch.float32, 1)
    r = asi.token_logprobs(x)
    assert r.logprob is None and r.top_index is None
    b = torch.ones(3, device="cuda")
    d = asi.token_logprobs_grad(x, None, None, b)
    assert d.logprob is None
    p = torch.softmax(x.double(), -1)
    want = -p * (p.log() + torch.special.entr(p).sum(-1, keepdim=True))
    _close(d.grad, want, 2000 * U * p + 1e-38, "entropy's gradient")


# ---- embedding --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("table_dtype", list(DTYPES))
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,vocab,dim", [(0, 5, 8), (1, 1, 1), (7, 11, 3), (5, 9, 8), (65, 100, 64), (33, 50, 100), (3, 40, 2048), (9, 30, 2052),
                                         (5, 20, 4100), (4, 7, 1001)])
def test_embedding(n, vocab, dim, dtype, table_dtype):
    g = _gen(dim)
    for pad, shift in ((0, 0), (8, 8), (1, 1)):
        flat = torch.empty(vocab * (dim + pad) + shift, device="cuda").normal_(generator=g).to(DTYPES[table_dtype])
        table = flat[shift:].as_strided((vocab, dim), (dim + pad, 1))
        tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        out = asi.embedding(tokens, table, scale=1.7, dtype=DTYPES[dtype])
        assert torch.equal(out, (table[tokens].float() * 1.7).to(DTYPES[dtype]))           # one product, one rounding
    if n > 3:
        tokens[0], tokens[2] = -1, vocab
        out = asi.embedding(tokens.view(1, -1), table, dtype=DTYPES[dtype])[0]
        assert torch.isnan(out[0]).all() and torch.isnan(out[2]).all() and torch.isfinite(out[1]).all()


def _tokens(n, vocab, kind, seed):
    g = _gen(seed)
    if kind == "uniform":
        return torch.randint(0, vocab, (n,), generator=g, device="cuda")
    if kind == "one":
        return torch.full((n,), vocab // 2, device="cuda")
    if kind == "two":                                    # long stretches of two tokens, the table's first and last
        return torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, 0, vocab - 1)
    rank = torch.exp(torch.rand(n, generator=g, device="cuda") * math.log(vocab + 1)).sub_(1).long().clamp_(0, vocab - 1)
    return torch.randperm(vocab, generator=g, device="cuda")[rank]


def _embedding_grad(tokens, grad_out, vocab, scale, padding=None):
    """Sum and sum of magnitudes in 64 bits, entries of each token."""
    keep = (tokens >= 0) & (tokens < vocab)
    if padding is not None:
        keep &= tokens != padding
    t, g = tokens[keep], grad_out[keep].double() * scale
    total = torch.zeros(vocab, grad_out.shape[1], dtype=torch.float64, device="cuda").index_put_((t,), g, accumulate=True)
    size = torch.zeros_like(total).index_put_((t,), g.abs(), accumulate=True)
    return total, size, torch.bincount(t, minlength=vocab)


GRADS = [(1024, 40, 24, "falling"), (1025, 40, 24, "falling"), (1024, 3, 301, "one"), (512, 40, 24, "falling"), (513, 40, 24, "falling"), (512, 3, 1000, "one"), (300, 300, 41, "two"), (1, 1, 1, "uniform"), (2, 5, 8, "one"), (31, 7, 16, "uniform"), (33, 40, 5, "falling"), (64, 64, 64, "uniform"), (257, 3, 24, "uniform"),
         (500, 1000, 72, "falling"), (1000, 50, 2056, "falling"), (4096, 777, 130, "one"), (5000, 5000, 64, "two"), (9001, 33, 33, "falling"),
         (40000, 900, 64, "one"), (70001, 70000, 8, "falling"), (140000, 12, 9, "two")]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("grad_dtype", list(DTYPES))
@pytest.mark.parametrize("n,vocab,dim,kind", GRADS)
def test_embedding_grad(n, vocab, dim, kind, grad_dtype, dtype):
    tokens = _tokens(n, vocab, kind, n + dim)
    if n > 30:
        tokens[n // 3], tokens[n // 2] = -7, vocab + 3           # count for nothing
    padding = int(tokens[0]) if n > 100 and kind != "one" else None
    flat = torch.empty(n * (dim + 3) + 1, device="cuda").normal_(generator=_gen(n)).to(DTYPES[dtype])
    total, size, count = None, None, None
    for grad_out in (flat[:n * dim].view(n, dim), flat[1:].as_strided((n, dim), (dim + 3, 1))):
        total, size, count = _embedding_grad(tokens, grad_out, vocab, 0.37, padding)
        # each term goes through as many sums as its token has entries at most, the product and the rounding
        bound = (count[:, None] + 4) * U * size + _round(DTYPES[grad_dtype]) * total.abs() * 1.01
        out = asi.embedding_grad(tokens, grad_out, vocab, scale=0.37, padding_idx=padding, dtype=DTYPES[grad_dtype])
        _close(out, total, bound, "dtable")
        assert torch.equal(out, asi.embedding_grad(tokens, grad_out, vocab, scale=0.37, padding_idx=padding, dtype=DTYPES[grad_dtype]))
        # added to what is there, in a table whose rows are apart
        held = torch.empty(vocab, dim + 5, device="cuda").normal_(generator=_gen(1)).to(DTYPES[grad_dtype])
        before = held.clone()
        asi.embedding_grad(tokens, grad_out, vocab, scale=0.37, padding_idx=padding, out=held[:, 2:2 + dim], accumulate=True)
        want = before[:, 2:2 + dim].double() + total
        _close(held[:, 2:2 + dim], want, (count[:, None] + 4) * U * size + _round(DTYPES[grad_dtype]) * 1.01 * (want.abs() + (count[:, None] + 4) * U * size),
               "added")
        assert torch.equal(held[count == 0], before[count == 0])
        assert torch.equal(held[:, :2], before[:, :2]) and torch.equal(held[:, 2 + dim:], before[:, 2 + dim:])


def test_embedding_grad_without_tokens():
    out = torch.full((5, 6), NAN, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert (asi.embedding_grad(none, torch.empty(0, 6, device="cuda"), 5, out=out) == 0).all()
    out.fill_(3)
    assert (asi.embedding_grad(none, torch.empty(0, 6, device="cuda"), 5, out=out, accumulate=True) == 3).all()
    gone = torch.full((9,), 100, device="cuda")                     # every token out of range
    assert (asi.embedding_grad(gone, torch.randn(9, 6, device="cuda"), 5, out=out) == 0).all()


def test_embedding_through_autograd_and_against_differences():
    g = _gen(4)
    table = torch.empty(50, 24, device="cuda").normal_(generator=g).requires_grad_(True)
    tokens = torch.randint(0, 50, (3, 40), generator=g, device="cuda")
    w = torch.empty(3, 40, 24, device="cuda").normal_(generator=g)
    out = asi.embedding(tokens, table, scale=2.0, padding_idx=7)
    (out * w).sum().backward()
    total, size, count = _embedding_grad(tokens.flatten(), w.view(-1, 24), 50, 2.0, 7)
    _close(table.grad, total, (count[:, None] + 4) * U * size + U * total.abs(), "grad")
    # the lookup is linear: a difference has no error but the roundings of 50 x 24 products and the difference's own cancellation
    v = torch.empty(50, 24, device="cuda").normal_(generator=g)
    v[7] = 0
    t = table.detach()
    f = [float((asi.embedding(tokens, t + s * v, scale=2.0).double() * w).sum()) for s in (0.5, -0.5)]
    assert abs((f[0] - f[1]) - float((table.grad.double() * v).sum())) <= 8 * U * float((w.double().abs().sum()) * 2 * (t.abs().max() + v.abs().max())) 
    half = t.to(torch.bfloat16).requires_grad_(True)
    (asi.embedding(tokens, half, scale=2.0) * w.to(torch.bfloat16)).sum().backward()
    assert half.grad.dtype == torch.bfloat16


# ---- norms of queries and keys with the position rotation ----------------------------------------------------
def _turned(n, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    a, b = (n[..., 0:rot:2], n[..., 1:rot:2]) if interleaved else (n[..., :rot // 2], n[..., rot // 2:rot])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)
    return torch.cat((y, n[..., rot:]), -1)


def _rotate(x, gain, cos, sin, positions, eps, interleaved):
    x = x.double()
    bad = (positions < 0) | (positions >= cos.shape[0])
    at = torch.where(bad, 0, positions)
    c, s = cos.double()[at], sin.double()[at]
    if c.shape[-1]:
        c = torch.where(bad[..., None], NAN, c)
    u = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return _turned(u * (1.0 if gain is None else gain.double()), c[:, :, None], s[:, :, None], interleaved)


# batch, tokens, q_heads, k_heads, head_dim, rot_dim
HEADS = [(1, 1, 1, 1, 2, 2), (2, 3, 3, 1, 7, 6), (1, 5, 2, 2, 16, 16), (3, 17, 4, 2, 32, 32), (8, 1, 32, 4, 64, 64), (2, 33, 5, 1, 64, 32), (1, 40, 3, 3, 80, 80),
         (2, 9, 6, 2, 96, 48), (2, 65, 4, 2, 128, 128), (1, 12, 2, 1, 160, 64), (2, 7, 3, 1, 256, 256), (1, 6, 2, 1, 256, 0), (1, 4, 2, 1, 1000, 500), (1, 3, 1, 1, 1024, 1024),
         (3, 11, 2, 0, 64, 64), (2, 8, 0, 3, 128, 64), (2, 5, 3, 2, 65, 10), (1, 700, 9, 3, 48, 48)]


def _qk_inputs(shape, dtype, seed, packed, gains=True):
    b, t, hq, hk, d, rot = shape
    g = _gen(seed)
    randn = lambda *s: torch.empty(*s, device="cuda").normal_(generator=g)  # noqa: E731
    if packed:
        qkv = (randn(b, t, (hq + 2 * hk) * d + 1) * 2).to(dtype)[..., 1:]       # one element into a row: no vector access
        q, k = qkv[..., :hq * d].unflatten(-1, (hq, d)), qkv[..., hq * d:(hq + hk) * d].unflatten(-1, (hk, d))
    else:
        q, k = (randn(b, t, hq, d) * 2).to(dtype), (randn(b, t, hk, d) * 0.5).to(dtype)
    gq, gk = ((1 + 0.3 * randn(d)).to(dtype if seed % 2 else torch.float32) for _ in range(2)) if gains else (None, None)
    cos, sin = asi.rotary_table(3000, rot)
    positions = torch.randint(0, 3000 - t, (b, 1), generator=g, device="cuda") + torch.arange(t, device="cuda")
    return q, k, gq, gk, cos, sin, positions


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", HEADS)
def test_qk_norm_rotate(shape, interleaved, dtype):
    rot = shape[5]
    for seed, (packed, heads_first, gains) in enumerate([(False, False, True), (False, True, True), (True, True, True), (False, False, False)]):
        q, k, gq, gk, cos, sin, positions = _qk_inputs(shape, DTYPES[dtype], seed, packed, gains)
        got = asi.qk_norm_rotate(q, k, gq, gk, cos, sin, positions, eps=1e-5, interleaved=interleaved, heads_first=heads_first)
        for y, x, gain in zip(got, (q, k), (gq, gk)):
            want = _rotate(x, gain, cos, sin, positions, 1e-5, interleaved)
            # the norm: 16 squares a lane and 6 sums across lanes (1024 entries: 16 a lane) at the most, the quotient, the
            # gain, two products and a sum of the two partners, each below the largest of |x / rms * gain|
            size = (x.double() / (x.double().square().mean(-1, keepdim=True) + 1e-5).sqrt() * (1.0 if gain is None else gain.double())).abs()
            size = size.amax(-1, keepdim=True)
            y = y.transpose(1, 2) if heads_first else y
            _close(y, want, 64 * U * size + _round(x.dtype) * want.abs() * 1.01, "y")
    assert rot == 2 * cos.shape[1]


def test_positions():
    q, k, gq, gk, cos, sin, positions = _qk_inputs((2, 5, 3, 1, 64, 32), torch.float32, 2, False)
    positions[1, 2], positions[0, 4] = 3000, -1
    got, _ = asi.qk_norm_rotate(q, k, gq, gk, cos, sin, positions)
    _close(got, _rotate(q, gq, cos, sin, positions, 1e-6, False), 64 * U * 8, "out of range")
    assert torch.isfinite(got[1, 2, :, 32:]).all()                    # what is not turned has a value all the same
    default = asi.qk_norm_rotate(q, k, gq, gk, cos, sin)[0]
    shared = asi.qk_norm_rotate(q, k, gq, gk, cos, sin, torch.arange(5, device="cuda"))[0]
    each = asi.qk_norm_rotate(q, k, gq, gk, cos, sin, torch.arange(5, device="cuda").expand(2, 5))[0]
    assert torch.equal(default, shared) and torch.equal(default, each)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", HEADS)
def test_qk_norm_rotate_grad(shape, interleaved, dtype):
    b, t, hq, hk, d, rot = shape
    for seed, (packed, heads_first, gains) in enumerate([(False, False, True), (False, True, True), (True, True, True), (False, False, False)]):
        q, k, gq, gk, cos, sin, positions = _qk_inputs(shape, DTYPES[dtype], seed, packed, gains)
        shape_of = (lambda h: (b, h, t, d)) if heads_first else (lambda h: (b, t, h, d))
        gy = [torch.empty(*shape_of(h), device="cuda").normal_(generator=_gen(50 + h)).to(q.dtype) for h in (hq, hk)]
        got = asi.qk_norm_rotate_grad(q, k, gq, gk, cos, sin, *gy, positions, eps=1e-5, interleaved=interleaved, heads_first=heads_first)
        again = asi.qk_norm_rotate_grad(q, k, gq, gk, cos, sin, *gy, positions, eps=1e-5, interleaved=interleaved, heads_first=heads_first)
        assert all(torch.equal(x, y) for x, y in zip(got, again))
        for dx, dg, x, gain, dy in zip(got[:2], got[2:], (q, k), (gq, gk), gy):
            if x.numel() == 0:
                assert (dg == 0).all()
                continue
            dy = (dy.transpose(1, 2) if heads_first else dy).double()
            w = torch.ones(d, device="cuda", dtype=torch.float64) if gain is None else gain.double()
            r = 1 / (x.double().square().mean(-1, keepdim=True) + 1e-5).sqrt()
            u = x.double() * r
            dn = _turned(dy, cos.double()[positions][:, :, None], -sin.double()[positions][:, :, None], interleaved)
            want = r * (w * dn - u * (w * dn * u).mean(-1, keepdim=True))
            # as forward: a sum of up to 16 + 6 terms, products and differences of magnitudes no larger than these
            most = (w * dn).abs().amax(-1, keepdim=True) + dy.abs().amax(-1, keepdim=True) * w.abs().max()
            size = r * (most + u.abs() * (w * dn * u).abs().mean(-1, keepdim=True))
            _close(dx, want, 64 * U * size + _round(x.dtype) * want.abs() * 1.01, "dx")
            terms = dn * u
            rows = terms.shape[0] * terms.shape[1] * terms.shape[2]
            # the rows a lane adds up, 16 to a workgroup at least, and the sums of the lanes, waves and workgroups
            _close(dg, terms.sum((0, 1, 2)), (rows / 16 + 128) * U * (dy.abs().amax(-1, keepdim=True) * 2 * u.abs()).sum((0, 1, 2)), "dgain")


def test_qk_norm_rotate_through_autograd_and_against_differences():
    shape = (2, 9, 4, 2, 64, 32)
    q, k, gq, gk, cos, sin, positions = _qk_inputs(shape, torch.float32, 3, False)
    leaves = [x.clone().requires_grad_(True) for x in (q, k, gq, gk)]
    out = asi.qk_norm_rotate(*leaves, cos, sin, positions, heads_first=True)
    w = [torch.empty_like(o).normal_(generator=_gen(8)) for o in out]
    sum((o * v).sum() for o, v in zip(out, w)).backward()
    # central differences in 64 bits of the definition: the gradient's own error (64 U of sizes below 30) and eps^2 times third
    # derivatives, which the norm bounds by |v|^3 / rms^3 of each head
    for k_leaf, leaf in enumerate(leaves):
        v = torch.empty_like(leaf).normal_(generator=_gen(60 + k_leaf)).double()
        eps = 1e-4
        f = []
        for s in (eps, -eps):
            args = [x.detach().double() + (s * v if i == k_leaf else 0) for i, x in enumerate(leaves)]
            y = [_rotate(args[i], args[2 + i], cos, sin, positions, 1e-6, False).transpose(1, 2) for i in range(2)]
            f.append(sum(float((a * b.double()).sum()) for a, b in zip(y, w)))
        slope, along = (f[0] - f[1]) / (2 * eps), float((leaf.grad.double() * v).sum())
        assert abs(slope - along) <= 64 * U * 30 * float(v.abs().sum()) + eps ** 2 * 100 * v.numel(), k_leaf


def test_qk_norm_rotate_in_place_and_packed_gradients():
    """Results over the inputs, gradients into one buffer of a packed projection, through the C entry points."""
    import ctypes as C
    from paper_2505_05086_amd import binding as B, lm
    q, k, gq, gk, cos, sin, positions = _qk_inputs((2, 33, 6, 2, 64, 64), torch.bfloat16, 1, False)
    want = asi.qk_norm_rotate(q, k, gq, gk, cos, sin, positions)
    for lie in (0, 1):                                       # whole vectors, and one element off
        buf = torch.empty(2, 33, 10 * 64 + lie, dtype=torch.bfloat16, device="cuda")[..., lie:]
        a, b = buf[..., :6 * 64].unflatten(-1, (6, 64)), buf[..., 6 * 64:8 * 64].unflatten(-1, (2, 64))
        a.copy_(q), b.copy_(k)
        buf[..., 8 * 64:] = 5
        desc = lm._qk_desc(*map(lm._geometry, (a, b, gq, gk, cos, sin, positions)), 1e-6, False)
        desc.q_out_stride[:], desc.k_out_stride[:] = a.stride()[:3], b.stride()[:3]
        st = torch.cuda.current_stream().cuda_stream
        p = lambda t: t.data_ptr()  # noqa: E731
        assert B.lib().asi_qk_norm_rotate(desc, p(a), p(b), p(gq), p(gk), p(positions), p(cos), p(sin), p(a), p(b), st) == 0
        # the two forms of the kernel add squares in different orders: an ulp of bf16
        for y, z in ((a, want[0]), (b, want[1])):
            _close(y, z, z.double().abs() * 2.0 ** -7, "in place")
        assert (buf[..., 8 * 64:] == 5).all()
        dy = [torch.empty_like(x).normal_(generator=_gen(2)) for x in (q, k)]
        ref = asi.qk_norm_rotate_grad(q, k, gq, gk, cos, sin, *dy, positions)
        a.copy_(q), b.copy_(k)
        desc.q_out_stride[:], desc.k_out_stride[:] = dy[0].stride()[:3], dy[1].stride()[:3]
        desc.dq_stride[:], desc.dk_stride[:] = a.stride()[:3], b.stride()[:3]
        dg = torch.empty(2, 64, device="cuda")
        ws = torch.empty(B.lib().asi_qk_norm_rotate_grad_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        assert B.lib().asi_qk_norm_rotate_grad(desc, p(a), p(b), p(gq), p(gk), p(positions), p(cos), p(sin), p(dy[0]), p(dy[1]), p(a), p(b),
                                               p(dg[0]), p(dg[1]), p(ws), ws.numel(), st) == 0
        for y, z in ((a, ref[0]), (b, ref[1])):
            _close(y, z, 2.0 ** -7 * z.double().abs() + 64 * U * 30, "gradient in place")
        assert (buf[..., 8 * 64:] == 5).all()


# ---- AdamW ------------------------------------------------------------------------------------------------
def _to_8bit(x, positive):
    """The format's definition on one tensor in fp32: codes (as their values) and scales."""
    n = x.numel()
    blocks = torch.cat((x, x.new_zeros(-n % 256))).view(-1, 256)
    scale = torch.where(torch.isfinite(blocks), blocks.abs(), 0.0).amax(-1) * (1.0 / 448.0)
    held = scale >= 2.0 ** -126
    inv = torch.where(held, 1.0 / scale.double(), 0.0).float()        # the quotient of fp32 numbers in 64 bits, rounded: correctly rounded
    value = (blocks * inv[:, None]).to(torch.float8_e4m3fn).float()
    if positive:
        value = torch.where(held[:, None] & (blocks > 0) & (value == 0), 2.0 ** -9, value)
    return value.flatten()[:n], torch.where(held, scale, 0.0)


def _expected_step(p, g, state, bits, hyper, step, gs):
    """One step on flat fp32 tensors, each operation rounded by itself as elementary torch operations are."""
    lr, (b1, b2), eps, wd = hyper
    g = g.float() * gs
    if bits == 32:
        m, v = state["exp_avg"].flatten(), state["exp_avg_sq"].flatten()
    else:
        wide = lambda c, s: c.flatten().float() * s.repeat_interleave(256)[:c.numel()]  # noqa: E731
        m, root = wide(state["exp_avg"], state["exp_avg_scale"]), wide(state["exp_avg_sqrt"], state["exp_avg_sqrt_scale"])
        v = root * root
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    root = v.sqrt()
    u = m / (root * (1.0 / math.sqrt(1 - b2 ** step)) + eps)
    p = p * (1 - lr * wd) - u * (lr / (1 - b1 ** step))
    return p, m, v, root


SHAPES = [(1,), (3,), (64, 4), (255,), (256,), (257,), (0,), (1000, 3), (4096,), (4097,), (33, 511), (12289,)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", ["f32", "bf16", "bf16+master", "bf16, fp32 gradients", "f32, bf16 gradients"])
def test_adamw_steps(kind, bits):
    g = _gen(7)
    pt = torch.bfloat16 if kind.startswith("bf16") else torch.float32
    gt = torch.float32 if kind in ("f32", "bf16, fp32 gradients") else torch.bfloat16
    master = "master" in kind
    hyper = (3e-3, (0.9, 0.99), 1e-8, 0.05)
    params = [torch.nn.Parameter(torch.empty(s, device="cuda").normal_(generator=g).to(pt)) for s in SHAPES * 4]     # more than one launch
    flat = torch.empty(3001, device="cuda").normal_(generator=g).to(pt)
    params += [torch.nn.Parameter(flat[1:2000]), torch.nn.Parameter(flat[2001:3001])]                                # no vector access
    opt = asi.AdamW(params, lr=hyper[0], betas=hyper[1], eps=hyper[2], weight_decay=hyper[3], state_bits=bits, master=master)
    gs = torch.tensor([0.7], device="cuda")
    for step in range(1, 5):
        grads = [(torch.empty(p.shape, device="cuda").normal_(generator=g) * torch.empty(p.shape, device="cuda").normal_(generator=g).exp()).to(gt) for p in params]
        before = [(p.detach().clone(), {k: v.clone() for k, v in opt.state[p].items()}) for p in params]
        if gt == pt:
            for p, d in zip(params, grads):
                p.grad = d
            opt.step(grad_scale=gs)
        else:
            opt.step(grad_scale=gs, grads=grads)
        for p, d, (old, state) in zip(params, grads, before):
            if not state:
                zero = {32: ("exp_avg", "exp_avg_sq"), 8: ("exp_avg", "exp_avg_sqrt")}[bits]
                state = {k: torch.zeros(p.numel(), device="cuda") for k in zero}
                if bits == 8:
                    state.update({k + "_scale": torch.zeros(-(-p.numel() // 256), device="cuda") for k in zero})
                if master:
                    state["master"] = old.float()
            start = (state["master"] if master else old.float()).flatten()
            q, m, v, root = _expected_step(start, d.flatten(), state, bits, hyper, step, gs)
            now = opt.state[p]
            if master:
                assert torch.equal(now["master"].flatten(), q)
            assert torch.equal(p.detach().flatten(), q.to(pt))
            if bits == 32:
                assert torch.equal(now["exp_avg"].flatten(), m) and torch.equal(now["exp_avg_sq"].flatten(), v)
            elif p.numel():
                for name, x, positive in (("exp_avg", m, False), ("exp_avg_sqrt", root, True)):
                    value, scale = _to_8bit(x, positive)
                    assert torch.equal(now[name + "_scale"], scale), name
                    assert torch.equal(now[name].flatten().float(), value), name
    assert opt.param_groups[0]["step"] == 4


def test_adamw_against_64_bits():
    """20 steps in fp32 against the formula in fp64: each step adds at most 16 roundings of the update and one of the parameter."""
    g = _gen(3)
    p = torch.nn.Parameter(torch.empty(5000, device="cuda").normal_(generator=g))
    q, m, v = p.detach().double(), torch.zeros(5000, dtype=torch.float64, device="cuda"), torch.zeros(5000, dtype=torch.float64, device="cuda")
    opt = asi.AdamW([p], lr=1e-2, weight_decay=0.1)
    for step in range(1, 21):
        p.grad = torch.empty(5000, device="cuda").normal_(generator=g)
        opt.step()
        d = p.grad.double()
        m, v = 0.9 * m + 0.1 * d, 0.999 * v + 0.001 * d * d
        q = q * (1 - 1e-3) - 1e-2 * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.999 ** step)).sqrt() + 1e-8)
    # an update is at most about 1 / sqrt(1 - beta2 ...) <= 4 of the rate here, its relative error grows with the states' 20 roundings
    _close(p.detach(), q, 20 * (U * 6 + 1e-2 * 4 * 80 * U), "parameter")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_states_that_are_not_finite_or_tiny(bits):
    p = torch.nn.Parameter(torch.zeros(1024, device="cuda"))
    d = torch.zeros(1024, device="cuda")
    d[5], d[300], d[301] = NAN, INF, 1.0
    d[512:768] = 1e-30                               # squares that vanish
    p.grad = d
    opt = asi.AdamW([p], state_bits=bits, weight_decay=0.0)
    opt.step()
    assert torch.isnan(p.detach()[5]) and torch.isnan(p.detach()[300])
    fine = torch.ones(1024, dtype=torch.bool, device="cuda")
    fine[5] = fine[300] = False
    assert torch.isfinite(p.detach()[fine]).all()
    if bits == 8:
        s = opt.state[p]
        assert torch.isfinite(s["exp_avg_scale"]).all() and torch.isfinite(s["exp_avg_sqrt_scale"]).all()
        assert torch.isnan(s["exp_avg"].float()[5]) and torch.isnan(s["exp_avg"].float()[300])
        assert torch.isfinite(s["exp_avg"].float()[fine]).all()
        assert abs(float(s["exp_avg"].float()[301] * s["exp_avg_scale"][1]) - 0.1) < 0.1 / 16
        # one large gradient in a block: the others' roots are small beside it but not zero
        p2 = torch.nn.Parameter(torch.zeros(256, device="cuda"))
        p2.grad = torch.full((256,), 1e-6, device="cuda")
        p2.grad[0] = 1.0
        o2 = asi.AdamW([p2], state_bits=8)
        o2.step()
        assert (o2.state[p2]["exp_avg_sqrt"].float() > 0).all()


def test_adamw_skip_groups_and_missing_gradients():
    a, b, c = (torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (10, 300, 5))
    opt = asi.AdamW([{"params": [a, b], "lr": 0.1}, {"params": [c], "lr": 0.01, "weight_decay": 0.0}], weight_decay=0.5)
    a.grad, c.grad = torch.ones_like(a), torch.ones_like(c)
    skip = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt.step(skip=skip + 1)
    assert (a == 1).all() and (c == 1).all() and (opt.state[a]["exp_avg"] == 0).all()
    opt.step(skip=skip)
    assert (b == 1).all() and b not in opt.state
    # second step (the first was skipped but counted), gradients 1: m / (1 - b1^2) over sqrt(v / (1 - b2^2))
    u = (0.1 / (1 - 0.81)) / math.sqrt(0.001 / (1 - 0.999 ** 2))
    _close(a.detach(), torch.full((10,), 0.95 - 0.1 * u, device="cuda"), 32 * U, "a")
    _close(c.detach(), torch.full((5,), 1.0 - 0.01 * u, device="cuda"), 32 * U, "c")
    b.grad = torch.ones_like(b)
    opt.step()
    assert (b != 1).all()


def test_adamw_follows_replaced_data():
    """Parameters and gradients whose data is exchanged between steps, as conversions of a model do."""
    p = torch.nn.Parameter(torch.ones(1000, device="cuda"))
    p.grad = torch.ones_like(p)
    opt = asi.AdamW([p], lr=0.5, weight_decay=0.0)
    opt.step()
    kept = p.data
    old = kept.clone()
    p.data = torch.full((1000,), 3.0, device="cuda")
    p.grad = torch.ones_like(p)
    opt.step()
    assert torch.equal(kept, old) and (p.data < 3.0).all()
    p.grad = None
    p.data = p.data.to(torch.bfloat16)
    p.grad = torch.ones_like(p)
    before = p.data.clone()
    opt.step()
    assert (p.data < before).all()
    p.data = torch.ones(10, 4, 5, 5, device="cuda").to(memory_format=torch.channels_last)
    p.grad = torch.ones_like(p)
    with pytest.raises(TypeError):
        opt.step()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_saved_and_loaded_goes_on_the_same(bits):
    def fresh():
        g = _gen(1)
        ps = [torch.nn.Parameter(torch.empty(s, device="cuda").normal_(generator=g).to(torch.bfloat16)) for s in ((300, 7), (5,))]
        return ps, asi.AdamW(ps, lr=1e-2, state_bits=bits, master=True)

    def go(ps, opt, seed):
        for k, p in enumerate(ps):
            p.grad = torch.empty(p.shape, device="cuda").normal_(generator=_gen(seed + k)).to(torch.bfloat16)
        opt.step()

    ps, opt = fresh()
    go(ps, opt, 10)
    saved, values = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in ps]
    go(ps, opt, 20)
    qs, other = fresh()
    go(qs, other, 77)                                 # its plan is made before the states are loaded
    other.load_state_dict(saved)
    for q, v in zip(qs, values):
        q.data.copy_(v)
    go(qs, other, 20)
    assert all(torch.equal(p, q) for p, q in zip(ps, qs))
    for p, q in zip(ps, qs):
        for key, t in opt.state[p].items():
            assert t.dtype == other.state[q][key].dtype and torch.equal(t.view(torch.uint8), other.state[q][key].view(torch.uint8))


# ---- offsets past 32 bits ------------------------------------------------------------------------------------
def test_logits_past_32_bits():
    rows, vocab = 66000, 66000                                    # 4.4e9 entries
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x[-3:] = _logits(3, vocab, torch.bfloat16, 1)
    targets = torch.arange(rows, device="cuda")
    a = torch.full((rows,), -1.0, device="cuda")
    r = asi.token_logprobs(x, targets, top=4)
    logprob, entropy, p, _ = _definition(x[-3:], targets[-3:], 1.0, -100)
    bound = _value_bound(x[-3:], 1.0)
    _close(r.logprob[-3:], logprob, bound, "logprob")
    assert torch.equal(r.top_index[-3:], _order(x[-3:], 4))
    assert abs(float(r.logprob[0]) + math.log(vocab)) < 300 * U and r.top_index[0].tolist() == [0, 1, 2, 3]
    last = x[-3:].clone()
    d = asi.token_logprobs_grad(x, targets, a, out=x)
    assert torch.equal(d.grad[-3:], asi.token_logprobs_grad(last, targets[-3:], a[-3:]).grad)


def test_tables_past_32_bits():
    vocab, dim = (1 << 21) + 5, 2052                              # 4.3e9 entries
    table = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda")
    table[-7:] = torch.empty(7, dim, device="cuda").normal_(generator=_gen(1)).to(torch.bfloat16)
    table[:2] = 1.0
    tokens = torch.cat((torch.arange(vocab - 7, vocab, device="cuda").repeat(200), torch.zeros(3, dtype=torch.int64, device="cuda")))
    assert torch.equal(asi.embedding(tokens, table, scale=2.0), (table[tokens].float() * 2.0).to(torch.bfloat16))
    grad_out = torch.ones(len(tokens), dim, dtype=torch.bfloat16, device="cuda")
    for n in (len(tokens), 100):                                  # sorted, and few
        out = asi.embedding_grad(tokens[-n:], grad_out[-n:], vocab, out=table)
        count = torch.bincount(tokens[-n:] % 1000003, minlength=0)          # ids as they are below a million, the last ones folded
        assert (out[-7:].float() == count[torch.arange(vocab - 7, vocab, device="cuda") % 1000003][:, None]).all()
        assert (out[0] == 3).all() and not out[1:-7].any()


def test_heads_past_32_bits():
    apart = (1 << 32) + 256
    buf = torch.empty(apart + 9 * 3 * 64, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((2, 9, 3, 64), (apart, 192, 64, 1))
    q.copy_(torch.empty(2, 9, 3, 64, device="cuda").normal_(generator=_gen(1)))
    near = q.contiguous()
    cos, sin = asi.rotary_table(20, 64)
    for a, b in zip(asi.qk_norm_rotate(q, q, None, None, cos, sin), asi.qk_norm_rotate(near, near, None, None, cos, sin)):
        assert torch.equal(a, b)
    g = torch.empty_like(near).normal_(generator=_gen(2))
    for a, b in zip(asi.qk_norm_rotate_grad(q, q, None, None, cos, sin, g, g), asi.qk_norm_rotate_grad(near, near, None, None, cos, sin, g, g)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_past_32_bits(bits):
    n, m = (1 << 32) + 1000, 1256
    p = torch.nn.Parameter(torch.zeros(n, dtype=torch.bfloat16, device="cuda"))
    p.grad = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    q = torch.nn.Parameter(torch.empty(m, device="cuda").normal_(generator=_gen(1)).to(torch.bfloat16))
    q.grad = torch.empty(m, device="cuda").normal_(generator=_gen(2)).to(torch.bfloat16)
    with torch.no_grad():
        p[-m:] = q
        p.grad[-m:] = q.grad                                      # blocks of 256 begin at the same place
    for x in (p, q):
        asi.AdamW([x], state_bits=bits).step()
    assert torch.equal(p[-m:], q) and not p[:-m].any()


# ---- streams, graphs ----------------------------------------------------------------------------------------
def _one_of_each(x, targets, table, tokens, q, k, gain, cos, sin, out):
    r = asi.token_logprobs(x, targets, top=5)
    d = asi.token_logprobs_grad(x, targets, r.logprob.neg(), r.entropy)
    e = asi.embedding(tokens, table, scale=3.0)
    w = asi.embedding_grad(tokens, e, table.shape[0])
    y = asi.qk_norm_rotate(q, k, gain, gain, cos, sin, heads_first=True)
    z = asi.qk_norm_rotate_grad(q, k, gain, gain, cos, sin, *y, heads_first=True)
    for o, v in zip(out, (r.logprob, r.entropy, r.top_logprob, r.top_index, d.grad, e, w, *y, *z)):
        o.copy_(v)


def _inputs_of_each(seed):
    g = _gen(seed)
    x = _logits(9, 5003, torch.bfloat16, seed)
    targets = torch.randint(0, 5003, (9,), generator=g, device="cuda")
    table = torch.empty(700, 96, device="cuda").normal_(generator=g)
    tokens = _tokens(3000, 700, "falling", seed)
    q, k, gain, _, cos, sin, _ = _qk_inputs((2, 50, 4, 2, 64, 64), torch.float32, seed, False)
    return [x, targets, table, tokens, q, k, gain, cos, sin]


def test_other_streams_and_graph_replays_match_eager():
    inputs = [_inputs_of_each(s) for s in (1, 3, 5)]
    shapes = [(9,), (9,), (9, 5), (9, 5), (9, 5003), (3000, 96), (700, 96), (2, 4, 50, 64), (2, 2, 50, 64), (2, 50, 4, 64), (2, 50, 2, 64), (64,), (64,)]
    dtypes = [torch.float32] * 3 + [torch.int64, torch.bfloat16] + [torch.float32] * 8
    new = lambda: [torch.empty(s, dtype=d, device="cuda") for s, d in zip(shapes, dtypes)]  # noqa: E731
    eager = []
    for args in inputs:
        eager.append(new())
        _one_of_each(*args, eager[-1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = new()
        _one_of_each(*inputs[1], out)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, eager[1]))
    static, out = [t.clone() for t in inputs[0]], new()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        _one_of_each(*static, out)
        torch.cuda.synchronize()
        graph.capture_begin()
        _one_of_each(*static, out)
        graph.capture_end()
    torch.cuda.synchronize()
    for rep in range(4):
        which = (rep + 1) % 3
        for a, b in zip(static, inputs[which]):
            a.copy_(b)
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        junk = (out[4].float() * 2).sum()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[which])) and junk == junk
