"""Token log probabilities from hidden states without the logits (asi_linear_logprobs) against their definition in 64 bits.

U = 2^-24 is half an fp32 ulp.  A logit is a sum of dim products, in fp32 inputs of six times as many (three bf16 parts a side; the
parts that are left out are below 2^-24 of a product): E = (6 dim + 16) U sum_k |h_k w_k| bounds its error whatever the order, and
what follows is a count of roundings on top; each bound is derived where it stands.
"""
import math

import pytest
import torch
from torch.autograd import forward_ad

import paper_2505_05086_amd as asi
from paper_2505_05086_amd import binding as B
from paper_2505_05086_amd.lm import _DTYPE, LinearLogprobs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORE = -100


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _round(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def _close(got, want, bound, what):
    """|got - want| <= bound entry by entry; where `want` is not finite the two are equal."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape, what
    bound = torch.as_tensor(bound, dtype=torch.float64, device=got.device).expand_as(want)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    assert torch.equal(got[odd].nan_to_num(7.0), want[odd].nan_to_num(7.0)), f"{what}: infinities"
    off = ((got - want).abs() - bound)[~odd]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{what}: {float(off.max()):.3g} over its bound"


def _inputs(rows, dim, vocab, dtype, seed, pad=0, shift=0, ignored=0.3, spread=2.5):
    g = _gen(seed)
    rand = lambda n, m, p, s, std: (torch.empty(n * (m + p) + s, device="cuda").normal_(0, std, generator=g).to(dtype)  # noqa: E731
                                    [s:].as_strided((n, m), (m + p, 1)))
    weight = rand(vocab, dim, pad, shift, spread * dim ** -0.5)
    hidden = rand(rows, dim, pad, shift, 1.0)
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    targets[torch.rand(rows, generator=g, device="cuda") < ignored] = IGNORE
    if rows:
        targets[0] = vocab - 1
    a, b = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    return hidden, weight, targets, a, b


class _Definition:
    """Values, gradients and the bounds of their errors."""

    def __init__(self, hidden, weight, targets, scale, a=None, b=None):
        h, w = hidden.double(), weight.double()
        r = _round(hidden.dtype)
        live = torch.ones(len(h), dtype=torch.bool, device=h.device) if targets is None else targets != IGNORE
        h = torch.where(live[:, None], h, 0.0)                            # a row that is left out is not read
        dim, vocab = w.shape[1], w.shape[0]
        z = h @ w.t().contiguous() * scale
        e = (6 * dim + 16) * U * (h.abs() @ w.abs().t().contiguous()).amax(-1) * scale      # of any logit of a row
        logp = torch.log_softmax(z, -1)
        p = logp.exp()
        entropy = torch.special.entr(p).sum(-1)
        # a logit, the difference to the largest, its product, the logarithm of a sum of up to 2^12 terms in a lane and 2^12 in parts,
        # of which no more than 128 in a row change its last bit
        values = 2 * e + U * (8 * z.abs().amax(-1) + 256)
        self.entropy = torch.where(live, entropy, 0.0)
        # -sum p log p: p off by 2 e of itself
        self.entropy_bound = torch.where(live, values * (2 + entropy), 0.0)
        self.logprob = None
        if targets is not None:
            fine = (targets >= 0) & (targets < vocab)
            at = torch.where(fine, targets, 0)[:, None]
            self.logprob = torch.where(fine, logp.gather(1, at)[:, 0], NAN)
            self.logprob[~live] = 0.0
            self.logprob_bound = torch.where(live, values, 0.0)
        if a is None and b is None:
            return
        hot = torch.zeros_like(z)
        if targets is not None:
            hot.scatter_(1, at, 1.0)
        a = torch.zeros(len(h), device=h.device) if a is None else a
        a, b = (torch.where(live, x.double(), 0.0)[:, None] for x in (a, torch.zeros_like(a) if b is None else b))
        dz = scale * (a * (hot - p) - b * p * (logp + entropy[:, None]))
        # p is off by 2 (e + the rounding of the logarithm) of itself and so is what is multiplied by it; dz is rounded to bf16 for bf16
        # inputs, and otherwise held to 2^-24 in three parts
        size = scale * (a.abs() * (hot + p) + b.abs() * p * (logp.abs() + entropy[:, None] + 1))
        off = size * (4 * values[:, None] * (1 + b.abs().sign() * (1 + entropy[:, None])) + 32 * U) + (r + U) * dz.abs()
        self.hidden = dz @ w
        self.weight = dz.t().contiguous() @ h
        # sums over the vocabulary (over rows) of products of numbers of either side, six times as many for fp32
        self.hidden_bound = off @ w.abs() + (6 * vocab + 64) * U * (dz.abs() @ w.abs()) + r * self.hidden.abs()
        self.weight_bound = off.t().contiguous() @ h.abs() + (6 * len(h) + 16) * U * (dz.abs().t().contiguous() @ h.abs()) + r * self.weight.abs()
        self.hidden = torch.where(live[:, None], self.hidden, 0.0)
        self.hidden_bound = torch.where(live[:, None], self.hidden_bound, 0.0)


def _check_values(r, want, targets):
    if targets is None:
        assert r.logprob is None
    else:
        _close(r.logprob, want.logprob, want.logprob_bound, "logprob")
    _close(r.entropy, want.entropy, want.entropy_bound, "entropy")


SIZES = [(1, 64, 1), (1, 1, 2), (2, 7, 5), (3, 33, 100), (8, 128, 1000), (15, 1000, 63), (16, 64, 4097), (17, 64, 127), (16, 200, 129), (33, 65, 128),
         (100, 192, 300), (127, 64, 257), (128, 128, 128), (129, 320, 1000), (300, 1000, 501), (257, 8, 3001), (1000, 64, 640)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_values(size, dtype):
    for k, (pad, shift, scale, ignored) in enumerate([(0, 0, 1.0, 0.3), (8, 0, 0.7, 0.0), (3, 1, 1.3, 0.6)]):
        hidden, weight, targets, _, _ = _inputs(*size, DTYPES[dtype], 1000 * size[0] + k, pad, shift, ignored)
        _check_values(asi.linear_logprobs(hidden, weight, targets, scale=scale), _Definition(hidden, weight, targets, scale), targets)
        _check_values(asi.linear_logprobs(hidden, weight, scale=scale), _Definition(hidden, weight, None, scale), None)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_gradients(size, dtype):
    for k, (pad, shift, scale, ignored) in enumerate([(0, 0, 1.0, 0.3), (8, 0, 0.7, 0.0), (3, 1, 1.3, 0.6)]):
        hidden, weight, targets, a, b = _inputs(*size, DTYPES[dtype], 2000 * size[0] + k, pad, shift, ignored)
        for wa, wb in ((a, None), (a, b), (None, b)):
            want = _Definition(hidden, weight, targets, scale, wa, wb)
            r = asi.linear_logprobs_grad(hidden, weight, targets, wa, wb, scale=scale)
            _check_values(r, want, targets)
            _close(r.hidden, want.hidden, want.hidden_bound, "hidden")
            _close(r.weight, want.weight, want.weight_bound, "weight")


@pytest.mark.parametrize("rows,dim,vocab,dtype", [(2100, 64, 20000, "bf16"), (2100, 65, 17000, "f32"), (20, 64, 40000, "f32"), (5000, 128, 7001, "bf16"),
                                                  (600, 1024, 2500, "bf16"), (9, 2048, 70001, "bf16"), (1100, 64, 39700, "f32"), (200, 72, 160000, "bf16")])
def test_several_pieces_of_the_vocabulary(rows, dim, vocab, dtype):
    hidden, weight, targets, a, b = _inputs(rows, dim, vocab, DTYPES[dtype], rows)
    want = _Definition(hidden, weight, targets, 1.0, a, b)
    r = asi.linear_logprobs_grad(hidden, weight, targets, a, b)
    _check_values(r, want, targets)
    _close(r.hidden, want.hidden, want.hidden_bound, "hidden")
    _close(r.weight, want.weight, want.weight_bound, "weight")
    again = asi.linear_logprobs_grad(hidden, weight, targets, a, b)
    assert all(torch.equal(x, y) for x, y in zip(r, again))                # equal calls, equal bits
    _check_values(asi.linear_logprobs(hidden, weight, targets), want, targets)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_autograd(dtype):
    hidden, weight, targets, a, b = _inputs(70, 96, 333, DTYPES[dtype], 5)
    want = asi.linear_logprobs_grad(hidden, weight, targets, a, b, scale=0.8)
    h, w = hidden.clone().requires_grad_(), weight.clone().requires_grad_()
    r = asi.linear_logprobs(h.view(7, 10, 96), w, targets.view(7, 10), scale=0.8)
    (r.logprob * a.view(7, 10) + r.entropy * b.view(7, 10)).sum().backward()
    assert torch.equal(r.logprob.flatten(), want.logprob) and torch.equal(r.entropy.flatten(), want.entropy)
    assert torch.equal(h.grad, want.hidden) and torch.equal(w.grad, want.weight)
    # one side only, one value only
    h2 = hidden.clone().requires_grad_()
    asi.linear_logprobs(h2, weight, targets, scale=0.8).logprob.sum().backward()
    one = asi.linear_logprobs_grad(hidden, weight, targets, torch.ones_like(a), scale=0.8, weight_grad=False)
    assert one.weight is None and torch.equal(h2.grad, one.hidden)
    w2 = weight.clone().requires_grad_()
    asi.linear_logprobs(hidden, w2, scale=0.8).entropy.sum().backward()
    one = asi.linear_logprobs_grad(hidden, weight, None, None, torch.ones_like(a), scale=0.8, hidden_grad=False)
    assert one.hidden is None and one.logprob is None and torch.equal(w2.grad, one.weight)
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(asi.linear_logprobs(h, w, targets).logprob.sum(), h, create_graph=True)
        g.sum().backward()


def test_gradients_against_differences():
    rows, dim, vocab, step = 24, 40, 90, 2.0 ** -6
    hidden, weight, targets, a, _ = _inputs(rows, dim, vocab, torch.float32, 11, ignored=0.2)
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    for side in ("hidden", "weight"):
        x = dict(hidden=hidden, weight=weight)[side]
        d = torch.randn(x.shape, generator=_gen(12), device="cuda") * dim ** -0.5
        at = lambda s: (dict(hidden=hidden, weight=weight) | {side: x + s * d})  # noqa: E731,B023
        both = [asi.linear_logprobs(at(s)["hidden"], at(s)["weight"], targets).logprob.double() @ a.double() for s in (step, -step)]
        slope = float((getattr(r, side).double() * d.double()).sum())
        want = _Definition(hidden, weight, targets, 1.0, a)
        # values' errors over 2 step; what x + step d is rounded by, at most U of it a side; the third derivative of a log sum along a
        # direction in which the logits change by m is at most their range's third power, 8 m^3
        move = (d.double() @ weight.double().t()).abs() if side == "hidden" else (hidden.double() @ d.double().t()).abs()
        rounding = U * 2 * ((hidden.double().abs() + step) @ (weight.double().abs() + step).t()).amax(-1)
        bound = ((want.logprob_bound * 2 + 2 * rounding) / (2 * step) + step ** 2 / 6 * 8 * move.amax(-1) ** 3) @ a.double().abs()
        slope_bound = float((getattr(want, side + "_bound") * d.double().abs()).sum())
        assert abs(float(both[0] - both[1]) / (2 * step) - slope) <= float(bound) + slope_bound


@pytest.mark.parametrize("rows", [7, 200])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_that_are_left_out(rows, dtype):
    hidden, weight, targets, a, b = _inputs(rows, 64, 300, DTYPES[dtype], 3, ignored=0.0)
    out = torch.arange(rows, device="cuda") % 3 == 1
    targets[out] = IGNORE
    clean = asi.linear_logprobs_grad(hidden, weight, targets, a, b)
    hidden[out] = NAN                                                     # padding may hold anything
    a[out], b[out] = INF, NAN
    r = asi.linear_logprobs_grad(hidden, weight, targets, a, b)
    assert all(torch.equal(x, y) for x, y in zip(r, clean))
    assert not r.logprob[out].any() and not r.entropy[out].any() and not r.hidden[out].any()
    f = asi.linear_logprobs(hidden, weight, targets)
    assert not f.logprob[out].any() and not f.entropy[out].any() and not torch.isnan(f.logprob).any()
    targets[:] = IGNORE
    r = asi.linear_logprobs_grad(hidden, weight, targets, a, b)
    assert not any(t.any() for t in r)
    assert not any(t.any() for t in asi.linear_logprobs(hidden, weight, targets))


@pytest.mark.parametrize("rows", [5, 150])
def test_targets_out_of_range_and_rows_that_are_not_numbers(rows):
    hidden, weight, targets, a, _ = _inputs(rows, 64, 200, torch.float32, 4, ignored=0.0)
    targets[1], targets[2] = 200, -1
    hidden[3, 5] = NAN
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    want = _Definition(hidden[:1], weight, targets[:1], 1.0, a[:1])
    assert torch.isnan(r.logprob[1:4]).all() and torch.isnan(r.hidden[1:4]).all() and torch.isnan(r.entropy[3])
    assert not torch.isnan(r.entropy[:3]).any() and not torch.isnan(r.logprob[4:]).any()
    _close(r.hidden[:1], want.hidden, want.hidden_bound, "hidden")
    assert torch.isnan(r.weight).all()
    f = asi.linear_logprobs(hidden, weight, targets)
    assert torch.isnan(f.logprob[1:4]).all() and not torch.isnan(f.entropy[:3]).any()


@pytest.mark.parametrize("rows", [3, 40])
def test_logits_of_infinity(rows):
    """A token whose weights hold -infinity in a column that every hidden state has at 1 may not come."""
    hidden, weight, targets, a, _ = _inputs(rows, 64, 300, torch.bfloat16, 6, ignored=0.0)
    hidden[:, 7] = 1.0
    never = torch.arange(300, device="cuda") % 4 == 1
    targets[never[targets]] = 0
    weight[never, 7] = -INF
    r = asi.linear_logprobs(hidden, weight, targets)
    kept = weight[~never].clone()
    place = torch.cumsum(~never, 0) - 1
    want = _Definition(hidden, kept, place[targets], 1.0)
    _check_values(r, want, targets)
    weight[:, 7] = -INF
    r = asi.linear_logprobs(hidden, weight, targets)
    assert (r.logprob == -INF).all() and not r.entropy.any()
    weight[5, 7] = INF
    assert torch.isnan(asi.linear_logprobs(hidden, weight, targets).logprob).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_large_logits_and_scales(dtype):
    """Logits of thousands, of which one or a few matter, and scales far from one."""
    for spread, scale in ((1000.0, 1.0), (2.5, 100.0), (2.5e4, 1e-4), (1e-3, 1e-3)):
        hidden, weight, targets, a, b = _inputs(50, 128, 700, DTYPES[dtype], 8, spread=spread)
        want = _Definition(hidden, weight, targets, scale, a, b)
        r = asi.linear_logprobs_grad(hidden, weight, targets, a, b, scale=scale)
        _check_values(r, want, targets)
        _close(r.hidden, want.hidden, want.hidden_bound, "hidden")
        _close(r.weight, want.weight, want.weight_bound, "weight")


@pytest.mark.parametrize("rows", [1, 5, 30, 300])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_nearly_sure_tokens(rows, dtype):
    """Log probabilities of targets with p near 1, and their gradients, are good to a share of themselves, not of 1: what is left is
    the others' sum, each of whose terms is off by twice the logits' error and a few roundings."""
    dim, vocab = 64, 700
    hidden, weight, targets, a, _ = _inputs(rows, dim, vocab, DTYPES[dtype], 16, ignored=0.0, spread=0.8)
    # the target's logit is about 24 * 64 * 0.01 = 15, the others' have a deviation of about 2: 700 of them sum up to 700 e^2 e^-15 = 2^-9 of it
    hidden = (hidden.float() + 24.0 * weight[targets].float()).to(hidden.dtype)
    z = hidden.double() @ weight.double().t().contiguous()
    e = (6 * dim + 16) * U * (hidden.double().abs() @ weight.double().abs().t().contiguous()).amax(-1)
    at = targets[:, None]
    others = (z - z.gather(1, at)).scatter(1, at, -INF).exp().sum(-1)
    assert float(others.min()) < 2.0 ** -8
    want = -torch.log1p(others)
    share = 2 * e + 256 * U
    for r in (asi.linear_logprobs(hidden, weight, targets), asi.linear_logprobs_grad(hidden, weight, targets, a)):
        _close(r.logprob, want, share * want.abs(), "logprob")
    # rows of which the target's own part of dz, a (1 - p), is all that W's row of it meets: the sum over the vocabulary cancels for
    # weights that are all the same, so dz is looked at through weights that are zero but for one token
    one = torch.zeros_like(weight)
    token = int(targets[0])
    one[token] = weight[token]
    r = asi.linear_logprobs_grad(hidden[:1], one, targets[:1], a[:1])
    z0 = (hidden[:1].double() @ one[token].double())[0]
    rest = (vocab - 1) * (-z0).exp()
    dz = float(a[0]) * float(rest / (1 + rest))
    want = dz * one[token].double()[None]
    bound = ((2 * e[0] + 256 * U + 2 * _round(weight.dtype)) * want.abs())
    _close(r.hidden, want, bound, "hidden")


def test_layouts():
    hidden, weight, targets, a, _ = _inputs(60, 64, 500, torch.bfloat16, 9)
    want = asi.linear_logprobs_grad(hidden, weight, targets, a)
    assert torch.equal(asi.linear_logprobs_grad(hidden.view(3, 20, 64), weight, targets.view(3, 20), a.view(3, 20)).hidden, want.hidden.view(3, 20, 64))
    across = hidden.t().contiguous().t()                                  # a row's entries are not next to each other
    assert torch.equal(asi.linear_logprobs_grad(across, weight, targets, a).weight, want.weight)
    apart = torch.empty(3, 25, 64, device="cuda", dtype=torch.bfloat16)
    apart[:, :20] = hidden.view(3, 20, 64)
    r = asi.linear_logprobs_grad(apart[:, :20], weight, targets.view(3, 20), a.view(3, 20))
    assert torch.equal(r.hidden.reshape(60, 64), want.hidden) and torch.equal(r.weight, want.weight)
    one = hidden[:1].expand(60, 64)                                       # rows at distance 0
    assert torch.equal(asi.linear_logprobs(one, weight, targets).logprob, asi.linear_logprobs(one.contiguous(), weight, targets).logprob)
    for n in (0,):
        none = asi.linear_logprobs_grad(hidden[:n], weight, targets[:n], a[:n])
        assert none.hidden.shape == (0, 64) and none.logprob.shape == (0,) and none.weight.shape == weight.shape and not none.weight.any()
        assert asi.linear_logprobs(hidden[:n], weight, targets[:n]).entropy.shape == (0,)


def test_another_stream_and_a_graph_with_eager_work_between_replays():
    hidden, weight, targets, a, _ = _inputs(300, 128, 2000, torch.bfloat16, 10)
    few = hidden[:4].clone()
    want = asi.linear_logprobs_grad(hidden, weight, targets, a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(r, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = asi.linear_logprobs_grad(hidden, weight, targets, a)
        values = asi.linear_logprobs(few, weight, targets[:4])
    for seed in range(4):
        h, _, t, _, _ = _inputs(300, 128, 2000, torch.bfloat16, 20 + seed, ignored=0.2 * seed)      # other rows are left out
        hidden.copy_(h)
        targets.copy_(t)
        few.copy_(h[:4])
        graph.replay()
        eager = asi.linear_logprobs_grad(h, weight, t, a)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, eager))
        assert torch.equal(values.logprob, asi.linear_logprobs(h[:4], weight, t[:4]).logprob)


def test_backward_into_a_graph():
    hidden, weight, targets, a, _ = _inputs(64, 64, 300, torch.float32, 13)
    want = asi.linear_logprobs_grad(hidden, weight, targets, a)
    h, w = hidden.clone().requires_grad_(), weight.clone().requires_grad_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(asi.linear_logprobs(h, w, targets).logprob, (h, w), a)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want.hidden) and torch.equal(got[1], want.weight)


@pytest.mark.skip(reason="torch's engine joins the captured stream with that of the leaves' living eager graph, which ends the capture and the "
                         "process; no operator can see it beforehand")
def test_backward_into_a_graph_while_an_eager_graph_of_the_same_leaves_lives():
    hidden, weight, targets, _, _ = _inputs(64, 64, 300, torch.float32, 13)
    h, w = hidden.clone().requires_grad_(), weight.clone().requires_grad_()
    lives = asi.linear_logprobs(h, w, targets).logprob.sum()
    want = torch.autograd.grad(asi.linear_logprobs(h, w, targets).logprob.sum(), (h, w))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = torch.autograd.grad(asi.linear_logprobs(h, w, targets).logprob.sum(), (h, w))
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    lives.backward()
    assert torch.equal(h.grad, want[0]) and torch.equal(w.grad, want[1])


def test_memory_stays_below_the_logits():
    rows, dim, vocab = 4096, 256, 64000
    hidden, weight, targets, a, _ = _inputs(rows, dim, vocab, torch.bfloat16, 14)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    used = torch.cuda.max_memory_allocated() - before - sum(t.numel() * t.element_size() for t in r)
    assert used < rows * vocab * 2 / 3                                    # the logits in bf16 are 524 MB
    assert math.isfinite(float(r.logprob.sum()))


def test_refusals():
    hidden, weight, targets, a, b = _inputs(6, 64, 100, torch.float32, 15)
    f, g = asi.linear_logprobs, asi.linear_logprobs_grad
    for bad in (lambda: f(hidden, weight[:, :32], targets), lambda: f(hidden, weight.bfloat16(), targets), lambda: f(hidden, weight[0], targets),
                lambda: f(hidden, weight, targets[:5]), lambda: f(hidden, weight.t().contiguous().t(), targets), lambda: f(hidden.cpu(), weight, targets),
                lambda: f(hidden, weight, targets.cpu()), lambda: g(hidden, weight, None, a), lambda: g(hidden, weight, targets, a[:3]),
                lambda: g(hidden, weight, targets, a.double()), lambda: f(hidden, weight[:0], targets)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(hidden.half(), weight.half(), targets), lambda: f(hidden, weight, targets.int())):
        with pytest.raises(TypeError):
            bad()
    for scale in (0.0, -1.0, NAN, INF, 1e30):
        with pytest.raises(asi.AsiError):
            f(hidden, weight, targets, scale=scale)
    with forward_ad.dual_level(), pytest.raises(NotImplementedError):
        f(forward_ad.make_dual(hidden, hidden), weight, targets)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,dim,vocab", [(rows, 8, 9001) for rows in (1, 5, 16, 17, 33, 40, 48, 49, 65, 97, 100, 112, 113, 128, 129, 300)] +
                         [(rows, 600, 1100) for rows in (17, 65, 129, 300)])
def test_nothing_is_written_behind_the_workspace(rows, dim, vocab, dtype):
    """A workspace of the stated size, full of NaN; what lies behind it stays as it is.  A narrow head over a large vocabulary has little
    behind its logits that a store too many could fall on."""
    hidden, weight, targets, a, b = _inputs(rows, dim, vocab, DTYPES[dtype], 40 + rows)
    want = _Definition(hidden, weight, targets, 1.0, a, b)
    desc = B.LinearLogprobDesc(rows, dim, vocab, hidden.stride(0), weight.stride(0), IGNORE, _DTYPE[hidden.dtype], 1.0, 0, 0)
    L = B.lib()
    for f in (L.asi_linear_logprobs_workspace_bytes, L.asi_linear_logprobs_grad_workspace_bytes):
        size = f(desc)
        ws = torch.full((size + (1 << 22),), 255, dtype=torch.uint8, device="cuda")
        logprob, entropy = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        if f is L.asi_linear_logprobs_workspace_bytes:
            status = L.asi_linear_logprobs(desc, hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), logprob.data_ptr(), entropy.data_ptr(),
                                           None, ws.data_ptr(), size, st)
        else:
            dh, dw = torch.empty_like(hidden), torch.empty_like(weight)
            status = L.asi_linear_logprobs_grad(desc, 0, hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), None, logprob.data_ptr(),
                                                entropy.data_ptr(), a.data_ptr(), b.data_ptr(), dh.data_ptr(), dw.data_ptr(), ws.data_ptr(), size, st)
            _close(dh, want.hidden, want.hidden_bound, "hidden")
            _close(dw, want.weight, want.weight_bound, "weight")
        assert status == 0
        _check_values(LinearLogprobs(logprob, entropy), want, targets)
        assert bool((ws[size:] == 255).all())


@pytest.mark.parametrize("rows,dim,vocab,dtype", [(40, 640, 3000, "bf16"), (100, 1024, 777, "bf16"), (300, 513, 1300, "bf16"), (1400, 512, 12000, "bf16"),
                                                  (70, 100, 4000, "f32"), (300, 129, 1111, "f32"), (1400, 128, 12000, "f32")])
def test_logits_that_are_kept_and_computed_again(rows, dim, vocab, dtype):
    """A call of both keeps the logits of these sizes, a backward pass behind a forward one computes them again: the same bits."""
    hidden, weight, targets, a, b = _inputs(rows, dim, vocab, DTYPES[dtype], 50 + rows)
    want = _Definition(hidden, weight, targets, 0.9, a, b)
    r = asi.linear_logprobs_grad(hidden, weight, targets, a, b, scale=0.9)
    _check_values(r, want, targets)
    _close(r.hidden, want.hidden, want.hidden_bound, "hidden")
    _close(r.weight, want.weight, want.weight_bound, "weight")
    h, w = hidden.clone().requires_grad_(), weight.clone().requires_grad_()
    again = asi.linear_logprobs(h, w, targets, scale=0.9)
    dh, dw = torch.autograd.grad((again.logprob, again.entropy), (h, w), (a, b))
    assert torch.equal(dh, r.hidden) and torch.equal(dw, r.weight)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_kept_logits_in_a_graph_whose_rows_change(dtype):
    hidden, weight, targets, a, _ = _inputs(300, 576, 2000, DTYPES[dtype], 60, ignored=0.0)
    asi.linear_logprobs_grad(hidden, weight, targets, a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = asi.linear_logprobs_grad(hidden, weight, targets, a)
    for seed in range(4):
        h, _, t, _, _ = _inputs(300, 576, 2000, DTYPES[dtype], 61 + seed, ignored=0.33 * seed)
        hidden.copy_(h)
        targets.copy_(t)
        graph.replay()
        eager = asi.linear_logprobs_grad(h, weight, t, a)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, eager))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,dim,ignored", [(4, 64, False), (16, 64, False), (40, 64, False), (100, 64, False), (256, 128, False), (258, 192, False), (700, 384, False),
                                              (700, 193, True), (2000, 512, True)])
def test_the_gradient_of_logits_is_not_rounded_to_bf16(rows, dim, ignored, dtype):
    """bf16 results are rounded once, however many rows there are, with or without a target.  All tokens have the same weights w, so p is
    1 / vocab; rows come in pairs with hidden states 1 and -1 in a column of their own, one target, and factors a and a (1 + 2^-9): what is
    left of dW in that column is 2^-9 of either summand, and nothing of dH, whose row sums dz to 0 times w."""
    vocab, g = 500, _gen(70 + rows)
    live = torch.arange(rows, device="cuda") // 2 % 2 == 0 if ignored else torch.ones(rows, dtype=torch.bool, device="cuda")
    row = torch.arange(int(live.sum()), device="cuda")
    hidden = torch.randn(rows, dim, generator=g, device="cuda")
    small = torch.zeros(len(row), dim, device="cuda")
    small[row, row // 2] = 1.0 - 2.0 * (row % 2)
    hidden[live] = small
    hidden = hidden.to(DTYPES[dtype])
    w = torch.randn(dim, generator=g, device="cuda").to(DTYPES[dtype])
    targets = torch.full((rows,), IGNORE, device="cuda")
    targets[live] = torch.randint(0, vocab, (len(row) // 2,), generator=g, device="cuda").repeat_interleave(2)
    a = torch.zeros(rows, device="cuda")
    a[live] = (1.0 + torch.rand(len(row) // 2, generator=g, device="cuda")).repeat_interleave(2) * (1.0 + 2.0 ** -9 * (row % 2))
    r = asi.linear_logprobs_grad(hidden, w.expand(vocab, dim).contiguous(), targets, a)
    size, at = a[live].double(), targets[live]
    p = 1.0 / vocab
    dz = torch.full((len(row), vocab), -p, dtype=torch.float64, device="cuda").scatter_(1, at[:, None], 1.0 - p) * size[:, None]
    # the logarithm of 500, 6.2, is off by 2 roundings of itself and of its product with log2 e: p by 30 U of itself, with the exponential's
    # and the products' roundings 40 U; two parts of bf16 hold 2^-16, three 2^-24, and for up to 16 rows it is fp32.  Sums over the rows of
    # products of which two are not 0, over the vocabulary of 500 (six times as many for fp32); the result's rounding
    off = (2.0 ** -16 if dtype == "bf16" and rows > 16 else U) + 40 * U
    times = 1 if dtype == "bf16" else 6
    want = dz.t().contiguous() @ small.double()
    each = dz.abs().t().contiguous() @ small.double().abs()
    _close(r.weight, want, (off + 4 * times * U) * each * (1 + U) + _round(hidden.dtype) * want.abs(), "weight")
    _close(r.hidden[live], torch.zeros(len(row), dim, device="cuda"), (off + (times * vocab + 64) * U) * dz.abs().sum(-1, keepdim=True) * w.double().abs(), "hidden")


def _shares(hidden, weight, targets, a):
    """_Definition's values and gradients and their bounds where a row of W is too long and there are too many of them for all of that in 64 bits
    at once: in pieces of the vocabulary, by the one identity log p = z - log sum exp z."""
    rows, dim, vocab = len(hidden), weight.shape[1], weight.shape[0]
    r = _round(hidden.dtype)
    live = targets != IGNORE
    h = torch.where(live[:, None], hidden.double(), 0.0)
    pieces = [slice(i, min(vocab, i + 4096)) for i in range(0, vocab, 4096)]
    z, size = torch.empty(rows, vocab, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    for s in pieces:
        w = weight[s].double()
        z[:, s] = h @ w.t().contiguous()
        size = torch.maximum(size, (h.abs() @ w.abs().t().contiguous()).amax(-1))
    logp = z - torch.logsumexp(z, -1, keepdim=True)
    p = logp.exp()
    entropy = torch.special.entr(p).sum(-1)
    times = 6 if hidden.dtype == torch.float32 else 1                     # products of bf16 numbers are exact
    values = 2 * (times * dim + 16) * U * size + U * (8 * z.abs().amax(-1) + 256)
    hot = torch.zeros_like(z).scatter_(1, torch.where(live, targets, 0)[:, None], 1.0)
    a = torch.where(live, a.double(), 0.0)[:, None]
    dz = a * (hot - p)
    off = a.abs() * (hot + p) * (4 * values[:, None] + 32 * U) + (2.0 ** -16 + U) * dz.abs()
    dh, dh_bound, near = (torch.zeros(rows, dim, dtype=torch.float64, device="cuda") for _ in range(3))
    for s in pieces:
        w = weight[s].double()
        dh += dz[:, s] @ w
        dh_bound += off[:, s] @ w.abs()
        near += dz[:, s].abs() @ w.abs()
    dh_bound += (6 * vocab + 64) * U * near + r * dh.abs()
    some = torch.cat([torch.arange(i, min(vocab, i + 97), device="cuda") for i in range(0, vocab, 4096 - 97)])      # of dW: rows of every piece
    part = dz[:, some].t().contiguous()
    dw = part @ h
    dw_bound = off[:, some].t().contiguous() @ h.abs() + (6 * rows + 16) * U * (part.abs() @ h.abs()) + r * dw.abs()
    return (torch.where(live, logp.gather(1, torch.where(live, targets, 0)[:, None])[:, 0], 0.0), torch.where(live, entropy, 0.0),
            torch.where(live, values, 0.0), torch.where(live, values * (2 + entropy), 0.0), dh, dh_bound, some, dw, dw_bound)


@pytest.mark.parametrize("rows,dim,vocab,dtype", [(200, 5120, 70000, "f32"), (200, 5120, 78336, "f32"), (256, 8192, 65536, "f32"), (512, 8320, 70000, "f32"),
                                                  (200, 12353, 70001, "bf16")])
def test_wide_heads_whose_pieces_take_smaller_tiles(rows, dim, vocab, dtype):
    """Rows of W so long that a piece of packed ones has too few tiles of 256 for the chip, the vocabulary an exact number of pieces or not."""
    # logits near 0, whose bounds are near 0.05: a part of the vocabulary that is lost moves the logarithm by more
    hidden, weight, targets, a, _ = _inputs(rows, dim, vocab, DTYPES[dtype], 80 + rows, spread=0.25)
    logprob, entropy, lp_bound, e_bound, dh, dh_bound, some, dw, dw_bound = _shares(hidden, weight, targets, a)
    desc = B.LinearLogprobDesc(rows, dim, vocab, dim, dim, IGNORE, _DTYPE[hidden.dtype], 1.0, 0, 0)
    L = B.lib()
    st = torch.cuda.current_stream().cuda_stream
    for f in (L.asi_linear_logprobs_workspace_bytes, L.asi_linear_logprobs_grad_workspace_bytes):
        size = f(desc)
        ws = torch.full((size + (1 << 24),), 255, dtype=torch.uint8, device="cuda")
        lp, en = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        if f is L.asi_linear_logprobs_workspace_bytes:
            assert L.asi_linear_logprobs(desc, hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), lp.data_ptr(), en.data_ptr(), None,
                                         ws.data_ptr(), size, st) == 0
        else:
            got_h, got_w = torch.empty_like(hidden), torch.empty_like(weight)
            assert L.asi_linear_logprobs_grad(desc, 0, hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), None, lp.data_ptr(), en.data_ptr(),
                                              a.data_ptr(), None, got_h.data_ptr(), got_w.data_ptr(), ws.data_ptr(), size, st) == 0
            _close(got_h, dh, dh_bound, "hidden")
            _close(got_w[some], dw, dw_bound, "weight")
        assert float(lp_bound.max()) < 0.1
        _close(lp, logprob, lp_bound, "logprob")
        _close(en, entropy, e_bound, "entropy")
        assert bool((ws[size:] == 255).all())
        del ws


@pytest.mark.parametrize("rows", [40, 65, 129, 300])
def test_infinite_and_largest_weights_in_fp32(rows):
    """As in bf16: tokens that -infinity in a column takes out, while what is multiplied has bits in every part of it; numbers above bf16's
    largest are numbers; an infinite hidden state makes logits of either infinity."""
    hidden, weight, targets, a, _ = _inputs(rows, 64, 300, torch.float32, 90, ignored=0.0)
    a *= 2.0 ** -10
    hidden[:, 7] = 1.0
    hidden[1::2, 7] = 1.0 + torch.rand(len(hidden[1::2]), generator=_gen(91), device="cuda")
    hidden[:, 9] = 2.0 ** -122
    weight[10:20, 9] = 3.4e38 * torch.tensor([1.0, -1.0], device="cuda").repeat(5)       # products of 64
    never = torch.arange(300, device="cuda") % 4 == 1
    targets[never[targets]] = 0
    kept, place = weight[~never].clone(), torch.cumsum(~never, 0) - 1
    want = _Definition(hidden, kept, place[targets], 1.0, a)
    weight[never, 7] = -INF
    _check_values(asi.linear_logprobs(hidden, weight, targets), want, targets)
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    _check_values(r, want, targets)
    others = torch.arange(64, device="cuda") != 7
    # the logits are up to 64 apart and more, so that p goes below 2^-126, the least normal number, where fp32 may hold 0: that is another 2^-126
    # that a dz or one of its three parts may be off by, and with it their products, six of which make one, may be as well (hidden states of 2^-122)
    least = 2.0 ** -126
    hidden_bound = want.hidden_bound + least * (3 * kept.double().abs().sum(0) + 6 * len(kept) + 1)
    weight_bound = want.weight_bound + least * (3 * hidden.double().abs().sum(0) + 6 * rows + 1)
    _close(r.hidden[:, others], want.hidden[:, others], hidden_bound[:, others], "hidden")
    assert torch.isnan(r.hidden[:, 7]).all()                              # 0 times infinity, as in dz @ W
    _close(r.weight[~never], want.weight, weight_bound, "weight")
    assert not r.weight[never].any()
    h, w = hidden.clone().requires_grad_(), weight.clone().requires_grad_()
    dh, dw = torch.autograd.grad(asi.linear_logprobs(h, w, targets).logprob, (h, w), a)
    assert torch.equal(dh[:, others], r.hidden[:, others]) and torch.equal(dw, r.weight)
    weight[:, 7] = -INF
    r = asi.linear_logprobs(hidden, weight, targets)
    assert (r.logprob == -INF).all() and not r.entropy.any()
    hidden[2, 7] = -1.5                                                   # and now +infinity
    r = asi.linear_logprobs(hidden, weight, targets)
    assert torch.isnan(r.logprob[2]) and (r.logprob[torch.arange(rows, device="cuda") != 2] == -INF).all()
    hidden[2, 7] = INF                                                    # infinity on both sides
    assert (asi.linear_logprobs(hidden, weight, targets).logprob == -INF).all()
    weight[:, 7] = 1.0
    r = asi.linear_logprobs(hidden, weight, targets)
    assert torch.isnan(r.logprob[2]) and torch.isfinite(r.logprob[3:]).all()
    hidden[2, 7] = -INF
    assert asi.linear_logprobs(hidden, weight, targets).logprob[2] == -INF


@pytest.mark.parametrize("rows", [3, 40, 100, 300])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_an_infinite_share_gives_infinite_gradients(rows, dtype):
    """A row's factor of infinity, an overflow say, is one in dW, with the sign of its terms, and no NaN beside what it does not cancel with."""
    hidden, weight, targets, a, _ = _inputs(rows, 64, 300, DTYPES[dtype], 95, ignored=0.0)
    hidden[0] = torch.where(hidden[0] >= 0, 1.0, -0.5).to(hidden.dtype)  # parts of it are 0
    a[0] = INF
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    hot = torch.nn.functional.one_hot(targets[0], 300) * 2 - 1
    assert torch.equal(r.weight, (hot[:, None] * hidden[0][None].sign() * INF).to(weight.dtype))
    want = _Definition(hidden[1:], weight, targets[1:], 1.0, a[1:])
    _close(r.hidden[1:], want.hidden, want.hidden_bound, "hidden")


@pytest.mark.parametrize("rows", [3, 12, 40, 150])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_a_left_out_rows_gradient_is_zero_beside_infinite_weights(rows, dtype):
    hidden, weight, targets, a, _ = _inputs(rows, 64, 300, DTYPES[dtype], 97, ignored=0.0)
    targets[1::2] = IGNORE
    weight[:, 7] = INF
    weight[5, 9] = NAN
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    assert not r.hidden[1::2].any() and not r.logprob[1::2].any() and not r.entropy[1::2].any()
    assert torch.isnan(r.hidden[::2]).all()
    h = hidden.clone().requires_grad_()
    dh, = torch.autograd.grad(asi.linear_logprobs(h, weight, targets).logprob, h, a)
    assert not dh[1::2].any()


@pytest.mark.parametrize("rows,dim,vocab,dtype", [(33, 72, 700, "bf16"), (40, 1000, 3000, "bf16"), (64, 200, 3000, "bf16"), (20, 1000, 3000, "bf16"),
                                                  (40, 128, 3000, "bf16"), (40, 72, 700, "f32"), (64, 1000, 2000, "f32"), (12, 128, 3000, "bf16"), (65, 72, 700, "f32")])
def test_nearly_sure_tokens_through_autograd(rows, dim, vocab, dtype):
    """The backward pass makes the logits in the order in which the forward pass made those that its statistics are of: the same bits as one call
    gives, and a (1 - p) to a share of itself where p is nearly 1."""
    hidden, weight, targets, a, _ = _inputs(rows, dim, vocab, DTYPES[dtype], 98, ignored=0.0, spread=0.8)
    hidden = (hidden.float() + 24.0 * weight[targets].float()).to(hidden.dtype)      # a target's logit is about 15, the others' are below 5
    h, w = hidden.clone().requires_grad_(), weight.clone().requires_grad_()
    dh, dw = torch.autograd.grad(asi.linear_logprobs(h, w, targets).logprob, (h, w), a)
    r = asi.linear_logprobs_grad(hidden, weight, targets, a)
    assert torch.equal(dh, r.hidden) and torch.equal(dw, r.weight)


@pytest.mark.parametrize("rows", [3, 100])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_logits_farther_apart_than_fp32_reaches(rows, dtype):
    """Logits of 2^127 and -2^127 are 2^128 apart, which fp32 does not hold, and 3.4e18 at a scale of 1e-20."""
    dim, vocab = 64, 40
    hidden = torch.zeros(rows, dim, dtype=DTYPES[dtype], device="cuda")
    weight = torch.zeros(vocab, dim, dtype=DTYPES[dtype], device="cuda")
    hidden[:, 3], weight[:, 3] = 2.0 ** 63, -2.0 ** 64
    weight[7, 3] = 2.0 ** 64
    targets = torch.arange(rows, device="cuda") % vocab
    scale = 1e-20
    a = torch.ones(rows, device="cuda")
    far = (2.0 ** 128) * float(torch.tensor(scale))
    want = torch.where(targets == 7, 0.0, -far).double()
    for r in (asi.linear_logprobs(hidden, weight, targets, scale=scale), asi.linear_logprobs_grad(hidden, weight, targets, a, scale=scale)):
        _close(r.logprob, want, 4 * U * want.abs(), "logprob")
        assert not r.entropy.any()
    # dz is scale (1 at the target, -1 at token 7): two products of numbers with few bits, the scale's rounding, the result's
    want = torch.where(targets == 7, 0.0, -far / 2.0 ** 63).double()
    _close(r.hidden[:, 3], want, (4 * U + (2.0 ** -8 + 2.0 ** -15 if dtype == "bf16" else 0.0)) * want.abs(), "hidden")


def test_no_rows_beside_more_weights_than_a_launch_has_threads():
    weight = torch.empty(1 << 20, 4104, dtype=torch.bfloat16, device="cuda")
    hidden = torch.empty(0, 4104, dtype=torch.bfloat16, device="cuda")
    targets = torch.empty(0, dtype=torch.int64, device="cuda")
    L, out = B.lib(), torch.full((weight.numel() + 64,), 1.0, dtype=torch.bfloat16, device="cuda")
    desc = B.LinearLogprobDesc(0, 4104, 1 << 20, 4104, 4104, IGNORE, _DTYPE[torch.bfloat16], 1.0, 0, 0)
    assert L.asi_linear_logprobs_grad(desc, 0, None, weight.data_ptr(), None, None, None, None, None, None, None, out.data_ptr(), None, 0,
                                      torch.cuda.current_stream().cuda_stream) == 0
    assert not out[:weight.numel()].any() and bool((out[weight.numel():] == 1).all())
    del out
    assert not asi.linear_logprobs_grad(hidden, weight, targets, torch.empty(0, device="cuda")).weight.any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", [(3, 70001, 130), (12, 65536, 200), (40, 20000, 300), (100, 16384, 257), (300, 9001, 500), (2, 262143, 65)])
def test_wide_heads_of_few_rows_and_tokens(size, dtype):
    hidden, weight, targets, a, b = _inputs(*size, DTYPES[dtype], 99, spread=0.25)
    want = _Definition(hidden, weight, targets, 1.0, a, b)
    _check_values(asi.linear_logprobs(hidden, weight, targets), want, targets)
    r = asi.linear_logprobs_grad(hidden, weight, targets, a, b)
    _check_values(r, want, targets)
    _close(r.hidden, want.hidden, want.hidden_bound, "hidden")
    _close(r.weight, want.weight, want.weight_bound, "weight")
