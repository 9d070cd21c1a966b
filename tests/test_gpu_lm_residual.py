"""The edge between two blocks (asi_residual_norm) against its definition in 64 bits.

U = 2^-24 is half an fp32 ulp.  A row's sums are of terms added in chains of at most 32 in a lane, 6 across lanes and 8 across waves, so
that a sum of squares is off by fewer than 48 U of itself and its root by 24 U; with the root's, the quotient's and the products' own
roundings, 64 U bounds what a norm's output is off by, 128 U what has been through two of them, relative to the magnitudes that are added.
"""
import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

import paper_2505_05086_amd as asi
from test_gpu_lm_dropout import kept

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")]


def _round(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def _close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bound = torch.as_tensor(bound, dtype=torch.float64, device=got.device).expand_as(want)
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), f"{what}: not finite elsewhere"
    off = ((got - want).abs() - bound)[torch.isfinite(want)]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{what}: {float(off.max()):.3g} over its bound"


def _rms(x, eps):
    return 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()


class Case:
    def __init__(self, shape, stream="f32", dtype="f32", gate=None, p=0.0, scale=1.0, post_norm=True, gains=True, gain_dtype=None, eps=1e-6, seed=1):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        dim = shape[-1]
        gd = DTYPES[gain_dtype or dtype]
        self.x, self.y = randn(*shape).to(DTYPES[stream]), (0.7 * randn(*shape)).to(DTYPES[dtype])
        self.post = (1 + 0.2 * randn(dim)).to(gd) if gains and post_norm else None
        self.pre = (1 + 0.2 * randn(dim)).to(gd) if gains else None
        self.gate = None if gate is None else (0.5 + 0.3 * randn(*gate)).to(gd)
        self.ds, self.do = randn(*shape).to(DTYPES[stream]), randn(*shape).to(DTYPES[dtype])
        self.options = dict(post_norm=post_norm, scale=scale, eps=eps, p=p, seed=12345 if p else None, offset=3)
        n = int(np.prod(shape))
        self.keep = torch.from_numpy(kept(0, n, p, 12345, 3)).cuda().view(shape).double() * (65536 / (65536 - round(p * 65536))) if p else 1.0

    def one(self, t):
        return 1.0 if t is None else t.double()

    def run(self):
        return asi.residual_norm(self.x, self.y, self.post, self.gate, self.pre, **self.options)

    def grad(self, stream, ds="given", do="given"):
        return asi.residual_norm_grad(self.ds if ds == "given" else ds, self.do if do == "given" else do, stream, self.y, self.post, self.gate,
                                      self.pre if self.pre is not None else None, **self.options)

    def check(self):
        o = self.options
        y, gate, post, pre = self.y.double(), self.one(self.gate), self.one(self.post), self.one(self.pre)
        ry = _rms(y, o["eps"]) if o["post_norm"] else 1.0
        u = y * ry
        add = o["scale"] * gate * self.keep * post * u
        r = self.run()
        want = self.x.double() + add
        _close(r.stream, want, 64 * U * add.abs() + (_round(self.x.dtype) + U) * (want.abs() + 64 * U * add.abs()), "stream")
        s = r.stream.double()                                            # the norm is that of the stream as it is held
        rs = _rms(s, o["eps"])
        out = s * rs * pre
        _close(r.out, out, (64 * U + _round(self.y.dtype)) * out.abs(), "out")
        for ds, do in ((self.ds, self.do), (None, self.do), (self.ds, None)):
            self.check_grad(r.stream, ds, do, u, ry, s, rs, gate, post, pre)
        return r

    def check_grad(self, stream, ds, do, u, ry, s, rs, gate, post, pre):
        o = self.options
        d = self.grad(stream, ds, do)
        dsd, dod = (0.0 if t is None else t.double() for t in (ds, do))
        v = s * rs
        g = dod * pre * torch.ones_like(s)
        dx = dsd + rs * (g - v * (g * v).mean(-1, keepdim=True)) * (0 if do is None else 1)
        size = abs(dsd) + rs * (g.abs() + v.abs() * (g * v).abs().mean(-1, keepdim=True))      # magnitudes that are added up
        _close(d.x, dx, 128 * U * size + _round(stream.dtype) * dx.abs(), "dx")
        rows = s[..., 0].numel()
        many = (128 + rows) * U                                           # and as many additions as there are rows
        over = tuple(range(s.dim() - 1))
        if do is None:
            assert not d.pre_gain.any()
        else:
            _close(d.pre_gain, (dod * v).sum(over), many * (dod * v).abs().sum(over), "dpre")
        t, size = o["scale"] * dx, abs(o["scale"]) * size
        if self.gate is not None:
            each, each_size = t * self.keep * post * u, size * self.keep * (post * u).abs()
            _close(d.gate, each.sum_to_size(self.gate.shape), many * each_size.sum_to_size(self.gate.shape), "dgate")
        else:
            assert d.gate is None
        t, size = t * gate * self.keep, size * abs(gate) * self.keep
        if o["post_norm"]:
            _close(d.post_gain, (t * u).sum(over), many * (size * u.abs()).sum(over), "dpost")
            w, size = t * post, size * abs(post)
            t = ry * (w - u * (w * u).mean(-1, keepdim=True))
            size = ry * (size + u.abs() * (size * u.abs()).mean(-1, keepdim=True))
        else:
            assert d.post_gain is None
        _close(d.y, t, 256 * U * size + _round(self.y.dtype) * t.abs(), "dy")


DIMS = [1, 3, 8, 33, 64, 65, 100, 128, 256, 257, 512, 1000, 1024, 1025, 2048, 2052, 4096, 5000, 8192, 9001, 16384]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_widths(dim, types):
    Case((5, dim), *types, gate=(dim,), p=0.2, scale=0.5).check()
    Case((3, 1, dim), *types, post_norm=False).check()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("shape", [(1, 64), (2, 3, 64), (4, 100, 96), (700, 200), (3, 1001, 72), (40, 31, 256), (2, 700, 1000), (64, 2, 2048)])
def test_gates(shape, types):
    lead = shape[:-1]
    gates = [None, shape[-1:], shape]
    if len(shape) == 3:
        gates += [(lead[0], 1, shape[-1]), (1, 1, shape[-1])]
    for n, gate in enumerate(gates):
        Case(shape, *types, gate=gate, p=(0.0, 0.25)[n % 2], scale=-0.7, gain_dtype=("f32", "bf16")[n // 2 % 2], seed=n).check()


def test_many_rows_of_few_entries_and_a_gate_for_each_of_many_sequences():
    Case((20011, 16), gate=(16,), p=0.1).check()
    Case((4000, 5, 24), "bf16", "bf16", gate=(4000, 1, 24), p=0.1).check()
    Case((3, 4001, 40), gate=(3, 1, 40)).check()
    Case((70000, 2, 8), gate=(70000, 1, 8)).check()
    Case((2, 9, 7, 24), gate=(2, 9, 1, 24)).check()


def test_without_gains_and_with_another_eps():
    Case((6, 300), gains=False).check()
    Case((6, 300), gains=False, eps=0.1).check()
    c = Case((4, 64), eps=0.0)
    c.x[0], c.y[0] = 0.0, 0.0                                            # the norm of nothing, without eps: not a number, in its row alone
    r = c.run()
    assert torch.isnan(r.stream[0]).all() and torch.isfinite(r.stream[1:]).all() and torch.isfinite(r.out[1:]).all()


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_a_norm_alone_and_a_sum_alone(types):
    for shape in ((9, 200), (2, 5, 2048)):
        c = Case(shape, *types)
        dtype = c.y.dtype
        r = asi.residual_norm(c.x, pre_gain=c.pre, dtype=dtype)
        assert r.stream is c.x
        s = c.x.double()
        rs = _rms(s, 1e-6)
        _close(r.out, s * rs * c.pre.double(), (64 * U + _round(dtype)) * (s * rs * c.pre.double()).abs(), "out")
        d = asi.residual_norm_grad(c.ds, c.do, c.x, pre_gain=c.pre)
        assert d.y is None and d.gate is None and d.post_gain is None
        c.check_grad(c.x, c.ds, c.do, c.y.double() * _rms(c.y.double(), 1e-6), _rms(c.y.double(), 1e-6), s, rs, 1.0, c.one(c.post), c.pre.double())
        only = asi.residual_norm(c.x, c.y, c.post, pre_norm=False)
        assert only.out is None and torch.equal(only.stream, asi.residual_norm(c.x, c.y, c.post).stream)
        d = asi.residual_norm_grad(c.ds, None, only.stream, c.y, c.post, pre_norm=False)
        assert d.pre_gain is None and torch.equal(d.x, c.ds)
        both = asi.residual_norm_grad(c.ds, None, only.stream, c.y, c.post)
        assert torch.equal(d.y, both.y) and torch.equal(d.post_gain, both.post_gain)


def test_strides():
    c = Case((4, 6, 96), gate=(4, 1, 96), p=0.2)
    want, grads = c.run(), c.grad(c.x)
    wide = torch.zeros(4, 6, 200, device="cuda")
    wide[..., 3:99], wide[..., 100:196] = c.x, c.y                        # rows apart, at addresses that are no multiple of 16
    x, y = wide[..., 3:99], wide[..., 100:196]
    r = asi.residual_norm(x, y, c.post, c.gate, c.pre, **c.options)
    assert torch.equal(r.stream, want.stream) and torch.equal(r.out, want.out)
    d = asi.residual_norm_grad(c.ds.transpose(0, 1).contiguous().transpose(0, 1), c.do, x, y, c.post, c.gate, c.pre, **c.options)
    assert all(torch.equal(a, b) for a, b in zip(d, grads))
    x = c.x.permute(2, 0, 1).contiguous().permute(1, 2, 0)                # a row's entries apart
    r = asi.residual_norm(x, c.y, c.post, c.gate, c.pre, **c.options)
    assert torch.equal(r.stream, want.stream) and r.stream.is_contiguous()
    x = c.x[:, :1].expand(4, 6, 96)                                       # one row for all
    assert torch.equal(asi.residual_norm(x, c.y).stream, asi.residual_norm(x.contiguous(), c.y).stream)


def test_what_is_dropped_may_hold_anything():
    c = Case((8, 256), post_norm=False, p=0.3, gate=(256,))
    want = c.run()
    c.y[c.keep == 0] = float("nan")
    r = c.run()
    assert torch.equal(r.stream, want.stream) and torch.equal(r.out, want.out)
    d = c.grad(r.stream)
    assert torch.isfinite(d.gate).all() and not d.y[c.keep == 0].any()


@pytest.mark.parametrize("types", TYPES)
def test_autograd(types):
    c = Case((3, 50, 136), *types, gate=(3, 1, 136), p=0.2, scale=0.5)
    leaves = [t.clone().requires_grad_() for t in (c.x, c.y, c.post, c.gate, c.pre)]
    r = asi.residual_norm(*leaves, **c.options)
    torch.autograd.backward((r.stream, r.out), (c.ds, c.do))
    want = c.grad(r.stream.detach())
    for leaf, g in zip(leaves, want):
        assert torch.equal(leaf.grad, g.to(leaf.dtype))
    only = [t.clone().requires_grad_() for t in (c.x, c.y, c.post, c.gate, c.pre)]
    asi.residual_norm(*only, **c.options).stream.backward(c.ds)           # what is behind the norm is not used
    assert torch.equal(only[1].grad, c.grad(r.stream.detach(), do=None).y) and not only[4].grad.any()
    x = c.x.clone().requires_grad_()
    first = asi.residual_norm(x, pre_gain=c.pre, dtype=c.y.dtype)
    assert first.stream is x
    torch.autograd.backward((first.stream, first.out), (c.ds, c.do))
    alone = asi.residual_norm_grad(None, c.do, c.x, pre_gain=c.pre)
    assert torch.equal(x.grad, alone.x + c.ds)
    y = c.y.clone().requires_grad_()
    asi.residual_norm(c.x, y, pre_norm=False).stream.sum().backward()     # a gradient that is one number for all
    assert torch.equal(y.grad, asi.residual_norm_grad(torch.ones_like(c.x), None, c.x, c.y, pre_norm=False).y)


def test_gradients_against_differences():
    c = Case((6, 40), gate=(40,), p=0.2, scale=0.8)
    names = ("x", "y", "post", "gate", "pre")
    r = c.run()
    got = dict(zip(names, c.grad(r.stream)))
    step = 2.0 ** -7
    for name in names:
        start = getattr(c, name).clone()
        g = torch.Generator(device="cuda")
        g.manual_seed(7)
        d = torch.randn(start.shape, generator=g, device="cuda")
        values, curves = [], []
        for k in (1, -1, 2, -2):
            setattr(c, name, start + k * step * d)
            r = c.run()
            values.append(float((r.stream.double() * c.ds.double()).sum() + (r.out.double() * c.do.double()).sum()))
        setattr(c, name, start)
        # by four points: what is left is of the fourth order in the step, taken from the two estimates' difference, which is of the second;
        # the values are off by fewer than 256 U of the magnitudes that are added
        one, two = (values[0] - values[1]) / (2 * step), (values[2] - values[3]) / (4 * step)
        slope = one + (one - two) / 3
        noise = 256 * U * float((r.stream.double() * c.ds.double()).abs().sum() + (r.out.double() * c.do.double()).abs().sum()) / step
        assert abs(slope - float((got[name].double() * d.double()).sum())) <= 2 * noise + abs(one - two), name


def test_another_stream_and_a_graph():
    c = Case((200, 128), "bf16", "bf16", gate=(128,), p=0.1)
    want, grads = c.run(), c.grad(c.x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r, d = c.run(), c.grad(c.x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(r.out, want.out) and all(torch.equal(a, b) for a, b in zip(d, grads))
    seed = torch.zeros(1, dtype=torch.int64, device="cuda")
    c.options["seed"] = seed
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = c.run()
        d = c.grad(r.stream)
    for k in range(4):
        seed.fill_(k)
        c.x.normal_()
        graph.replay()
        eager = c.run()
        torch.cuda.synchronize()
        assert torch.equal(r.stream, eager.stream) and torch.equal(r.out, eager.out)
        assert all(torch.equal(a, b) for a, b in zip(d, c.grad(eager.stream)))


def test_backward_into_a_graph():
    c = Case((30, 64), gate=(64,))
    r = c.run()
    want = asi.residual_norm_grad(None, c.do, r.stream, c.y, c.post, c.gate, c.pre)
    leaves = [t.clone().requires_grad_() for t in (c.x, c.y, c.post, c.gate, c.pre)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(asi.residual_norm(*leaves).out, leaves, c.do)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.skip(reason="torch's engine joins the captured stream with that of the leaves' living eager graph, which ends the capture and the "
                         "process; no operator can see it beforehand")
def test_backward_into_a_graph_while_an_eager_graph_of_the_same_leaves_lives():
    c = Case((30, 64), gate=(64,))
    leaves = [t.clone().requires_grad_() for t in (c.x, c.y, c.post, c.gate, c.pre)]
    lives = asi.residual_norm(*leaves).out.sum()
    want = torch.autograd.grad(asi.residual_norm(*leaves).out.sum(), leaves)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = torch.autograd.grad(asi.residual_norm(*leaves).out.sum(), leaves)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    lives.backward()
    assert torch.equal(leaves[0].grad, want[0])


def test_nothing_to_do_and_refusals():
    c = Case((4, 64), gate=(64,))
    none = asi.residual_norm(c.x[:0], c.y[:0], c.post, c.gate, c.pre)
    assert none.stream.shape == (0, 64) and none.out.shape == (0, 64)
    d = asi.residual_norm_grad(c.ds[:0], c.do[:0], c.x[:0], c.y[:0], c.post, c.gate, c.pre)
    assert d.x.shape == (0, 64) and not d.pre_gain.any() and not d.post_gain.any() and not d.gate.any()
    f, g = asi.residual_norm, asi.residual_norm_grad
    for bad in (lambda: f(c.x, c.y[:2]), lambda: f(c.x, None, c.post), lambda: f(c.x, None, gate=c.gate), lambda: f(c.x, c.y, c.post, post_norm=False),
                lambda: f(c.x, c.y, pre_gain=c.pre, pre_norm=False), lambda: f(c.x, pre_norm=False), lambda: f(c.x, c.y, c.post[:3]),
                lambda: f(c.x, c.y, gate=c.gate[:3]), lambda: f(c.x, c.y, gate=c.x[:2]), lambda: f(c.x, c.y, c.post, c.gate.bfloat16()), lambda: f(c.x, c.y, p=0.1),
                lambda: f(c.x, c.y, p=1.0, seed=1), lambda: f(c.x.cpu(), c.y), lambda: g(None, None, c.x, c.y), lambda: g(c.ds[:2], None, c.x, c.y),
                lambda: g(c.ds, c.do.bfloat16(), c.x, c.y), lambda: g(c.ds, c.do, c.x, c.y, pre_norm=False), lambda: f(c.x[:, :0], c.y[:, :0])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: f(c.x.half(), c.y.half()), lambda: f(c.x, c.y, c.post.half())):
        with pytest.raises(TypeError):
            bad()
    wide = torch.zeros(2, 16385, device="cuda")
    for bad in (lambda: f(c.x.bfloat16(), c.y), lambda: f(wide, wide), lambda: f(c.x, c.y, eps=-1.0), lambda: f(c.x, c.y, scale=float("inf"))):
        with pytest.raises(asi.AsiError):
            bad()
    with forward_ad.dual_level(), pytest.raises(NotImplementedError):
        f(c.x, forward_ad.make_dual(c.y, c.y))
