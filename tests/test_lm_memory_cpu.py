"""Refusals of the operators that keep no logits, no mask and no copy of a norm's input, without a GPU: bad arguments are answered with
a status before anything is launched."""
import pytest
import torch

import paper_2505_05086_amd as asi
from paper_2505_05086_amd import binding as B

P = 0x10000          # non-null, 256-aligned, never dereferenced by validation
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
MANY = 1 << 50


def _of(cls, values, changed):
    values.update(changed)
    return cls(*[values[n] for n, _ in cls._fields_])


def _head(**kw):
    return _of(B.LinearLogprobDesc, dict(rows=40, dim=64, vocab=100, hidden_stride=64, weight_stride=64, ignore_index=-100, dtype=1, scale=1.0,
                                         any_address=0, reserved=0), kw)


def _values(d, h=P, w=P, t=P, logprob=P, entropy=P, stats=P, ws=P, size=MANY):
    return B.lib().asi_linear_logprobs(d, h, w, t, logprob, entropy, stats, ws, size, None)


def _grad(d, given=0, h=P, w=P, t=P, stats=P, logprob=P, entropy=P, a=P, b=P, dh=P, dw=P, ws=P, size=MANY):
    return B.lib().asi_linear_logprobs_grad(d, given, h, w, t, stats, logprob, entropy, a, b, dh, dw, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(vocab=0), INVALID), (dict(hidden_stride=63), INVALID), (dict(weight_stride=63), INVALID),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=1e-30), UNSUPPORTED), (dict(scale=1e30), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED), (dict(any_address=2), INVALID), (dict(reserved=1), INVALID), (dict(rows=1 << 24), UNSUPPORTED),
    (dict(dim=1 << 18, hidden_stride=1 << 18, weight_stride=1 << 18), UNSUPPORTED), (dict(vocab=1 << 28), UNSUPPORTED), (dict(rows=1 << 20, vocab=1 << 20), UNSUPPORTED),
    (dict(rows=(1 << 24) - 1, dim=(1 << 18) - 1, hidden_stride=1 << 18, weight_stride=1 << 18), UNSUPPORTED)])
def test_head_descriptors(bad, status):
    d = _head(**bad)
    assert _values(d) == status and _grad(d) == status
    assert B.lib().asi_linear_logprobs_workspace_bytes(d) == 0 and B.lib().asi_linear_logprobs_grad_workspace_bytes(d) == 0


def test_head_arguments():
    assert _values(None) == INVALID and _grad(None) == INVALID
    d = _head()
    for kw in (dict(h=None), dict(w=None), dict(t=None), dict(h=P + 1), dict(w=P + 8), dict(t=P + 4), dict(logprob=P + 2), dict(entropy=P + 1), dict(stats=P + 3)):
        assert _values(d, **kw) == INVALID, kw
        assert _grad(d, **kw) == INVALID or "stats" in kw and kw["stats"] is None, kw
    for kw in (dict(given=2), dict(given=1, stats=None), dict(given=1, entropy=None), dict(dh=P + 1), dict(dw=P + 1), dict(a=P + 2), dict(b=P + 1), dict(t=None, logprob=None)):
        assert _grad(d, **kw) == INVALID, kw
    for size, f in ((B.lib().asi_linear_logprobs_workspace_bytes(d), _values), (B.lib().asi_linear_logprobs_grad_workspace_bytes(d), _grad)):
        assert size > 0 and size % 256 == 0
        for kw in (dict(ws=None), dict(ws=P + 64), dict(size=size - 1)):
            assert f(d, **kw) == WORKSPACE, kw
    assert _values(_head(rows=0), h=None, w=None, t=None) == OK and _grad(_head(rows=0), h=None, w=None, dw=None) == OK


def test_head_scratch_holds_no_more_than_a_piece_of_the_logits():
    need = B.lib().asi_linear_logprobs_grad_workspace_bytes
    small, large = (need(_head(rows=4096, dim=1024, vocab=v, hidden_stride=1024, weight_stride=1024)) for v in (20000, 200000))
    assert large - small < 4096 * 180000 * 2 / 8                          # the values of the tiles alone grow
    assert need(_head(any_address=1)) > need(_head())


def _drop(**kw):
    return _of(B.DropoutDesc, dict(rows=4, dim=10, x_stride=10, y_stride=10, seed=1, offset=2, p=0.1, dtype=0, reserved=0), kw)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(x_stride=9), INVALID), (dict(y_stride=9), INVALID), (dict(p=-0.1), INVALID), (dict(p=1.0), INVALID),
    (dict(p=0.999999), INVALID), (dict(p=float("nan")), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(reserved=1), INVALID),
    (dict(dim=1 << 31, x_stride=(1 << 31) + 1, y_stride=1 << 31), UNSUPPORTED), (dict(rows=1 << 30, dim=1 << 30, x_stride=1 << 30, y_stride=1 << 30), UNSUPPORTED)])
def test_dropout_descriptors(bad, status):
    assert B.lib().asi_dropout(_drop(**bad), P, None, 2 * P, None) == status


def test_dropout_arguments():
    f = B.lib().asi_dropout
    assert f(None, P, None, P, None) == INVALID and f(_drop(), None, None, P, None) == INVALID and f(_drop(), P, None, None, None) == INVALID
    assert f(_drop(), P + 2, None, P, None) == INVALID and f(_drop(), P, None, P + 2, None) == INVALID and f(_drop(), P, P + 4, P, None) == INVALID
    assert f(_drop(x_stride=12), P, None, P, None) == INVALID              # in place with another stride
    assert f(_drop(rows=0), None, None, None, None) == OK


def _edge(**kw):
    return _of(B.ResidualDesc, dict(rows=12, dim=64, x_stride=64, y_stride=64, gate_rows=3, seed=1, offset=0, p=0.1, stream_dtype=0, dtype=0, gain_dtype=0,
                                    post_norm=1, scale=1.0, eps=1e-6), kw)


def _forward(d, x=P, y=P, post=P, gate=P, pre=P, seed=None, s=2 * P, out=P):
    return B.lib().asi_residual_norm(d, x, y, post, gate, pre, seed, s, out, None)


def _backward(d, ds=P, do=P, s=P, y=P, post=P, gate=P, pre=P, seed=None, dx=P, dy=P, dpost=P, dgate=P, dpre=P, ws=P, size=MANY):
    return B.lib().asi_residual_norm_grad(d, ds, do, s, y, post, gate, pre, seed, dx, dy, dpost, dgate, dpre, ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(x_stride=63), INVALID), (dict(y_stride=63), INVALID), (dict(gate_rows=-1), INVALID), (dict(gate_rows=5), INVALID),
    (dict(gate_rows=24), INVALID), (dict(post_norm=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(p=1.0), INVALID), (dict(p=-1.0), INVALID), (dict(stream_dtype=2), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(gain_dtype=2), UNSUPPORTED), (dict(stream_dtype=1), UNSUPPORTED), (dict(dim=16385, x_stride=16385, y_stride=16385), UNSUPPORTED), (dict(rows=3 << 40), UNSUPPORTED)])
def test_residual_descriptors(bad, status):
    d = _edge(**bad)
    assert _forward(d) == status and _backward(d) == status and B.lib().asi_residual_norm_grad_workspace_bytes(d) == 0


def test_residual_arguments():
    assert _forward(None) == INVALID and _backward(None) == INVALID
    d = _edge()
    for kw in (dict(x=None), dict(y=None), dict(s=None), dict(gate=None), dict(x=P + 2), dict(y=P + 1), dict(post=P + 2), dict(gate=P + 1), dict(pre=P + 3), dict(seed=P + 4),
               dict(s=P + 2), dict(out=P + 1)):
        assert _forward(d, **kw) == INVALID, kw
    assert _forward(_edge(post_norm=0)) == INVALID and _forward(_edge(gate_rows=0)) == INVALID
    assert _forward(_edge(gate_rows=0), y=None, post=None, gate=None, s=None, out=None) == INVALID
    assert _forward(_edge(x_stride=80), s=P) == INVALID                    # in place with another stride
    for kw in (dict(ds=None, do=None), dict(s=None), dict(y=None), dict(dy=None), dict(gate=None), dict(ds=P + 2), dict(do=P + 1), dict(dx=P + 2), dict(dy=P + 2),
               dict(dpost=P + 2), dict(dgate=P + 1), dict(dpre=P + 3)):
        assert _backward(d, **kw) == INVALID, kw
    size = B.lib().asi_residual_norm_grad_workspace_bytes(d)
    assert size > 0 and size % 256 == 0
    for kw in (dict(ws=None), dict(ws=P + 64), dict(size=size - 1)):
        assert _backward(d, **kw) == WORKSPACE, kw
    none = _edge(rows=0, gate_rows=0)
    assert _forward(none, x=None, y=None) == OK


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x = torch.zeros(4, 64)
    for bad in (lambda: asi.dropout(x, 0.1, 1), lambda: asi.residual_norm(x, x), lambda: asi.linear_logprobs(x, x)):
        with pytest.raises(ValueError):
            bad()


def test_the_version_tells_libraries_with_these_entry_points_apart():
    assert B.asi_version() >= 1004
