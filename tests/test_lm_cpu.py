"""Refusals of the language-model operators that need no GPU: bad arguments are answered with a status before
anything is launched, and the Python layer refuses tensors that are not on a GPU."""
import ctypes as C

import pytest
import torch

import paper_2505_05086_amd as asi
from paper_2505_05086_amd import binding as B

P = 0x10000          # non-null, 256-aligned, never dereferenced by validation
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def _lp(**kw):
    d = dict(rows=4, vocab=100, row_stride=100, grad_stride=100, ignore_index=-100, dtype=0, top=0, scale=1.0, reserved=0)
    d.update(kw)
    return B.LogprobDesc(*[d[n] for n, _ in B.LogprobDesc._fields_])


def _forward(desc, logits=P, targets=P, logprob=P, top=(P, P)):
    return B.lib().asi_token_logprobs(desc, logits, targets, logprob, P, P, *top, None, 0, None)


def _backward(desc, logits=P, targets=P, a=P, dlogits=2 * P):
    return B.lib().asi_token_logprobs_grad(desc, logits, targets, a, P, dlogits, P, P, None)


@pytest.mark.parametrize("bad,status", [
    (dict(vocab=0), INVALID), (dict(rows=-1), INVALID), (dict(row_stride=99), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=1e-30), UNSUPPORTED),
    (dict(reserved=1), INVALID), (dict(vocab=1 << 29, row_stride=1 << 29, grad_stride=1 << 29), UNSUPPORTED), (dict(rows=1 << 32), UNSUPPORTED)])
def test_logprob_descriptors(bad, status):
    assert _forward(_lp(**bad)) == status
    assert _backward(_lp(**bad)) == status


def test_logprob_arguments():
    assert _forward(_lp(top=-1)) == INVALID and _forward(_lp(top=65)) == INVALID and _forward(_lp(vocab=10, top=11)) == INVALID
    assert _forward(_lp(), logits=None) == INVALID and _forward(_lp(), targets=None) == INVALID and _forward(_lp(), logits=P + 2) == INVALID
    assert _forward(_lp(top=3), top=(None, P)) == INVALID and _forward(_lp(top=3), top=(P, None)) == INVALID and _forward(_lp(top=3), top=(P, P + 4)) == INVALID
    assert _forward(None) == INVALID and _backward(None) == INVALID
    assert _forward(_lp(rows=0), logits=None) == OK
    assert _backward(_lp(grad_stride=99)) == INVALID
    assert _backward(_lp(row_stride=120), dlogits=P) == INVALID                   # in place with another stride
    assert _backward(_lp(), dlogits=None) == INVALID and _backward(_lp(), targets=None) == INVALID and _backward(_lp(rows=0), logits=None, dlogits=None) == OK


def test_logprob_scratch_of_rows_in_parts():
    few = _lp(rows=5, vocab=200000, row_stride=200000, top=3)
    need = B.lib().asi_token_logprobs_workspace_bytes(few)
    assert need > 0 and need % 256 == 0 and B.lib().asi_token_logprobs_workspace_bytes(_lp()) == 0
    assert B.lib().asi_token_logprobs_workspace_bytes(_lp(rows=5, vocab=200000, row_stride=1)) == 0
    for ws, size in ((None, need), (P, need - 1), (P + 64, need)):
        assert B.lib().asi_token_logprobs(few, P, P, P, P, P, P, P, ws, size, None) == WORKSPACE


def _em(**kw):
    d = dict(tokens=10, vocab=50, dim=8, table_stride=8, out_stride=8, padding_index=-1, table_dtype=0, out_dtype=0, scale=1.0, reserved=0)
    d.update(kw)
    return B.EmbeddingDesc(*[d[n] for n, _ in B.EmbeddingDesc._fields_])


@pytest.mark.parametrize("bad,status", [
    (dict(tokens=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(table_stride=7), INVALID), (dict(out_stride=7), INVALID),
    (dict(table_dtype=3), UNSUPPORTED), (dict(out_dtype=-1), UNSUPPORTED), (dict(scale=float("inf")), INVALID), (dict(reserved=2), INVALID),
    (dict(tokens=1 << 30), UNSUPPORTED), (dict(vocab=1 << 30), UNSUPPORTED), (dict(dim=1 << 25, table_stride=1 << 25, out_stride=1 << 25), UNSUPPORTED)])
def test_embedding_descriptors(bad, status):
    L = B.lib()
    assert L.asi_embedding(_em(**bad), P, P, P, None) == status
    assert L.asi_embedding_grad_workspace_bytes(_em(**bad)) == 0
    assert L.asi_embedding_grad(_em(**bad), P, P, P, 0, P, 1 << 30, None) == status


def test_embedding_arguments():
    L = B.lib()
    for args in ((None, P, P), (P, None, P), (P, P, None), (P + 4, P, P), (P, P + 2, P), (P, P, P + 1)):
        assert L.asi_embedding(_em(), *args, None) == INVALID
    assert L.asi_embedding(None, P, P, P, None) == INVALID
    assert L.asi_embedding(_em(tokens=0), None, None, None, None) == OK
    many = _em(tokens=2000)                                       # few tokens need no scratch
    need = L.asi_embedding_grad_workspace_bytes(many)
    assert need > 0 and need % 256 == 0 and L.asi_embedding_grad_workspace_bytes(_em()) == 0
    for ws, size in ((None, need), (P, need - 1), (P + 128, need)):
        assert L.asi_embedding_grad(many, P, P, P, 0, ws, size, None) == WORKSPACE
    for args in ((None, P, P), (P, None, P), (P, P, None), (P, P + 2, P)):
        assert L.asi_embedding_grad(_em(), *args, 0, P, need, None) == INVALID
        assert L.asi_embedding_grad(many, *args, 0, P, need, None) == INVALID
    assert L.asi_embedding_grad(_em(tokens=0), None, None, P, 1, None, 0, None) == OK


def _qk(**kw):
    d = B.QkDesc()
    v = dict(batch=2, tokens=3, max_position=100, position_stride=3, q_heads=4, k_heads=2, head_dim=64, rot_dim=64, interleaved=0, dtype=0,
             gain_dtype=0, eps=1e-6)
    v.update(kw)
    for name, value in v.items():
        setattr(d, name, value)
    for f in ("q_stride", "q_out_stride", "dq_stride"):
        getattr(d, f)[:] = (768, 256, 64)
    for f in ("k_stride", "k_out_stride", "dk_stride"):
        getattr(d, f)[:] = (384, 128, 64)
    return d


def _rotate(d, q=P, k=P, gain=P, pos=P, cos=P, sin=P, out=P):
    return B.lib().asi_qk_norm_rotate(d, q, k, gain, gain, pos, cos, sin, out, out, None)


def _rotate_grad(d, q=P, dy=P, dx=P, dg=P, ws=P, size=None, cos=P):
    need = B.lib().asi_qk_norm_rotate_grad_workspace_bytes(d) if d is not None else 0
    return B.lib().asi_qk_norm_rotate_grad(d, q, P, P, P, P, cos, P, dy, dy, dx, dx, dg, dg, ws, need if size is None else size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(batch=-1), INVALID), (dict(tokens=-1), INVALID), (dict(q_heads=-1), INVALID), (dict(head_dim=0), INVALID), (dict(rot_dim=3), INVALID),
    (dict(rot_dim=66), INVALID), (dict(rot_dim=-2), INVALID), (dict(interleaved=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(max_position=-1), INVALID), (dict(position_stride=-1), INVALID), (dict(dtype=7), UNSUPPORTED), (dict(gain_dtype=7), UNSUPPORTED),
    (dict(head_dim=1025), UNSUPPORTED), (dict(batch=1 << 20, tokens=1 << 20), UNSUPPORTED), (dict(k_heads=1 << 17), UNSUPPORTED)])
def test_qk_descriptors(bad, status):
    assert _rotate(_qk(**bad)) == status
    assert B.lib().asi_qk_norm_rotate_grad_workspace_bytes(_qk(**bad)) == 0
    assert _rotate_grad(_qk(**bad)) == status


def test_qk_arguments():
    for bad in (dict(q=None), dict(k=None), dict(out=None), dict(cos=None), dict(sin=None), dict(q=P + 2), dict(gain=P + 2), dict(pos=P + 4), dict(cos=P + 2)):
        assert _rotate(_qk(), **bad) == INVALID, bad
    assert _rotate(None) == INVALID and _rotate_grad(None) == INVALID
    for empty in (dict(batch=0), dict(tokens=0), dict(q_heads=0, k_heads=0)):
        assert _rotate(_qk(**empty), q=None, k=None, out=None) == OK
    for bad in (dict(q=None), dict(dy=None), dict(dx=None), dict(dg=P + 2), dict(cos=None)):
        assert _rotate_grad(_qk(), **bad) == INVALID, bad
    need = B.lib().asi_qk_norm_rotate_grad_workspace_bytes(_qk())
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=P + 64), dict(size=need - 1)):
        assert _rotate_grad(_qk(), **bad) == WORKSPACE, bad


def _adamw(tensors, bits=32, b1=0.9, b2=0.999, eps=1e-8, step=1, gs=None, skip=None):
    arr = (B.AdamwTensor * max(1, len(tensors)))(*tensors)
    return B.lib().asi_adamw(len(tensors), C.addressof(arr), bits, b1, b2, eps, step, gs, skip, None)


def _tensor(**kw):
    d = dict(param=P, grad=P, master=None, exp_avg=P, exp_avg_sq=P, exp_avg_scale=None, exp_avg_sq_scale=None, count=10, param_dtype=0, grad_dtype=0,
             lr=1e-3, weight_decay=0.1)
    d.update(kw)
    return B.AdamwTensor(*[d[n] for n, _ in B.AdamwTensor._fields_])


def test_adamw_arguments():
    assert _adamw([]) == OK and _adamw([_tensor(count=0, param=None, grad=None, exp_avg=None, exp_avg_sq=None)]) == OK
    for bad in (dict(param=None), dict(grad=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(count=-1), dict(count=(1 << 40) + 1), dict(param_dtype=2), dict(grad_dtype=5),
                dict(param=P + 2), dict(exp_avg=P + 1), dict(lr=float("nan")), dict(weight_decay=float("inf")), dict(master=P + 2)):
        assert _adamw([_tensor(), _tensor(**bad)]) == INVALID, bad
    assert _adamw([_tensor(exp_avg_scale=P)], bits=8) == INVALID                 # scales are needed for 8 bits
    for bad, status in ((dict(bits=16), UNSUPPORTED), (dict(b1=1.0), INVALID), (dict(b2=-0.1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("inf")), INVALID),
                        (dict(step=0), INVALID), (dict(gs=P + 2), INVALID), (dict(skip=P + 1), INVALID)):
        assert _adamw([_tensor()], **bad) == status, bad
    assert B.lib().asi_adamw(1, None, 32, 0.9, 0.99, 1e-8, 1, None, None, None) == INVALID
    assert B.lib().asi_adamw(-1, None, 32, 0.9, 0.99, 1e-8, 1, None, None, None) == INVALID


def test_optimiser_refusals():
    p = torch.nn.Parameter(torch.zeros(3))
    with pytest.raises(ValueError):
        asi.AdamW([p], state_bits=16)
    with pytest.raises(ValueError):
        asi.AdamW([p], betas=(1.0, 0.9))
    with pytest.raises(ValueError):
        asi.AdamW([p]).step(grads=[])


@pytest.mark.parametrize("call", [
    lambda: asi.token_logprobs(torch.zeros(3, 4, dtype=torch.float16)),
    lambda: asi.token_logprobs(torch.zeros(3, 4), torch.zeros(3, dtype=torch.int32)),
    lambda: asi.embedding(torch.zeros(3, dtype=torch.int32), torch.zeros(4, 4)),
    lambda: asi.qk_norm_rotate(torch.zeros(1, 1, 1, 4), torch.zeros(1, 1, 1, 4), None, None, torch.zeros(5, 2), torch.zeros(5, 2), torch.zeros(1, 1)),
])
def test_types_are_refused(call):
    with pytest.raises((TypeError, ValueError, RuntimeError)):
        call()


@pytest.mark.parametrize("call", [
    lambda: asi.token_logprobs(torch.zeros(3, 4), torch.zeros(4, dtype=torch.int64)),
    lambda: asi.token_logprobs(torch.zeros(4, 3).t()),
    lambda: asi.token_logprobs(torch.zeros(2, 5, 4)[:, :-1]),
    lambda: asi.token_logprobs_grad(torch.zeros(3, 4), None, torch.zeros(4)),
    lambda: asi.token_logprobs_grad(torch.zeros(3, 4), None, torch.zeros(3, dtype=torch.bfloat16)),
    lambda: asi.embedding(torch.zeros(3, dtype=torch.int64), torch.zeros(4)),
    lambda: asi.embedding_grad(torch.zeros(3, dtype=torch.int64), torch.zeros(4, 4), 9),
    lambda: asi.embedding_grad(torch.zeros(3, dtype=torch.int64), torch.zeros(3, 4), 9, accumulate=True),
    lambda: asi.embedding_grad(torch.zeros(3, dtype=torch.int64), torch.zeros(3, 4), 9, out=torch.zeros(8, 4)),
    lambda: asi.qk_norm_rotate(torch.zeros(1, 2, 1, 4), torch.zeros(1, 1, 1, 4), None, None, torch.zeros(5, 2), torch.zeros(5, 2)),
    lambda: asi.qk_norm_rotate(torch.zeros(1, 2, 1, 4), torch.zeros(1, 2, 1, 4), torch.zeros(3), None, torch.zeros(5, 2), torch.zeros(5, 2)),
    lambda: asi.qk_norm_rotate(torch.zeros(1, 2, 1, 4), torch.zeros(1, 2, 1, 4), None, None, torch.zeros(5, 2), torch.zeros(4, 2)),
])
def test_shapes_are_refused(call):
    with pytest.raises(ValueError):
        call()
