"""The operators of a language model's fine-tuning step that stand beside the compressed layers: token log
probabilities and their gradient (from logits, or from hidden states without any), embedding, norms of queries and keys with the
position rotation, dropout without a stored mask, the edge between two blocks, AdamW.

Thin layer over the C ABI of include/asi_lm.h: it checks and marshals arguments, allocates results and scratch from
torch's allocator on the current stream, and wires the calls into autograd where an input requires a gradient.  All
arithmetic runs in the HIP kernels; there is no CPU fallback.

Calls and their gradient functions can be captured into a graph.  A backward pass by torch's engine can be, with leaves that no living eager
graph holds: the engine would join the captured stream with theirs, which ends the process.
"""
from __future__ import annotations

import functools
import itertools
import operator
from typing import List, NamedTuple, Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding as B

_DTYPE = {torch.float32: B.ASI_F32, torch.bfloat16: B.ASI_BF16}
IGNORE_INDEX = -100


# ---- argument checks --------------------------------------------------------------------------------------
# Small calls last as long as their marshalling: what follows from shapes, strides and types alone (the checks, the descriptor, the
# scratch) is worked out once for each of them and kept by those, never by a tensor or its address: numbers are made plain ones first.
_plans = functools.lru_cache(maxsize=1024)


def _dtype(dtype: torch.dtype, what: str) -> int:
    d = _DTYPE.get(dtype)
    if d is None:
        raise TypeError(f"{what} is fp32 or bf16, not {dtype}")
    return d


def _place(first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """The current GPU's index; every tensor has to be there, without a tangent of forward-mode differentiation."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in (first, *others)):
        raise NotImplementedError("forward-mode derivatives are not implemented")
    device = first.get_device()
    for t in others:
        if t is not None and t.get_device() != device:
            device = -1
    if device < 0 or device != torch._C._cuda_getDevice():
        raise ValueError("every tensor has to be on the current GPU (there is no CPU fallback)")
    return device


def _geometry(t: Optional[torch.Tensor]):
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _dense(shape, stride) -> bool:
    n = 1
    for s, d in zip(reversed(shape), reversed(stride)):
        if s != 1 and d != n and 0 not in shape:
            return False
        n *= s
    return True


def _whole(t: torch.Tensor, what: str) -> torch.Tensor:
    if t.dtype != torch.int64:
        raise TypeError(f"{what} are int64, not {t.dtype}")
    return t if t.is_contiguous() else t.contiguous()


def _weights(t: Optional[torch.Tensor], shape, what: str) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape:
        raise ValueError(f"{what} is an fp32 tensor of shape {tuple(shape)}")
    return t if t.is_contiguous() else t.contiguous()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _scratch(nbytes: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None


def _written(t: torch.Tensor) -> torch.Tensor:
    """A caller's tensor that a kernel has written: a backward pass that saved it before has to know."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)
    return t


# ---- token log probabilities ------------------------------------------------------------------------------
class TokenLogprobs(NamedTuple):
    logprob: Optional[torch.Tensor]        # fp32, of each row's target; None without targets
    entropy: torch.Tensor                  # fp32
    top_logprob: Optional[torch.Tensor]    # fp32 (..., top), descending; not differentiable
    top_index: Optional[torch.Tensor]      # int64 (..., top)


class TokenLogprobsGrad(NamedTuple):
    logprob: torch.Tensor
    entropy: torch.Tensor
    grad: torch.Tensor                     # of the logits, in their type


def _row_layout(shape, stride, what: str):
    """Rows, vocabulary and the rows' distance of logits of any number of dimensions."""
    if not shape:
        raise ValueError(f"{what} have a dimension of the vocabulary")
    vocab, rows, apart = shape[-1], 1, None
    if 0 in shape[:-1]:
        return 0, vocab, vocab
    if vocab < 1 or (stride[-1] != 1 and vocab > 1):
        raise ValueError(f"the vocabulary is the innermost dimension of {what}, its entries next to each other")
    for n, d in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if n != 1:
            if apart is None:
                apart = d
            elif d != apart * rows:
                raise ValueError(f"{what} of more than two dimensions need rows at equal distances; shift the targets rather than "
                                 "slicing the logits")
        rows *= n
    return rows, vocab, vocab if apart is None else apart


@_plans
def _logprob_plan(geometry, top, scale, ignore_index, out):
    """Descriptor, scratch, shape of the rows, and for the gradient the shape and strides of a new result."""
    shape, stride, dtype = geometry
    rows, vocab, apart = _row_layout(shape, stride, "logits")
    lead = shape[:-1]
    new = None
    if out is None:
        # rows that lie in their 16 bytes as those of the logits do, so that both are accessed in whole vectors
        grad = vocab + (apart - vocab) % (16 // dtype.itemsize)
        if grad != vocab:
            strides, d = [], grad
            for n in reversed(lead):
                strides.insert(0, d)
                d *= n
            new = (shape, (*strides, 1))
    else:
        if out[0] != shape or out[2] != dtype:
            raise ValueError("out has the logits' shape and type")
        grad = _row_layout(out[0], out[1], "out")[2]
    desc = B.LogprobDesc(rows, vocab, apart, grad, ignore_index, _dtype(dtype, "logits"), top, scale, 0)
    return desc, int(B.lib().asi_token_logprobs_workspace_bytes(desc)), lead, new


def _targets(targets: Optional[torch.Tensor], shape) -> Optional[torch.Tensor]:
    if targets is None:
        return None
    if targets.shape != shape:
        raise ValueError(f"one target for each row: shape {tuple(shape)}, not {tuple(targets.shape)}")
    return _whole(targets, "targets")


def _token_logprobs(logits, targets, top, scale, ignore_index) -> TokenLogprobs:
    desc, nbytes, shape, _ = _logprob_plan(_geometry(logits), top, scale, ignore_index, None)
    targets = _targets(targets, shape)
    device = _place(logits, targets)
    logprob = None if targets is None else logits.new_empty(shape, dtype=torch.float32)
    entropy = logits.new_empty(shape, dtype=torch.float32)
    top_logprob = top_index = None
    if top:
        top_logprob = logits.new_empty(shape + (top,), dtype=torch.float32)
        top_index = logits.new_empty(shape + (top,), dtype=torch.int64)
    ws = _scratch(nbytes, logits)
    status = B.lib().asi_token_logprobs(desc, logits.data_ptr(), _ptr(targets), _ptr(logprob), entropy.data_ptr(), None,
                                        _ptr(top_logprob), _ptr(top_index), _ptr(ws), nbytes, _stream(device))
    if status:
        B._check(status, "asi_token_logprobs")
    return TokenLogprobs(logprob, entropy, top_logprob, top_index)


class _TokenLogprobsFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, top, scale, ignore_index):
        r = _token_logprobs(logits, targets, top, scale, ignore_index)
        ctx.save_for_backward(logits, targets)
        ctx.scale, ctx.ignore_index = scale, ignore_index
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*[t for t in (r.top_logprob, r.top_index) if t is not None])
        return tuple(r)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_logprob, grad_entropy, *_):
        logits, targets = ctx.saved_tensors
        if grad_logprob is None and grad_entropy is None:
            return None, None, None, None, None
        r = token_logprobs_grad(logits, targets, grad_logprob, grad_entropy, scale=ctx.scale, ignore_index=ctx.ignore_index)
        return r.grad, None, None, None, None


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, *, top: int = 0, scale: float = 1.0,
                   ignore_index: int = IGNORE_INDEX) -> TokenLogprobs:
    """Log probabilities of `targets` under softmax(scale * logits), the entropy of each row and its `top` alternatives
    (equal logits by ascending index).  logits (..., vocab) fp32 or bf16, targets (...) int64; logprob and entropy are
    differentiable in the logits."""
    top, scale, ignore_index = operator.index(top), float(scale), operator.index(ignore_index)
    if torch.is_grad_enabled() and logits.requires_grad:
        return TokenLogprobs(*_TokenLogprobsFn.apply(logits, targets, top, scale, ignore_index))
    return _token_logprobs(logits, targets, top, scale, ignore_index)


def token_logprobs_grad(logits: torch.Tensor, targets: Optional[torch.Tensor], grad_logprob: Optional[torch.Tensor],
                        grad_entropy: Optional[torch.Tensor] = None, *, scale: float = 1.0, ignore_index: int = IGNORE_INDEX,
                        out: Optional[torch.Tensor] = None) -> TokenLogprobsGrad:
    """Gradient of sum(grad_logprob * logprob + grad_entropy * entropy) in the logits, with both values, in one pass over
    the logits.  For a loss whose weights are known beforehand this replaces forward and backward.  `out` may be `logits`
    themselves: the gradient then takes their place."""
    desc, _, shape, new = _logprob_plan(_geometry(logits), 0, float(scale), operator.index(ignore_index), _geometry(out))
    targets = _targets(targets, shape)
    grad_logprob, grad_entropy = _weights(grad_logprob, shape, "grad_logprob"), _weights(grad_entropy, shape, "grad_entropy")
    device = _place(logits, targets, grad_logprob, grad_entropy, out)
    given = out is not None
    if not given:
        out = logits.new_empty(logits.shape) if new is None else logits.new_empty_strided(*new)
    logprob = None if targets is None else logits.new_empty(shape, dtype=torch.float32)
    entropy = logits.new_empty(shape, dtype=torch.float32)
    status = B.lib().asi_token_logprobs_grad(desc, logits.data_ptr(), _ptr(targets), _ptr(grad_logprob), _ptr(grad_entropy),
                                             out.data_ptr(), _ptr(logprob), entropy.data_ptr(), _stream(device))
    if status:
        B._check(status, "asi_token_logprobs_grad")
    return TokenLogprobsGrad(logprob, entropy, _written(out) if given else out)


# ---- embedding --------------------------------------------------------------------------------------------
def _matrix(geometry, what: str) -> int:
    """The distance of a matrix's rows."""
    shape, stride, _ = geometry
    if len(shape) != 2 or shape[1] < 1 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{what} is a matrix whose rows' entries are next to each other")
    return stride[0] if shape[0] > 1 else shape[1]


@_plans
def _embedding_plan(shape, table, scale, dtype):
    vocab, dim = table[0][0], table[0][-1]
    desc = B.EmbeddingDesc(shape.numel(), vocab, dim, _matrix(table, "table"), dim, -1, _dtype(table[2], "table"),
                           _dtype(dtype, "the result"), scale, 0)
    return desc, shape + (dim,)


def _embedding(tokens, table, scale, dtype) -> torch.Tensor:
    tokens = _whole(tokens, "tokens")
    dtype = dtype or table.dtype
    desc, shape = _embedding_plan(tokens.shape, _geometry(table), scale, dtype)
    device = _place(tokens, table)
    out = table.new_empty(shape, dtype=dtype)
    status = B.lib().asi_embedding(desc, tokens.data_ptr(), table.data_ptr(), out.data_ptr(), _stream(device))
    if status:
        B._check(status, "asi_embedding")
    return out


class _EmbeddingFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale, padding_idx, dtype):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.scale, ctx.padding_idx, ctx.dtype = table.shape[0], scale, padding_idx, table.dtype
        return _embedding(tokens, table, scale, dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        tokens, = ctx.saved_tensors
        return None, embedding_grad(tokens, grad_out, ctx.vocab, scale=ctx.scale, padding_idx=ctx.padding_idx, dtype=ctx.dtype), \
            None, None, None


def embedding(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, padding_idx: Optional[int] = None,
              dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * table[tokens] in `dtype` (the table's own by default), differentiable in the table.  The row of `padding_idx`
    gets no gradient; a token outside the table gives a row of NaN and no gradient."""
    scale, padding_idx = float(scale), None if padding_idx is None else operator.index(padding_idx)
    if torch.is_grad_enabled() and table.requires_grad:
        return _EmbeddingFn.apply(tokens, table, scale, padding_idx, dtype)
    return _embedding(tokens, table, scale, dtype)


def embedding_grad(tokens: torch.Tensor, grad_out: torch.Tensor, vocab: int, *, scale: float = 1.0,
                   padding_idx: Optional[int] = None, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                   accumulate: bool = False) -> torch.Tensor:
    """Gradient of the table of embedding(): (vocab, dim) in `dtype`, or written to `out`; with `accumulate` added to it,
    which leaves rows without a token alone.  Sums are in fp32 and in the order of the tokens: equal calls, equal bits."""
    scale, vocab, padding_idx = float(scale), operator.index(vocab), None if padding_idx is None else operator.index(padding_idx)
    tokens = _whole(tokens, "tokens")
    if grad_out.dim() != 2:
        if grad_out.dim() < 1 or grad_out.shape[:-1] != tokens.shape:
            raise ValueError("grad_out has the tokens' shape and one more dimension")
        grad_out = grad_out.reshape(tokens.numel(), grad_out.shape[-1])
    if accumulate and out is None:
        raise ValueError("accumulate adds to `out`")
    desc, nbytes, dense, shape = _embedding_grad_plan(tokens.shape, _geometry(grad_out), vocab, scale, padding_idx, dtype, _geometry(out))
    if not dense:
        grad_out = grad_out.contiguous()
    device = _place(tokens, grad_out, out)
    given = out is not None
    if not given:
        out = grad_out.new_empty(shape, dtype=dtype)
    ws = _scratch(nbytes, grad_out)
    status = B.lib().asi_embedding_grad(desc, tokens.data_ptr(), grad_out.data_ptr(), out.data_ptr(), int(accumulate), _ptr(ws), nbytes,
                                        _stream(device))
    if status:
        B._check(status, "asi_embedding_grad")
    return _written(out) if given else out


@_plans
def _embedding_grad_plan(tokens, grad_out, vocab, scale, padding_idx, dtype, out):
    """Descriptor, scratch, whether grad_out can be taken as it lies, shape of a new result."""
    n = tokens.numel()
    shape, stride, grad_dtype = grad_out
    if shape[0] != n:
        raise ValueError("grad_out has the tokens' shape and one more dimension")
    dim = shape[1]
    taken = (stride[1] == 1 or dim == 1) and (n <= 1 or stride[0] >= dim)
    if out is not None:
        if out[0] != (vocab, dim):
            raise ValueError(f"out is ({vocab}, {dim})")
        dtype, apart = out[2], _matrix(out, "out")
    else:
        apart = dim
    if padding_idx is not None and not 0 <= padding_idx < vocab:
        raise ValueError("padding_idx is a token of the table")
    desc = B.EmbeddingDesc(n, vocab, dim, apart, stride[0] if taken and n > 1 else dim, -1 if padding_idx is None else padding_idx,
                           _dtype(dtype, "the gradient"), _dtype(grad_dtype, "grad_out"), scale, 0)
    return desc, int(B.lib().asi_embedding_grad_workspace_bytes(desc)), taken, (vocab, dim)


# ---- norms of queries and keys with the position rotation -----------------------------------------------------
def rotary_table(length: int, rot_dim: int, base: float = 10000.0, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """cos and sin of position * base^(-2 e / rot_dim), fp32 (length, rot_dim / 2), computed in fp64."""
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    angle = torch.arange(length, dtype=torch.float64, device=device)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def _head_shape(shape, heads_first: bool):
    b, t, h, d = shape
    return (b, h, t, d) if heads_first else (b, t, h, d)


def _strides(geometry, heads_first: bool, what: str):
    """(batch, token, head) distances of a tensor of heads."""
    shape, stride, _ = geometry
    if len(shape) != 4 or (stride[3] != 1 and shape[3] > 1):
        raise ValueError(f"{what} has four dimensions, a head's entries next to each other")
    return (stride[0], stride[2], stride[1]) if heads_first else stride[:3]


def _qk_desc(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved) -> B.QkDesc:
    """The descriptor of these geometries, the results' strides not yet in it."""
    desc = B.QkDesc()
    desc.q_stride[:], desc.k_stride[:] = _strides(q, False, "q"), _strides(k, False, "k")
    batch, tokens, heads, dim = q[0]
    if k[0][0] != batch or k[0][1] != tokens or k[0][3] != dim or k[2] != q[2]:
        raise ValueError("q and k have the same batch, tokens, head_dim and type")
    gains = [g for g in (q_gain, k_gain) if g is not None]
    if any(g[0] != (dim,) or not _dense(*g[:2]) or g[2] != gains[0][2] for g in gains):
        raise ValueError("the gains are contiguous tensors of head_dim entries, both of one type")
    if len(cos[0]) != 2 or cos[0] != sin[0] or any(c[2] != torch.float32 or not _dense(*c[:2]) for c in (cos, sin)):
        raise ValueError("cos and sin are contiguous fp32 tables (positions, rot_dim / 2)")
    if positions is not None:
        shape, stride, dtype = positions
        if dtype != torch.int64:
            raise TypeError("positions are int64")
        if shape not in ((tokens,), (batch, tokens)) or (tokens > 1 and stride[-1] != 1):
            raise ValueError("positions are (tokens) or (batch, tokens), those of a batch entry next to each other")
        desc.position_stride = stride[0] if len(shape) == 2 and batch > 1 else 0
    desc.batch, desc.tokens, desc.max_position = batch, tokens, cos[0][0]
    desc.q_heads, desc.k_heads, desc.head_dim, desc.rot_dim = heads, k[0][2], dim, 2 * cos[0][1]
    desc.interleaved, desc.dtype, desc.eps = bool(interleaved), _dtype(q[2], "q"), eps
    desc.gain_dtype = _dtype(gains[0][2], "a gain") if gains else B.ASI_F32
    return desc


def _lying(shape):
    """Strides of a new tensor of heads."""
    _, b, c, d = shape
    return b * c * d, c * d, d, 1


@_plans
def _qk_plan(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first):
    desc = _qk_desc(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    shapes = [_head_shape(x[0], heads_first) for x in (q, k)]
    desc.q_out_stride[:], desc.k_out_stride[:] = (_strides((s, _lying(s), None), heads_first, "") for s in shapes)
    return desc, *shapes


def _qk_norm_rotate(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first):
    desc, q_shape, k_shape = _qk_plan(_geometry(q), _geometry(k), _geometry(q_gain), _geometry(k_gain), _geometry(cos), _geometry(sin),
                                      _geometry(positions), eps, interleaved, heads_first)
    device = _place(q, k, q_gain, k_gain, cos, sin, positions)
    q_out, k_out = q.new_empty(q_shape), k.new_empty(k_shape)
    status = B.lib().asi_qk_norm_rotate(desc, q.data_ptr(), k.data_ptr(), _ptr(q_gain), _ptr(k_gain), _ptr(positions), cos.data_ptr(),
                                        sin.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), _stream(device))
    if status:
        B._check(status, "asi_qk_norm_rotate")
    return q_out, k_out


class _QkNormRotateFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first):
        ctx.save_for_backward(q, k, q_gain, k_gain, cos, sin, positions)
        ctx.options = eps, interleaved, heads_first
        return _qk_norm_rotate(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_q, grad_k):
        q, k, q_gain, k_gain, cos, sin, positions = ctx.saved_tensors
        eps, interleaved, heads_first = ctx.options
        dq, dk, dqg, dkg = qk_norm_rotate_grad(q, k, q_gain, k_gain, cos, sin, grad_q, grad_k, positions, eps=eps,
                                               interleaved=interleaved, heads_first=heads_first)
        return (dq, dk, None if q_gain is None else dqg.to(q_gain.dtype), None if k_gain is None else dkg.to(k_gain.dtype)) + (None,) * 6


def qk_norm_rotate(q: torch.Tensor, k: torch.Tensor, q_gain: Optional[torch.Tensor], k_gain: Optional[torch.Tensor],
                   cos: torch.Tensor, sin: torch.Tensor, positions: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
                   interleaved: bool = False, heads_first: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """Each head of q (batch, tokens, q_heads, head_dim) and k divided by its root mean square (there is no form without that),
    multiplied by the gain and turned by its token's position.  q and k may be views into one projection's output.  cos and sin (rotary_table) have
    rot_dim / 2 columns; the first rot_dim entries of a head are turned, in halves or (interleaved) in neighbouring pairs.
    positions (batch, tokens) or (tokens) int64, 0, 1, ... by default; one behind the table's end gives NaN.  heads_first:
    the results are (batch, heads, tokens, head_dim).  Differentiable in q, k and the gains."""
    eps, interleaved, heads_first = float(eps), bool(interleaved), bool(heads_first)
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or any(g is not None and g.requires_grad for g in (q_gain, k_gain))):
        return _QkNormRotateFn.apply(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first)
    return _qk_norm_rotate(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first)


@_plans
def _qk_grad_plan(q, k, q_gain, k_gain, cos, sin, positions, grad_q, grad_k, eps, interleaved, heads_first):
    desc = _qk_desc(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    for g, x, what in ((grad_q, q, "grad_q"), (grad_k, k, "grad_k")):
        if g[0] != _head_shape(x[0], heads_first) or g[2] != x[2]:
            raise ValueError(f"{what} has the result's shape and type")
    desc.q_out_stride[:], desc.k_out_stride[:] = _strides(grad_q, heads_first, "grad_q"), _strides(grad_k, heads_first, "grad_k")
    desc.dq_stride[:], desc.dk_stride[:] = _lying(q[0])[:3], _lying(k[0])[:3]
    return desc, int(B.lib().asi_qk_norm_rotate_grad_workspace_bytes(desc))


def qk_norm_rotate_grad(q, k, q_gain, k_gain, cos, sin, grad_q: torch.Tensor, grad_k: torch.Tensor, positions=None, *,
                        eps: float = 1e-6, interleaved: bool = False, heads_first: bool = False):
    """Gradients (dq, dk, dq_gain, dk_gain) of qk_norm_rotate from those of its results.  dq and dk are contiguous in the
    shape of q and k, the gains' gradients fp32 whether or not there are gains."""
    eps, interleaved, heads_first = float(eps), bool(interleaved), bool(heads_first)
    if grad_q.dim() == 4 and grad_q.stride(3) != 1:
        grad_q = grad_q.contiguous()
    if grad_k.dim() == 4 and grad_k.stride(3) != 1:
        grad_k = grad_k.contiguous()
    desc, nbytes = _qk_grad_plan(_geometry(q), _geometry(k), _geometry(q_gain), _geometry(k_gain), _geometry(cos), _geometry(sin),
                                 _geometry(positions), _geometry(grad_q), _geometry(grad_k), eps, interleaved, heads_first)
    device = _place(q, k, q_gain, k_gain, cos, sin, positions, grad_q, grad_k)
    dq, dk = q.new_empty(q.shape), k.new_empty(k.shape)
    dqg, dkg = (q.new_empty(q.shape[3], dtype=torch.float32) for _ in range(2))
    ws = _scratch(nbytes, q)
    status = B.lib().asi_qk_norm_rotate_grad(desc, q.data_ptr(), k.data_ptr(), _ptr(q_gain), _ptr(k_gain), _ptr(positions), cos.data_ptr(),
                                             sin.data_ptr(), grad_q.data_ptr(), grad_k.data_ptr(), dq.data_ptr(), dk.data_ptr(),
                                             dqg.data_ptr(), dkg.data_ptr(), _ptr(ws), nbytes, _stream(device))
    if status:
        B._check(status, "asi_qk_norm_rotate_grad")
    return dq, dk, dqg, dkg


# ---- token log probabilities without the logits ------------------------------------------------------------
class LinearLogprobs(NamedTuple):
    logprob: Optional[torch.Tensor]        # fp32, of each row's target; None without targets
    entropy: torch.Tensor                  # fp32


class LinearLogprobsGrad(NamedTuple):
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    hidden: Optional[torch.Tensor]         # gradients, in their tensors' type
    weight: Optional[torch.Tensor]


@_plans
def _linear_plan(hidden, weight, any_address, scale, ignore_index, grad):
    """Descriptor, scratch, the rows' shape, and whether hidden has to be laid out anew."""
    shape, stride, dtype = hidden
    if len(weight[0]) != 2 or not shape or shape[-1] != weight[0][1] or weight[2] != dtype or 0 in weight[0]:
        raise ValueError("hidden is (..., dim) and weight (vocab, dim), both of one type, neither dimension empty")
    dense = False
    try:
        rows, dim, apart = _row_layout(shape, stride, "hidden")
    except ValueError:
        rows, dim, apart, dense = shape[:-1].numel(), shape[-1], shape[-1], True
    if rows and apart < dim:
        apart, dense = dim, True
    vocab = weight[0][0]
    desc = B.LinearLogprobDesc(rows, dim, vocab, apart, _matrix(weight, "weight"), ignore_index, _dtype(dtype, "hidden"), scale, any_address, 0)
    L = B.lib()
    size = (L.asi_linear_logprobs_grad_workspace_bytes if grad else L.asi_linear_logprobs_workspace_bytes)(desc)
    return desc, int(size), shape[:-1], dense


def _linear_start(hidden, weight, scale, ignore_index, grad):
    desc, nbytes, shape, dense = _linear_plan(_geometry(hidden), _geometry(weight), int(weight.data_ptr() % 16 != 0), scale, ignore_index, grad)
    return desc, nbytes, shape, hidden.contiguous() if dense else hidden


def _linear_logprobs(hidden, weight, targets, scale, ignore_index, want_stats):
    desc, nbytes, shape, hidden = _linear_start(hidden, weight, scale, ignore_index, False)
    targets = _targets(targets, shape)
    device = _place(hidden, weight, targets)
    logprob = None if targets is None else hidden.new_empty(shape, dtype=torch.float32)
    entropy = hidden.new_empty(shape, dtype=torch.float32)
    stats = hidden.new_empty(shape + (2,), dtype=torch.float32) if want_stats else None
    ws = _scratch(nbytes, hidden)
    status = B.lib().asi_linear_logprobs(desc, hidden.data_ptr(), weight.data_ptr(), _ptr(targets), _ptr(logprob), entropy.data_ptr(),
                                         _ptr(stats), _ptr(ws), nbytes, _stream(device))
    if status:
        B._check(status, "asi_linear_logprobs")
    return logprob, entropy, stats


def _linear_grad(hidden, weight, targets, grad_logprob, grad_entropy, scale, ignore_index, kept, hidden_grad, weight_grad):
    """kept: (entropy, stats) of a forward call, or None."""
    like = hidden
    desc, nbytes, shape, hidden = _linear_start(hidden, weight, scale, ignore_index, True)
    targets = _targets(targets, shape)
    if targets is None and grad_logprob is not None:
        raise ValueError("grad_logprob weighs the targets' log probabilities: there are no targets")
    grad_logprob, grad_entropy = _weights(grad_logprob, shape, "grad_logprob"), _weights(grad_entropy, shape, "grad_entropy")
    device = _place(hidden, weight, targets, grad_logprob, grad_entropy)
    if kept is None:
        logprob = None if targets is None else hidden.new_empty(shape, dtype=torch.float32)
        entropy, stats = hidden.new_empty(shape, dtype=torch.float32), None
    else:
        logprob, (entropy, stats) = None, kept
    dhidden = like.new_empty(like.shape) if hidden_grad else None
    dweight = weight.new_empty(weight.shape) if weight_grad else None
    ws = _scratch(nbytes, hidden)
    status = B.lib().asi_linear_logprobs_grad(desc, int(kept is not None), hidden.data_ptr(), weight.data_ptr(), _ptr(targets), _ptr(stats),
                                              _ptr(logprob), _ptr(entropy), _ptr(grad_logprob), _ptr(grad_entropy), _ptr(dhidden),
                                              _ptr(dweight), _ptr(ws), nbytes, _stream(device))
    if status:
        B._check(status, "asi_linear_logprobs_grad")
    return LinearLogprobsGrad(logprob, entropy, dhidden, dweight)


class _LinearLogprobsFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, scale, ignore_index):
        logprob, entropy, stats = _linear_logprobs(hidden, weight, targets, scale, ignore_index, True)
        ctx.save_for_backward(hidden, weight, targets, entropy, stats)
        ctx.options = scale, ignore_index
        ctx.set_materialize_grads(False)
        return logprob, entropy

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_logprob, grad_entropy):
        if grad_logprob is None and grad_entropy is None:
            return (None,) * 5
        hidden, weight, targets, entropy, stats = ctx.saved_tensors
        r = _linear_grad(hidden, weight, targets, grad_logprob, grad_entropy, *ctx.options, (entropy, stats), *ctx.needs_input_grad[:2])
        return r.hidden, r.weight, None, None, None


def linear_logprobs(hidden: torch.Tensor, weight: torch.Tensor, targets: Optional[torch.Tensor] = None, *, scale: float = 1.0,
                    ignore_index: int = IGNORE_INDEX) -> LinearLogprobs:
    """Log probabilities of `targets` under softmax(scale * hidden @ weight.T) and the entropy of each row, without the logits: none
    are in memory in the forward pass, a piece of them and of their gradient in the backward pass (all of them for few rows, 64 at most).  Weights
    that cannot be multiplied as they lie, fp32 ones above all, are copied by pieces of up to 768 MiB, which for few rows is more than
    their logits; bf16 weights whose rows are a multiple of 64 entries, at multiples of 16 bytes, are read in place.  hidden (..., dim), weight (vocab, dim), fp32
    or bf16; targets (...) int64.  A row whose target is ignore_index is left out: logprob and entropy 0, no gradient, whatever it
    holds.  Differentiable in hidden and weight."""
    scale, ignore_index = float(scale), operator.index(ignore_index)
    if torch.is_grad_enabled() and (hidden.requires_grad or weight.requires_grad):
        return LinearLogprobs(*_LinearLogprobsFn.apply(hidden, weight, targets, scale, ignore_index))
    return LinearLogprobs(*_linear_logprobs(hidden, weight, targets, scale, ignore_index, False)[:2])


def linear_logprobs_grad(hidden: torch.Tensor, weight: torch.Tensor, targets: Optional[torch.Tensor], grad_logprob: Optional[torch.Tensor],
                         grad_entropy: Optional[torch.Tensor] = None, *, scale: float = 1.0, ignore_index: int = IGNORE_INDEX,
                         hidden_grad: bool = True, weight_grad: bool = True) -> LinearLogprobsGrad:
    """Gradients of sum(grad_logprob * logprob + grad_entropy * entropy) in hidden and weight, with both values, in one call: for a
    loss whose weights are known beforehand it replaces forward and backward.  Either gradient may be left out."""
    return _linear_grad(hidden, weight, targets, grad_logprob, grad_entropy, float(scale), operator.index(ignore_index), None, hidden_grad,
                        weight_grad)


# ---- dropout without a stored mask -------------------------------------------------------------------------
def _seed(seed, p: float):
    """A seed as the tensor that is read on the GPU, or as a number."""
    if isinstance(seed, torch.Tensor):
        if seed.dtype != torch.int64 or seed.numel() != 1:
            raise ValueError("a seed on the GPU is an int64 tensor of one entry")
        return seed, 0
    if seed is None:
        if p:
            raise ValueError("dropout needs a seed")
        return None, 0
    seed = operator.index(seed)
    if not -2 ** 63 <= seed < 2 ** 64:
        raise ValueError("a seed has 64 bits")
    return None, seed - 2 ** 64 if seed >= 2 ** 63 else seed


def _dropout_options(p, offset):
    p, offset = float(p), operator.index(offset)
    if not 0.0 <= p < 1.0 or round(p * 65536) > 65535:
        raise ValueError("p is at least 0 and, as a multiple of 2^-16, less than 1")
    if not -2 ** 63 <= offset < 2 ** 63:
        raise ValueError("offset has 64 bits")
    return p, offset


def _drawn(desc, number: int, offset: int):
    """The descriptor with a call's numbers; the kept one stays as it is."""
    desc = type(desc).from_buffer_copy(desc)
    desc.seed, desc.offset = number, offset
    return desc


@_plans
def _dropout_plan(geometry, p):
    shape, stride, dtype = geometry
    dense = False
    if _dense(shape, stride) or not shape:
        rows, dim, apart = 1 if 0 not in shape else 0, max(1, shape.numel()), max(1, shape.numel())
    else:
        try:
            rows, dim, apart = _row_layout(shape, stride, "x")
        except ValueError:
            dense = True
        if dense or (rows and apart < dim):
            rows, dim, apart, dense = 1, shape.numel(), shape.numel(), True
    return B.DropoutDesc(rows, dim, apart, dim, 0, 0, p, _dtype(dtype, "x"), 0), dense


def _dropout(x, p, seed, number, offset) -> torch.Tensor:
    desc, dense = _dropout_plan(_geometry(x), p)
    desc = _drawn(desc, number, offset)
    if dense:
        x = x.contiguous()
    device = _place(x, seed)
    y = x.new_empty(x.shape)
    status = B.lib().asi_dropout(desc, x.data_ptr(), _ptr(seed), y.data_ptr(), _stream(device))
    if status:
        B._check(status, "asi_dropout")
    return y


class _DropoutFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, number, offset):
        ctx.save_for_backward(seed)
        ctx.options = p, number, offset
        return _dropout(x, p, seed, number, offset)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        seed, = ctx.saved_tensors
        p, number, offset = ctx.options
        return _dropout(grad, p, seed, number, offset), None, None, None, None


def dropout(x: torch.Tensor, p: float, seed=None, offset: int = 0) -> torch.Tensor:
    """Each entry of x (fp32 or bf16) with probability p replaced by 0, the others divided by 1 - p; p is taken to the nearest multiple of
    2^-16.  Which ones is a function of the entry's place in x, the seed and the offset (a layer's number, say) alone, so no mask is kept:
    the gradient draws it again, and dropout(grad, p, seed, offset) is that gradient.  seed: an int, or an int64 tensor of one entry that
    is read on the GPU when the call runs (a captured step takes other numbers as the tensor changes).  Differentiable in x."""
    p, offset = _dropout_options(p, offset)
    seed, number = _seed(seed, p)
    if torch.is_grad_enabled() and x.requires_grad:
        return _DropoutFn.apply(x, p, seed, number, offset)
    return _dropout(x, p, seed, number, offset)


# ---- the edge between two blocks ---------------------------------------------------------------------------
class ResidualNorm(NamedTuple):
    stream: torch.Tensor                   # the new stream, x's type
    out: Optional[torch.Tensor]            # its norm, the block's type; None without


class ResidualNormGrad(NamedTuple):
    x: torch.Tensor
    y: Optional[torch.Tensor]
    post_gain: Optional[torch.Tensor]      # fp32, as those below; None where there is no such norm or gate
    gate: Optional[torch.Tensor]
    pre_gain: Optional[torch.Tensor]


class _ResidualOptions(NamedTuple):
    post_norm: bool
    pre_norm: bool
    scale: float
    eps: float
    p: float


def _rows_apart(shape, stride, what: str):
    """Rows and their distance, or None where they have to be laid out anew."""
    try:
        rows, dim, apart = _row_layout(shape, stride, what)
    except ValueError:
        return None
    return apart if not rows or apart >= dim else None


@_plans
def _residual_plan(x, y, post_gain, gate, pre_gain, dtype, options, grad):
    """Descriptor, scratch, and which of x and y have to be laid out anew."""
    shape = x[0]
    if not shape or not shape[-1]:
        raise ValueError("x is (..., dim)")
    dim, rows = shape[-1], shape[:-1].numel()
    if y is not None and y[0] != shape:
        raise ValueError("x and y have one shape")
    if y is None and (post_gain is not None or gate is not None):
        raise ValueError("post_gain and gate are those of a block's output y")
    if (post_gain is not None and not options.post_norm) or (pre_gain is not None and not options.pre_norm):
        raise ValueError("a gain is given for a norm that is not")
    if y is None and not options.pre_norm:
        raise ValueError("neither y nor a norm of the stream: there is nothing to do")
    given = [g for g in (post_gain, pre_gain, gate) if g is not None]
    for g in (post_gain, pre_gain):
        if g is not None and (g[0] != (dim,) or not _dense(*g[:2])):
            raise ValueError("the gains are contiguous tensors of dim entries")
    if any(g[2] != given[0][2] for g in given):
        raise ValueError("the gains and the gate have one type")
    gates = 0
    if gate is not None:
        if not _dense(*gate[:2]):
            raise ValueError("the gate is contiguous")
        if gate[0] == (dim,):
            gates = 1
        else:
            # leading dimensions as x's, then ones
            lead, n = gate[0][:-1], len(gate[0])
            k = next((i for i, s in enumerate(lead) if s == 1 and shape[i:i + 1] != (1,)), len(lead)) if n == len(shape) else -1
            if k < 0 or gate[0][-1] != dim or lead[:k] != shape[:k] or any(s != 1 for s in lead[k:]):
                raise ValueError("the gate is (dim), or x's shape with ones in place of the last dimensions before dim")
            gates = shape[:k].numel()
    out = y[2] if y is not None else dtype or x[2]
    apart = [_rows_apart(g[0], g[1], "x") if g is not None else dim for g in (x, y)]
    desc = B.ResidualDesc(rows, dim, apart[0] or dim, apart[1] or dim, gates if rows else 0, 0, 0, options.p,
                          _dtype(x[2], "x"), _dtype(out, "y"), _dtype(given[0][2], "a gain") if given else B.ASI_F32,
                          bool(options.post_norm and y is not None), options.scale, options.eps)
    return desc, int(B.lib().asi_residual_norm_grad_workspace_bytes(desc)) if grad else 0, out, apart[0] is None, apart[1] is None


def _residual(x, y, post_gain, gate, pre_gain, seed, draw, dtype, options):
    desc, _, out_dtype, x_anew, y_anew = _residual_plan(_geometry(x), _geometry(y), _geometry(post_gain), _geometry(gate), _geometry(pre_gain),
                                                        dtype, options, False)
    if options.p:
        desc = _drawn(desc, *draw)
    x, y = x.contiguous() if x_anew else x, y.contiguous() if y_anew else y
    device = _place(x, y, post_gain, gate, pre_gain, seed)
    stream = None if y is None else x.new_empty(x.shape)
    out = x.new_empty(x.shape, dtype=out_dtype) if options.pre_norm else None
    status = B.lib().asi_residual_norm(desc, x.data_ptr(), _ptr(y), _ptr(post_gain), _ptr(gate) if desc.gate_rows else None, _ptr(pre_gain),
                                       _ptr(seed), _ptr(stream), _ptr(out), _stream(device))
    if status:
        B._check(status, "asi_residual_norm")
    return stream, out


def _residual_grad(grad_stream, grad_out, stream, y, post_gain, gate, pre_gain, seed, draw, options, gains):
    desc, nbytes, out_dtype, s_anew, y_anew = _residual_plan(_geometry(stream), _geometry(y), _geometry(post_gain), _geometry(gate),
                                                             _geometry(pre_gain), None if grad_out is None else grad_out.dtype, options, True)
    if options.p:
        desc = _drawn(desc, *draw)
    for g, dtype, what in ((grad_stream, stream.dtype, "grad_stream"), (grad_out, out_dtype, "grad_out")):
        if g is not None and (g.shape != stream.shape or g.dtype != dtype):
            raise ValueError(f"{what} has the result's shape and type")
    if grad_out is not None and not options.pre_norm:
        raise ValueError("grad_out is the gradient of a norm that is not")
    if grad_stream is None and grad_out is None:
        raise ValueError("one gradient at least")
    grad_stream, grad_out = (g if g is None or g.is_contiguous() else g.contiguous() for g in (grad_stream, grad_out))
    s, y_rows = stream.contiguous() if s_anew else stream, y.contiguous() if y_anew else y
    device = _place(s, y_rows, post_gain, gate, pre_gain, seed, grad_stream, grad_out)
    dx, dy = stream.new_empty(stream.shape), None if y is None else y.new_empty(y.shape)
    dim = stream.shape[-1]
    new = lambda shape, there: stream.new_empty(shape, dtype=torch.float32) if there and gains else None  # noqa: E731
    dpost, dpre = new(dim, options.post_norm and y is not None), new(dim, options.pre_norm)
    dgate = None if gate is None else new(gate.shape, True)
    if dgate is not None and not desc.gate_rows:
        dgate.zero_()
    ws = _scratch(nbytes, stream)
    status = B.lib().asi_residual_norm_grad(desc, _ptr(grad_stream), _ptr(grad_out), s.data_ptr(), _ptr(y_rows), _ptr(post_gain),
                                            _ptr(gate) if desc.gate_rows else None, _ptr(pre_gain), _ptr(seed), dx.data_ptr(), _ptr(dy),
                                            _ptr(dpost), _ptr(dgate) if desc.gate_rows else None, _ptr(dpre), _ptr(ws), nbytes, _stream(device))
    if status:
        B._check(status, "asi_residual_norm_grad")
    return ResidualNormGrad(dx, dy, dpost, dgate, dpre)


class _ResidualNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, post_gain, gate, pre_gain, seed, draw, dtype, options):
        stream, out = _residual(x, y, post_gain, gate, pre_gain, seed, draw, dtype, options)
        ctx.save_for_backward(x if stream is None else stream, y, post_gain, gate, pre_gain, seed)
        ctx.draw, ctx.options = draw, options
        ctx.set_materialize_grads(False)
        return stream, out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_stream, grad_out):
        if grad_stream is None and grad_out is None:
            return (None,) * 9
        stream, y, post_gain, gate, pre_gain, seed = ctx.saved_tensors
        r = _residual_grad(grad_stream, grad_out, stream, y, post_gain, gate, pre_gain, seed, ctx.draw, ctx.options,
                           any(ctx.needs_input_grad[2:5]))
        of = lambda g, t: None if t is None or g is None else g.to(t.dtype)  # noqa: E731
        return r.x, r.y, of(r.post_gain, post_gain), of(r.gate, gate), of(r.pre_gain, pre_gain), None, None, None, None


def _residual_options(post_norm, pre_norm, scale, eps, p, seed, offset):
    p, offset = _dropout_options(p, offset)
    seed, number = _seed(seed, p)
    return _ResidualOptions(bool(post_norm), bool(pre_norm), float(scale), float(eps), p), seed, (number, offset)


def residual_norm(x: torch.Tensor, y: Optional[torch.Tensor] = None, post_gain: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, pre_gain: Optional[torch.Tensor] = None, *, post_norm: bool = True,
                  pre_norm: bool = True, scale: float = 1.0, eps: float = 1e-6, p: float = 0.0, seed=None, offset: int = 0,
                  dtype: Optional[torch.dtype] = None) -> ResidualNorm:
    """The edge between two blocks: stream = x + scale * gate * dropout(norm(y) * post_gain) and out = norm(stream) * pre_gain, the norms by the
    root of a row's mean square.  x (..., dim), the stream so far, fp32 or bf16; y, the block's output, of its shape, bf16 or x's type;
    out has y's type.  gate (dim), or x's shape with ones in place of the last dimensions before dim (a gate for each sequence, or for
    each token).  Without y the stream is x itself and out its norm, in `dtype` (x's by default); post_norm and pre_norm leave either norm out.
    p, seed and offset are dropout()'s.  The norm is that of the stream as it is rounded to its type.  For the gradients the stream and y are
    kept, nothing else.  Differentiable in x, y, the gains and the gate."""
    options, seed, draw = _residual_options(post_norm, pre_norm, scale, eps, p, seed, offset)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, y, post_gain, gate, pre_gain)):
        stream, out = _ResidualNormFn.apply(x, y, post_gain, gate, pre_gain, seed, draw, dtype, options)
    else:
        stream, out = _residual(x, y, post_gain, gate, pre_gain, seed, draw, dtype, options)
    return ResidualNorm(x if stream is None else stream, out)


def residual_norm_grad(grad_stream: Optional[torch.Tensor], grad_out: Optional[torch.Tensor], stream: torch.Tensor,
                       y: Optional[torch.Tensor] = None, post_gain: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                       pre_gain: Optional[torch.Tensor] = None, *, post_norm: bool = True, pre_norm: bool = True, scale: float = 1.0,
                       eps: float = 1e-6, p: float = 0.0, seed=None, offset: int = 0) -> ResidualNormGrad:
    """Gradients of residual_norm from those of its results (one of them may be None) and the stream that it gave (x where there is no
    y).  The gains' and the gate's are fp32; their sums over rows have an order that the shapes alone decide."""
    options, seed, draw = _residual_options(post_norm, pre_norm, scale, eps, p, seed, offset)
    return _residual_grad(grad_stream, grad_out, stream, y, post_gain, gate, pre_gain, seed, draw, options, True)


# ---- AdamW ------------------------------------------------------------------------------------------------
_CODES = (torch.float8_e4m3fn, torch.uint8)


class AdamW(torch.optim.Optimizer):
    """AdamW whose step updates all tensors of a group in one launch for up to 40 of them.

    state_bits 32: exp_avg and exp_avg_sq in fp32.  state_bits 8: exp_avg and exp_avg_sqrt, the root of the second moment,
    as 8-bit floats with an fp32 scale for each 256 elements (include/asi_lm.h).  master: bf16 parameters get an fp32 copy
    that the step updates and rounds into them; without it their updates are rounded away where they are below a
    parameter's last bit.  Parameters are contiguous and fp32 or bf16.  The number of steps is a group's ("step"); it and the
    rates are the host's, so that a captured step repeats them.  Whoever writes other values into a bf16 parameter writes them into
    its copy (state "master") too, or removes that: it is made anew.  A step takes `state` as it is then and keeps nothing else; a
    state that does not fit its parameter, or was made with other state_bits, is refused.
    """

    def __init__(self, params, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 1e-2, *, state_bits: int = 32, master: bool = False):
        if state_bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        if not (0.0 <= betas[0] < 1.0 and 0.0 <= betas[1] < 1.0 and eps >= 0.0):
            raise ValueError("betas are in [0, 1) and eps is not negative")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                                      master=master, step=0))

    def load_state_dict(self, state_dict) -> None:
        super().load_state_dict(state_dict)
        # torch casts floating states to their parameter's type on the way: put back what this optimiser keeps in other types
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        mine = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(saved, mine):
            for key, value in state_dict["state"].get(i, {}).items():
                if isinstance(value, torch.Tensor):
                    self.state[p][key] = value.detach().to(p.device).clone(memory_format=torch.contiguous_format)

    def _state(self, p: torch.Tensor, bits: int, master: bool) -> None:
        """Makes what a parameter lacks of its state, and refuses what a record cannot be made of."""
        s = self.state[p]
        if p.dtype not in _DTYPE or not p.is_contiguous():
            raise TypeError("parameters are contiguous and fp32 or bf16")
        second = "exp_avg_sq" if bits == 32 else "exp_avg_sqrt"
        blocks = -(-p.numel() // B.ADAMW_BLOCK)
        if "exp_avg" not in s:
            held = torch.float32 if bits == 32 else torch.float8_e4m3fn
            zeros = lambda shape, dtype: torch.zeros(shape, dtype=torch.uint8 if dtype.itemsize == 1 else dtype,  # noqa: E731
                                                     device=p.device).view(dtype)
            s["exp_avg"] = zeros(p.shape, held)
            s[second] = zeros(p.shape, held)
            if bits == 8:
                s["exp_avg_scale"], s["exp_avg_sqrt_scale"] = zeros((blocks,), torch.float32), zeros((blocks,), torch.float32)
        if master and p.dtype == torch.bfloat16 and "master" not in s:
            s["master"] = p.detach().float().clone()
        moments = (torch.float32,) if bits == 32 else _CODES
        want = {"exp_avg": (p.numel(), moments), second: (p.numel(), moments)}
        if bits == 8:
            want.update(exp_avg_scale=(blocks, (torch.float32,)), exp_avg_sqrt_scale=(blocks, (torch.float32,)))
        if "master" in s:
            want["master"] = p.numel(), (torch.float32,)
        for name, (count, dtypes) in want.items():
            t = s.get(name)
            if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.numel() != count or t.device != p.device or not t.is_contiguous():
                raise ValueError(f"the state {name!r} of a parameter with {p.numel()} entries and states of {bits} bits is a contiguous "
                                 f"tensor of {count} entries on its GPU, {' or '.join(map(str, dtypes))}")

    def _ready(self, members, given, bits: int, master: bool) -> List[torch.Tensor]:
        """The gradients in their parameters' layout, where the records could not be made at once."""
        _place(*members)
        for p, g in zip(members, given):
            self._state(p, bits, master)
            if g.is_sparse or g.shape != p.shape or g.dtype not in _DTYPE or g.device != p.device:
                raise ValueError("a gradient is dense, of its parameter's shape and device, in fp32 or bf16")
        return [g.contiguous() for g in given]

    @torch.no_grad()
    def step(self, closure=None, *, grad_scale: Optional[torch.Tensor] = None, skip: Optional[torch.Tensor] = None,
             grads: Optional[Sequence[Optional[torch.Tensor]]] = None):
        """One step.  grad_scale: fp32 tensor of one entry that every gradient is multiplied by (the factor that clips
        their norm, say); skip: int32 tensor of one entry, not zero to leave everything as it is (the step still counts).
        Both are read on the GPU.  grads: one gradient (or None) for each parameter in the order of the groups, in place of
        the parameters' own: fp32 gradients of bf16 parameters, as asi_weight_grad_linear gives."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for t, dtype in ((grad_scale, torch.float32), (skip, torch.int32)):
            if t is not None and (t.dtype != dtype or t.numel() != 1):
                raise ValueError("grad_scale is an fp32 and skip an int32 tensor of one entry")
        if grads is not None and len(grads) != sum(len(g["params"]) for g in self.param_groups):
            raise ValueError("one gradient (or None) for each parameter")
        at = 0
        for group in self.param_groups:
            members = group["params"]
            given = [p.grad for p in members] if grads is None else list(grads[at:at + len(members)])
            at += len(members)
            if not all(map(operator.is_not, given, itertools.repeat(None))):
                members = [p for p, g in zip(members, given) if g is not None]
                given = [g for g in given if g is not None]
            if not members:
                continue
            bits, master = group["state_bits"], group["master"]
            device = _place(members[0], grad_scale, skip)
            options = self.state, bits == 8, master, device, group["lr"], group["weight_decay"]
            records = B.adamw_records(members, given, *options)
            if records is None:
                given = self._ready(members, given, bits, master)
                records = B.adamw_records(members, given, *options)
                if records is None:
                    raise ValueError("parameters, states and gradients are dense tensors on one GPU")
            stream = _stream(device)
            group["step"] += 1
            b1, b2 = group["betas"]
            B._check(B.lib().asi_adamw(len(members), records, bits, b1, b2, group["eps"], group["step"], _ptr(grad_scale), _ptr(skip), stream),
                     "asi_adamw")
        return loss
