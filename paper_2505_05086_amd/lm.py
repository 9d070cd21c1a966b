"""The operators of a language model's fine-tuning step that stand beside the compressed layers: token log
probabilities and their gradient, embedding, norms of queries and keys with the position rotation, AdamW.

Thin layer over the C ABI of include/asi_lm.h: it checks and marshals arguments, allocates results and scratch from
torch's allocator on the current stream, and wires the calls into autograd where an input requires a gradient.  All
arithmetic runs in the HIP kernels; there is no CPU fallback.
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
