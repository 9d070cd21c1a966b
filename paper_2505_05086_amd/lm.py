"""The operators of a language model's fine-tuning step that stand beside the compressed layers: token log
probabilities and their gradient, embedding, norms of queries and keys with the position rotation, AdamW.

Thin layer over the C ABI of include/asi_lm.h: it checks and marshals arguments, allocates results and scratch from
torch's allocator on the current stream, and wires the calls into autograd where an input requires a gradient.  All
arithmetic runs in the HIP kernels; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
from typing import List, NamedTuple, Optional, Sequence, Tuple

import numpy as np
import torch

from . import binding as B

_DTYPE = {torch.float32: B.ASI_F32, torch.bfloat16: B.ASI_BF16}
IGNORE_INDEX = -100


# ---- argument checks --------------------------------------------------------------------------------------
def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise TypeError(f"{what} is fp32 or bf16, not {t.dtype}")
    return d


def _place(*ts: Optional[torch.Tensor]) -> int:
    """The current device's index; every tensor has to be there."""
    here = torch.cuda.current_device()
    for t in ts:
        if t is not None and (not t.is_cuda or t.device.index != here):
            raise ValueError("every tensor has to be on the current GPU (there is no CPU fallback)")
    return here


def _f32(t: Optional[torch.Tensor], shape, what: str) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != shape:
        raise ValueError(f"{what} is an fp32 tensor of shape {tuple(shape)}")
    return t.contiguous()


def _whole(t: torch.Tensor, what: str) -> torch.Tensor:
    if t.dtype != torch.int64:
        raise TypeError(f"{what} are int64, not {t.dtype}")
    return t.contiguous()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream(device: int) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _scratch(nbytes: int, device: int) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=f"cuda:{device}") if nbytes else None


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


def _rows(logits: torch.Tensor) -> torch.Tensor:
    if logits.dim() == 2:
        x = logits
    elif logits.dim() == 0:
        raise ValueError("logits have a dimension of the vocabulary")
    else:
        try:
            x = logits.view(-1, logits.shape[-1])
        except RuntimeError as e:
            raise ValueError("logits of more than two dimensions need rows at equal distances; shift the targets rather "
                             "than slicing the logits") from e
    if x.shape[1] < 1 or (x.stride(1) != 1 and x.shape[1] > 1):
        raise ValueError("the vocabulary is the innermost dimension of the logits, its entries next to each other")
    return x


def _logprob_desc(x: torch.Tensor, scale: float, ignore_index: int, top: int, grad_stride: int) -> B.LogprobDesc:
    rows, vocab = x.shape
    return B.LogprobDesc(rows, vocab, x.stride(0) if rows > 1 else vocab, grad_stride, ignore_index, _dtype(x, "logits"),
                         top, scale, 0)


def _token_logprobs(logits, targets, top, scale, ignore_index) -> TokenLogprobs:
    x = _rows(logits)
    shape = logits.shape[:-1]
    if targets is not None:
        if targets.shape != shape:
            raise ValueError(f"one target for each row: shape {tuple(shape)}, not {tuple(targets.shape)}")
        targets = _whole(targets, "targets")
    device = _place(x, targets)
    desc = _logprob_desc(x, scale, ignore_index, top, 0)
    new = dict(device=x.device, dtype=torch.float32)
    logprob = None if targets is None else torch.empty(shape, **new)
    entropy = torch.empty(shape, **new)
    top_logprob = top_index = None
    if top:
        top_logprob = torch.empty(shape + (top,), **new)
        top_index = torch.empty(shape + (top,), device=x.device, dtype=torch.int64)
    L = B.lib()
    ws = _scratch(L.asi_token_logprobs_workspace_bytes(desc), device)
    B._check(L.asi_token_logprobs(desc, x.data_ptr(), _ptr(targets), _ptr(logprob), entropy.data_ptr(), None, _ptr(top_logprob),
                                  _ptr(top_index), _ptr(ws), 0 if ws is None else ws.numel(), _stream(device)),
             "asi_token_logprobs")
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
    if torch.is_grad_enabled() and logits.requires_grad:
        return TokenLogprobs(*_TokenLogprobsFn.apply(logits, targets, top, scale, ignore_index))
    return _token_logprobs(logits, targets, top, scale, ignore_index)


def token_logprobs_grad(logits: torch.Tensor, targets: Optional[torch.Tensor], grad_logprob: Optional[torch.Tensor],
                        grad_entropy: Optional[torch.Tensor] = None, *, scale: float = 1.0, ignore_index: int = IGNORE_INDEX,
                        out: Optional[torch.Tensor] = None) -> TokenLogprobsGrad:
    """Gradient of sum(grad_logprob * logprob + grad_entropy * entropy) in the logits, with both values, in one pass over
    the logits.  For a loss whose weights are known beforehand this replaces forward and backward.  `out` may be `logits`
    themselves: the gradient then takes their place."""
    x = _rows(logits)
    shape = logits.shape[:-1]
    if targets is not None:
        if targets.shape != shape:
            raise ValueError(f"one target for each row: shape {tuple(shape)}, not {tuple(targets.shape)}")
        targets = _whole(targets, "targets")
    grad_logprob, grad_entropy = _f32(grad_logprob, shape, "grad_logprob"), _f32(grad_entropy, shape, "grad_entropy")
    device = _place(x, targets, grad_logprob, grad_entropy, out)
    rows, vocab = x.shape
    if out is None:
        # rows that lie in their 16 bytes as those of the logits do, so that both are accessed in whole vectors
        stride = vocab + (x.stride(0) - vocab) % (16 // x.element_size()) if rows > 1 else vocab
        if stride == vocab:
            out = torch.empty(logits.shape, dtype=x.dtype, device=x.device)
            dx = out.view(-1, vocab)
        else:
            dx = torch.empty_strided((rows, vocab), (stride, 1), dtype=x.dtype, device=x.device)
            out = dx.view(logits.shape)
    else:
        if out.shape != logits.shape or out.dtype != logits.dtype:
            raise ValueError("out has the logits' shape and type")
        dx = _rows(out)
        stride = dx.stride(0) if rows > 1 else vocab
    new = dict(device=x.device, dtype=torch.float32)
    logprob = None if targets is None else torch.empty(shape, **new)
    entropy = torch.empty(shape, **new)
    desc = _logprob_desc(x, scale, ignore_index, 0, stride)
    B._check(B.lib().asi_token_logprobs_grad(desc, x.data_ptr(), _ptr(targets), _ptr(grad_logprob), _ptr(grad_entropy),
                                             dx.data_ptr(), _ptr(logprob), entropy.data_ptr(), _stream(device)),
             "asi_token_logprobs_grad")
    return TokenLogprobsGrad(logprob, entropy, out)


# ---- embedding --------------------------------------------------------------------------------------------
def _matrix(t: torch.Tensor, what: str) -> torch.Tensor:
    if t.dim() != 2 or t.shape[1] < 1 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} is a matrix whose rows' entries are next to each other")
    return t


def _row_stride(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _embedding(tokens, table, scale, dtype) -> torch.Tensor:
    tokens = _whole(tokens, "tokens")
    _matrix(table, "table")
    device = _place(tokens, table)
    vocab, dim = table.shape
    out = torch.empty(tokens.shape + (dim,), dtype=dtype or table.dtype, device=table.device)
    desc = B.EmbeddingDesc(tokens.numel(), vocab, dim, _row_stride(table), dim, -1, _dtype(table, "table"), _dtype(out, "the result"),
                           scale, 0)
    B._check(B.lib().asi_embedding(desc, tokens.data_ptr(), table.data_ptr(), out.data_ptr(), _stream(device)), "asi_embedding")
    return out


class _EmbeddingFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, tokens, table, scale, padding_idx, dtype):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.scale, ctx.padding_idx, ctx.dtype = table.shape[0], scale, padding_idx, table.dtype
        return _embedding(tokens, table, scale, dtype)

    @staticmethod
    def backward(ctx, grad_out):
        tokens, = ctx.saved_tensors
        return None, embedding_grad(tokens, grad_out, ctx.vocab, scale=ctx.scale, padding_idx=ctx.padding_idx, dtype=ctx.dtype), \
            None, None, None


def embedding(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, padding_idx: Optional[int] = None,
              dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """scale * table[tokens] in `dtype` (the table's own by default), differentiable in the table.  The row of `padding_idx`
    gets no gradient; a token outside the table gives a row of NaN and no gradient."""
    if torch.is_grad_enabled() and table.requires_grad:
        return _EmbeddingFn.apply(tokens, table, scale, padding_idx, dtype)
    return _embedding(tokens, table, scale, dtype)


def embedding_grad(tokens: torch.Tensor, grad_out: torch.Tensor, vocab: int, *, scale: float = 1.0,
                   padding_idx: Optional[int] = None, dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None,
                   accumulate: bool = False) -> torch.Tensor:
    """Gradient of the table of embedding(): (vocab, dim) in `dtype`, or written to `out`; with `accumulate` added to it,
    which leaves rows without a token alone.  Sums are in fp32 and in the order of the tokens: equal calls, equal bits."""
    tokens = _whole(tokens, "tokens")
    if grad_out.shape[:-1] != tokens.shape or grad_out.dim() < 1:
        raise ValueError("grad_out has the tokens' shape and one more dimension")
    dim = grad_out.shape[-1]
    if grad_out.dim() != 2:
        grad_out = grad_out.reshape(-1, dim)
    if grad_out.stride(1) != 1 or (grad_out.shape[0] > 1 and grad_out.stride(0) < dim):
        grad_out = grad_out.contiguous()
    if accumulate and out is None:
        raise ValueError("accumulate adds to `out`")
    if out is None:
        out = torch.empty((vocab, dim), dtype=dtype, device=grad_out.device)
    elif out.shape != (vocab, dim):
        raise ValueError(f"out is ({vocab}, {dim})")
    _matrix(out, "out")
    device = _place(tokens, grad_out, out)
    if padding_idx is not None and not 0 <= padding_idx < vocab:
        raise ValueError("padding_idx is a token of the table")
    desc = B.EmbeddingDesc(tokens.numel(), vocab, dim, _row_stride(out), _row_stride(grad_out), -1 if padding_idx is None else padding_idx,
                           _dtype(out, "the gradient"), _dtype(grad_out, "grad_out"), scale, 0)
    L = B.lib()
    ws = _scratch(L.asi_embedding_grad_workspace_bytes(desc), device)
    B._check(L.asi_embedding_grad(desc, tokens.data_ptr(), grad_out.data_ptr(), out.data_ptr(), int(accumulate), _ptr(ws),
                                  0 if ws is None else ws.numel(), _stream(device)), "asi_embedding_grad")
    return out


# ---- norms of queries and keys with the position rotation -----------------------------------------------------
def rotary_table(length: int, rot_dim: int, base: float = 10000.0, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """cos and sin of position * base^(-2 e / rot_dim), fp32 (length, rot_dim / 2), computed in fp64."""
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    angle = torch.arange(length, dtype=torch.float64, device=device)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def _heads(t: torch.Tensor, what: str) -> torch.Tensor:
    if t.dim() != 4 or (t.stride(3) != 1 and t.shape[3] > 1):
        raise ValueError(f"{what} is (batch, tokens, heads, head_dim), a head's entries next to each other")
    return t


def _qk_desc(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved):
    _heads(q, "q")
    _heads(k, "k")
    batch, tokens, hq, dim = q.shape
    if k.shape[0] != batch or k.shape[1] != tokens or k.shape[3] != dim or k.dtype != q.dtype:
        raise ValueError("q and k have the same batch, tokens, head_dim and type")
    gain = None
    for g in (q_gain, k_gain):
        if g is not None:
            if g.shape != (dim,) or not g.is_contiguous() or (gain is not None and gain.dtype != g.dtype):
                raise ValueError("the gains are contiguous tensors of head_dim entries, both of one type")
            gain = g
    if cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32 or \
            not (cos.is_contiguous() and sin.is_contiguous()):
        raise ValueError("cos and sin are contiguous fp32 tables (positions, rot_dim / 2)")
    stride = 0
    if positions is not None:
        if positions.dtype != torch.int64:
            raise TypeError("positions are int64")
        if positions.shape == (tokens,):
            positions = positions.contiguous()
        elif positions.shape == (batch, tokens):
            if positions.stride(1) != 1 or positions.stride(0) < 0:
                positions = positions.contiguous()
            stride = positions.stride(0) if batch > 1 else 0
        else:
            raise ValueError("positions are (tokens) or (batch, tokens)")
    desc = B.QkDesc()
    desc.batch, desc.tokens, desc.max_position, desc.position_stride = batch, tokens, cos.shape[0], stride
    desc.q_stride[:], desc.k_stride[:] = q.stride()[:3], k.stride()[:3]
    desc.q_heads, desc.k_heads, desc.head_dim, desc.rot_dim = hq, k.shape[2], dim, 2 * cos.shape[1]
    desc.interleaved, desc.dtype, desc.eps = bool(interleaved), _dtype(q, "q"), eps
    desc.gain_dtype = B.ASI_F32 if gain is None else _dtype(gain, "a gain")
    return desc, positions


def _out_strides(t: torch.Tensor, heads_first: bool):
    a, b, c, _ = t.stride()
    return (a, c, b) if heads_first else (a, b, c)


def _head_shape(x: torch.Tensor, heads_first: bool):
    b, t, h, d = x.shape
    return (b, h, t, d) if heads_first else (b, t, h, d)


def _qk_norm_rotate(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first):
    desc, positions = _qk_desc(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    device = _place(q, k, q_gain, k_gain, cos, sin, positions)
    q_out = torch.empty(_head_shape(q, heads_first), dtype=q.dtype, device=q.device)
    k_out = torch.empty(_head_shape(k, heads_first), dtype=q.dtype, device=q.device)
    desc.q_out_stride[:], desc.k_out_stride[:] = _out_strides(q_out, heads_first), _out_strides(k_out, heads_first)
    B._check(B.lib().asi_qk_norm_rotate(desc, q.data_ptr(), k.data_ptr(), _ptr(q_gain), _ptr(k_gain), _ptr(positions), cos.data_ptr(),
                                        sin.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), _stream(device)), "asi_qk_norm_rotate")
    return q_out, k_out


class _QkNormRotateFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first):
        ctx.save_for_backward(q, k, q_gain, k_gain, cos, sin, positions)
        ctx.options = eps, interleaved, heads_first
        return _qk_norm_rotate(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first)

    @staticmethod
    def backward(ctx, grad_q, grad_k):
        q, k, q_gain, k_gain, cos, sin, positions = ctx.saved_tensors
        eps, interleaved, heads_first = ctx.options
        dq, dk, dqg, dkg = qk_norm_rotate_grad(q, k, q_gain, k_gain, cos, sin, grad_q, grad_k, positions, eps=eps,
                                               interleaved=interleaved, heads_first=heads_first)
        return (dq, dk, None if q_gain is None else dqg.to(q_gain.dtype), None if k_gain is None else dkg.to(k_gain.dtype)) + (None,) * 6


def qk_norm_rotate(q: torch.Tensor, k: torch.Tensor, q_gain: Optional[torch.Tensor], k_gain: Optional[torch.Tensor],
                   cos: torch.Tensor, sin: torch.Tensor, positions: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
                   interleaved: bool = False, heads_first: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """Each head of q (batch, tokens, q_heads, head_dim) and k divided by its root mean square, multiplied by the gain and
    turned by its token's position.  q and k may be views into one projection's output.  cos and sin (rotary_table) have
    rot_dim / 2 columns; the first rot_dim entries of a head are turned, in halves or (interleaved) in neighbouring pairs.
    positions (batch, tokens) or (tokens) int64, 0, 1, ... by default; one behind the table's end gives NaN.  heads_first:
    the results are (batch, heads, tokens, head_dim).  Differentiable in q, k and the gains."""
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or any(g is not None and g.requires_grad for g in (q_gain, k_gain))):
        return _QkNormRotateFn.apply(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first)
    return _qk_norm_rotate(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, heads_first)


def qk_norm_rotate_grad(q, k, q_gain, k_gain, cos, sin, grad_q: torch.Tensor, grad_k: torch.Tensor, positions=None, *,
                        eps: float = 1e-6, interleaved: bool = False, heads_first: bool = False):
    """Gradients (dq, dk, dq_gain, dk_gain) of qk_norm_rotate from those of its results.  dq and dk are contiguous in the
    shape of q and k, the gains' gradients fp32 whether or not there are gains."""
    desc, positions = _qk_desc(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    for g, x, what in ((grad_q, q, "grad_q"), (grad_k, k, "grad_k")):
        if g.shape != _head_shape(x, heads_first) or g.dtype != x.dtype:
            raise ValueError(f"{what} has the result's shape and type")
    grad_q, grad_k = (g if g.stride(3) == 1 or g.shape[3] == 1 else g.contiguous() for g in (grad_q, grad_k))
    device = _place(q, k, q_gain, k_gain, cos, sin, positions, grad_q, grad_k)
    dq, dk = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    dqg, dkg = (torch.empty(q.shape[3], dtype=torch.float32, device=q.device) for _ in range(2))
    desc.q_out_stride[:], desc.k_out_stride[:] = _out_strides(grad_q, heads_first), _out_strides(grad_k, heads_first)
    desc.dq_stride[:], desc.dk_stride[:] = dq.stride()[:3], dk.stride()[:3]
    L = B.lib()
    ws = _scratch(L.asi_qk_norm_rotate_grad_workspace_bytes(desc), device)
    B._check(L.asi_qk_norm_rotate_grad(desc, q.data_ptr(), k.data_ptr(), _ptr(q_gain), _ptr(k_gain), _ptr(positions), cos.data_ptr(),
                                       sin.data_ptr(), grad_q.data_ptr(), grad_k.data_ptr(), dq.data_ptr(), dk.data_ptr(), dqg.data_ptr(),
                                       dkg.data_ptr(), _ptr(ws), 0 if ws is None else ws.numel(), _stream(device)),
             "asi_qk_norm_rotate_grad")
    return dq, dk, dqg, dkg


# ---- AdamW ------------------------------------------------------------------------------------------------
class _Plan:
    """The records of a group's tensors, kept between steps: only parameters' and gradients' addresses are read anew."""

    def __init__(self, params, states, grads, bits):
        self.params, self.grads = params, grads
        self.first = [s["exp_avg"] for s in states]
        self.states = states
        self.records = (B.AdamwTensor * max(1, len(params)))()
        words = C.sizeof(B.AdamwTensor) // 8
        self.words = np.frombuffer(self.records, dtype=np.int64).reshape(-1, words)[:len(params)]
        self.reals = np.frombuffer(self.records, dtype=np.float64).reshape(-1, words)[:len(params)]
        for r, p, s, g in zip(self.records, params, states, grads):
            r.master = _ptr(s.get("master"))
            r.exp_avg = s["exp_avg"].data_ptr()
            r.exp_avg_sq = s["exp_avg_sq" if bits == 32 else "exp_avg_sqrt"].data_ptr()
            if bits == 8:
                r.exp_avg_scale, r.exp_avg_sq_scale = s["exp_avg_scale"].data_ptr(), s["exp_avg_sqrt_scale"].data_ptr()
            r.count, r.param_dtype, r.grad_dtype = p.numel(), _DTYPE[p.dtype], _DTYPE[g.dtype]

    def serves(self, params, grads) -> bool:
        return len(params) == len(self.params) and all(a is b for a, b in zip(params, self.params)) and \
            all(a is b or a.dtype == b.dtype for a, b in zip(grads, self.grads)) and \
            all(s["exp_avg"] is a for s, a in zip(self.states, self.first))


class AdamW(torch.optim.Optimizer):
    """AdamW whose step updates all tensors of a group in one launch for up to 40 of them.

    state_bits 32: exp_avg and exp_avg_sq in fp32.  state_bits 8: exp_avg and exp_avg_sqrt, the root of the second moment,
    as 8-bit floats with an fp32 scale for each 256 elements (include/asi_lm.h).  master: bf16 parameters get an fp32 copy
    that the step updates and rounds into them; without it their updates are rounded away where they are below a
    parameter's last bit.  Parameters are contiguous and fp32 or bf16.  The number of steps is a group's ("step").
    """

    def __init__(self, params, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 1e-2, *, state_bits: int = 32, master: bool = False):
        if state_bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        if not (0.0 <= betas[0] < 1.0 and 0.0 <= betas[1] < 1.0 and eps >= 0.0):
            raise ValueError("betas are in [0, 1) and eps is not negative")
        self._plans = {}
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                                      master=master, step=0))

    def __setstate__(self, state) -> None:
        super().__setstate__(state)
        self._plans = {}

    def load_state_dict(self, state_dict) -> None:
        super().load_state_dict(state_dict)
        self._plans.clear()
        # torch casts floating states to their parameter's type on the way: put back what this optimiser keeps in other types
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        mine = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(saved, mine):
            for key, value in state_dict["state"].get(i, {}).items():
                if isinstance(value, torch.Tensor):
                    self.state[p][key] = value.detach().clone().to(p.device)

    def _state(self, p: torch.Tensor, bits: int, master: bool) -> dict:
        s = self.state[p]
        if "exp_avg" not in s:
            if p.dtype not in _DTYPE or not p.is_contiguous():
                raise TypeError("parameters are contiguous and fp32 or bf16")
            held = torch.float32 if bits == 32 else torch.float8_e4m3fn
            zeros = lambda shape, dtype: torch.zeros(shape, dtype=torch.uint8 if dtype.itemsize == 1 else dtype,  # noqa: E731
                                                     device=p.device).view(dtype)
            s["exp_avg"] = zeros(p.shape, held)
            s["exp_avg_sq" if bits == 32 else "exp_avg_sqrt"] = zeros(p.shape, held)
            if bits == 8:
                blocks = -(-p.numel() // B.ADAMW_BLOCK)
                s["exp_avg_scale"], s["exp_avg_sqrt_scale"] = zeros((blocks,), torch.float32), zeros((blocks,), torch.float32)
        if master and p.dtype == torch.bfloat16 and "master" not in s:
            s["master"] = p.detach().float().clone()
        return s

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
        device = _place(grad_scale, skip)
        stream = _stream(device)
        at = 0
        for n, group in enumerate(self.param_groups):
            members = group["params"]
            given = [p.grad for p in members] if grads is None else grads[at:at + len(members)]
            at += len(members)
            if any(g is None for g in given):
                members = [p for p, g in zip(members, given) if g is not None]
                given = [g for g in given if g is not None]
            if not members:
                continue
            bits = group["state_bits"]
            plan = self._plans.get(n)
            if plan is None or not plan.serves(members, given):
                _place(*members)
                states = [self._state(p, bits, group["master"]) for p in members]
                _place(*[t for s in states for t in s.values() if isinstance(t, torch.Tensor)])
                plan = self._plans[n] = _Plan(list(members), states, list(given), bits)
                self._check_grads(plan, given, True)
            else:
                self._check_grads(plan, given, False)
            plan.words[:, 0] = [p.data_ptr() for p in members]
            plan.words[:, 1] = [g.data_ptr() for g in plan.grads]
            plan.reals[:, -2] = group["lr"]
            plan.reals[:, -1] = group["weight_decay"]
            group["step"] += 1
            b1, b2 = group["betas"]
            B._check(B.lib().asi_adamw(len(members), C.addressof(plan.records), bits, b1, b2, group["eps"], group["step"],
                                       _ptr(grad_scale), _ptr(skip), stream), "asi_adamw")
        return loss

    @staticmethod
    def _check_grads(plan: _Plan, given: List[torch.Tensor], fresh: bool) -> None:
        for i, (g, p) in enumerate(zip(given, plan.params)):
            if g is plan.grads[i] and not fresh:
                continue
            if g.is_sparse or g.shape != p.shape or g.dtype not in _DTYPE or g.device != p.device:
                raise ValueError("a gradient is dense, of its parameter's shape and device, in fp32 or bf16")
            plan.grads[i] = g.contiguous()
