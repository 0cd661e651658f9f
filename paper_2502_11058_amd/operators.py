"""The operators of a transformer's forward and backward pass on torch tensors: norms, rotary positions, attention and the
cross entropy of a language model's head, each in the library's own kernels.

Two forms of each.  `*_forward` and `*_backward` are the calls themselves: they check their tensors, allocate outputs and workspace
with torch, and enqueue kernels on torch's current stream.  `norm`, `rotary`, `attention` and `linear_cross_entropy` are the same
with gradients by autograd, for a model whose parameters `overlap.BackwardOverlap` holds.  Autograd does not record the kernels of a backward
pass: a second derivative through any of them (`create_graph=True`) raises RuntimeError.

Tensors are fp32 or bf16 (all of a call's tensors the same, statistics and losses fp32) on one GPU, which must be the current device.
Their last dimension is contiguous; the others may have any strides.  Arguments that do not fit raise ValueError or TypeError, what the library
refuses raises binding.DdpError.  Tensors made on another stream have to be ordered before the call by the caller, as with any torch operator.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

_DTYPES = {torch.float32: B.DDP_F32, torch.bfloat16: B.DDP_BF16}
_KINDS = {"layer": B.DDP_NORM_LAYER, "rms": B.DDP_NORM_RMS}
_LAYOUTS = {"half": B.DDP_ROTARY_HALF, "interleaved": B.DDP_ROTARY_INTERLEAVED}
_SCALINGS = {"plain": B.DDP_ROTARY_PLAIN, "linear": B.DDP_ROTARY_LINEAR, "stretched": B.DDP_ROTARY_STRETCHED, "by_wavelength": B.DDP_ROTARY_BY_WAVELENGTH}


_F32 = torch.float32
_device = torch._C._cuda_getDevice  # the current one; asked only where a tensor is on a GPU


# A small model's call is as long as its host side: a call looks at its tensors in a few expressions, and only what does not fit is
# looked at again for the message.

def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _typed(first: torch.Tensor) -> int:
    """The library's number of the type."""
    dtype = _DTYPES.get(first.dtype)
    if dtype is None:
        raise TypeError(f"tensors have to be float32 or bfloat16, not {first.dtype}")
    if not first.is_cuda:
        raise ValueError("tensors have to be on a GPU")
    # (the kernels go to the current device's stream: elsewhere they would run unordered with what makes and frees the tensors)
    if first.get_device() != _device():
        raise ValueError(f"tensors are on {first.device}, which is not the current device, cuda:{_device()}")
    return dtype


def _like(name: str, t: torch.Tensor, dtype: torch.dtype, first: torch.Tensor) -> None:
    """Of a type, on the first tensor's GPU."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} has to be {dtype}, not {t.dtype}")
    if t.device != first.device:
        raise ValueError(f"{name} is on {t.device}, not on {first.device}")


def _plain(name: str, t: torch.Tensor, shape, dtype: torch.dtype, first: torch.Tensor) -> None:
    """A contiguous tensor of one shape and type."""
    if t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.device == first.device:
        return
    if t.shape != shape:
        raise ValueError(f"{name} has to be {list(shape)}, not {list(t.shape)}")
    _like(name, t, dtype, first)
    raise ValueError(f"{name} has to be contiguous")


def _rows(name: str, t: torch.Tensor) -> Tuple[torch.Tensor, int, int]:
    """[.., cols] as rows with a single stride between them, without a copy where the strides allow it.  -> tensor, rows, stride."""
    s = t.shape
    if len(s) and t.is_contiguous():
        cols = s[-1]
        return t, t.numel() // cols if cols else 0, cols
    if not (t.dim() >= 1):
        raise ValueError(f"{name} needs a dimension")
    r = t if t.dim() == 2 else t.reshape(-1, t.shape[-1])
    if (r.shape[1] > 1 and r.stride(1) != 1) or (r.shape[0] > 1 and r.stride(0) < r.shape[1]):
        r = r.contiguous()
    return r, r.shape[0], r.stride(0)


def _alike(x: torch.Tensor, plain: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor like x; `plain` is x where x is contiguous for certain."""
    return torch.empty_like(x) if plain is x and x.is_contiguous() else torch.empty_like(x, memory_format=torch.contiguous_format)


def _workspace(n: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    return like.new_empty(n, dtype=torch.uint8) if n else None


# ------------------------------------------------------------------------------------------------------------
# norm
# ------------------------------------------------------------------------------------------------------------

def norm_forward(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *, kind: str = "layer",
                 eps: float = 1e-5) -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """Layer norm ("layer") or its root-mean-square form ("rms") over the last dimension.  -> y, mean (None for "rms"), rstd."""
    dtype = _typed(x)
    if kind not in _KINDS:
        raise ValueError(f"kind has to be one of {sorted(_KINDS)}, not {kind!r}")
    xr, rows, stride = _rows("x", x)
    _plain("weight", weight, x.shape[-1:], x.dtype, x)
    if bias is not None:
        _plain("bias", bias, x.shape[-1:], x.dtype, x)
    y = _alike(x, xr)
    rstd = x.new_empty(rows, dtype=_F32)
    mean = x.new_empty(rows, dtype=_F32) if kind == "layer" else None
    cols = x.shape[-1]
    B.ddp_norm_forward(B.ddp_norm(_KINDS[kind], dtype, rows, cols, stride, cols, eps), xr, weight, bias, y, mean, rstd)
    return y, mean, rstd


def norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: Optional[torch.Tensor], rstd: torch.Tensor, *, kind: str = "layer",
                  bias: bool = False) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """-> dx, dweight, dbias (None unless `bias`) from the forward call's x, weight, mean and rstd."""
    dtype = _typed(x)
    if kind not in _KINDS:
        raise ValueError(f"kind has to be one of {sorted(_KINDS)}, not {kind!r}")
    if dy.shape != x.shape:
        raise ValueError(f"dy has to be {list(x.shape)}, not {list(dy.shape)}")
    _like("dy", dy, x.dtype, x)
    cols = x.shape[-1]
    xr, rows, stride = _rows("x", x)
    dyr, _, dy_stride = _rows("dy", dy)
    _plain("weight", weight, x.shape[-1:], x.dtype, x)
    _plain("rstd", rstd, (rows,), _F32, x)
    if kind == "layer":
        _need(mean is not None, "mean is missing")
        _plain("mean", mean, (rows,), _F32, x)
    dx = _alike(x, xr)
    dw = torch.empty_like(weight)
    db = torch.empty_like(weight) if bias else None
    shape = B.ddp_norm(_KINDS[kind], dtype, rows, cols, stride, dy_stride, 0.0, cols)
    n = B.ddp_norm_backward_workspace(shape)
    B.ddp_norm_backward(shape, dyr, xr, weight, mean, rstd, dx, dw, db, _workspace(n, x), n)
    return dx, dw, db


# ------------------------------------------------------------------------------------------------------------
# rotary positions
# ------------------------------------------------------------------------------------------------------------

def rotary_table(rows: int, rotated: int, *, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                 context: float = 8192.0, amplitude: float = 1.0, device=None) -> torch.Tensor:
    """fp32 [rows, rotated / 2, 2]: cosine and sine of position * frequency, times `amplitude`; the frequencies changed for long contexts by
    `scaling`: "plain", "linear" (divided by factor), "stretched" (a larger base) or "by_wavelength" (see the header)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling has to be one of {sorted(_SCALINGS)}, not {scaling!r}")
    freq = B.ddp_rotary_frequencies(_SCALINGS[scaling], rotated, base, factor, low, high, context)
    table = torch.empty((rows, rotated // 2, 2), dtype=torch.float32, device=device or torch.device("cuda", torch.cuda.current_device()))
    _typed(table)
    B.ddp_rotary_table(rotated, freq, amplitude, rows, table)
    return table


def _tokens(name: str, x: torch.Tensor) -> Tuple[torch.Tensor, int, int]:
    """[.., heads, dim] as tokens with a single stride between them, without a copy where the strides allow it.  -> tensor, and the strides of
    tokens and heads."""
    s = x.shape
    if len(s) >= 2 and x.is_contiguous():
        return x, s[-2] * s[-1], s[-1]
    if not (x.dim() >= 2):
        raise ValueError(f"{name} has to be [.., heads, dim]")
    y = x if x.dim() == 3 else x.reshape((-1,) + x.shape[-2:]) if x.dim() > 3 else x[None]
    if y.shape[2] > 1 and y.stride(2) != 1:
        y = y.contiguous()
    return y, y.stride(0), y.stride(1)


def _rotary(q, k, table, positions, layout, inverse):
    dtype = _typed(q)
    if layout not in _LAYOUTS:
        raise ValueError(f"layout has to be one of {sorted(_LAYOUTS)}, not {layout!r}")
    q3, q_token, q_head = _tokens("q", q)
    lead = q.shape
    heads, dim = lead[-2], lead[-1]
    qo = _alike(q, q3)
    k3 = ko = None
    k_heads = k_token = k_head = 0
    if k is not None:
        _like("k", k, q.dtype, q)
        of_k = k.shape
        if not (len(of_k) == len(lead) and of_k[-1] == dim and (of_k[0] == lead[0] if len(lead) == 3 else of_k[:-2] == lead[:-2])):
            raise ValueError("q and k differ in more than their heads")
        k3, k_token, k_head = _tokens("k", k)
        k_heads = of_k[-2]
        ko = _alike(k, k3)
    of_table = table.shape
    if not (len(of_table) == 3 and of_table[2] == 2):
        raise ValueError("table has to be [rows, pairs, 2]")
    if not (table.dtype is _F32 and table.is_contiguous() and table.device == q.device):
        _plain("table", table, of_table, _F32, q)
    tokens = q.numel() // (heads * dim) if heads * dim else 0
    width, size = lead[-3] if len(lead) > 2 else 1, 4
    if positions is not None:
        if positions.numel() != tokens:
            raise ValueError(f"{positions.numel()} positions for {tokens} tokens")
        # (as many in another order, such as [tokens, batch], would turn tokens by each other's angles)
        if positions.dim() != 1 and positions.shape != lead[:-2] and [n for n in positions.shape if n != 1] != [n for n in lead[:-2] if n != 1]:
            raise ValueError(f"positions have to be {list(lead[:-2])} as the tokens are, or in one row, not {list(positions.shape)}")
        if positions.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"positions have to be int32 or int64, not {positions.dtype}")
        if positions.device != q.device:
            raise ValueError(f"positions are on {positions.device}, not on {q.device}")
        if not positions.is_contiguous():
            positions = positions.contiguous()
        size = 8 if positions.dtype is torch.int64 else 4
    B.ddp_rotary(B.ddp_rotary_shape(_LAYOUTS[layout], dtype, tokens, heads, k_heads, dim, 2 * of_table[1], q_token, q_head, k_token, k_head, heads * dim, dim,
                                    k_heads * dim, dim, of_table[0], max(width, 1), size, inverse), q3, k3, table, positions, qo, ko)
    return qo, ko


def rotary_forward(q: torch.Tensor, k: Optional[torch.Tensor], table: torch.Tensor, positions: Optional[torch.Tensor] = None, *, layout: str = "half"):
    """q [.., tokens, heads, dim] and k (or None) with the first 2 * pairs channels of each head rotated by their tokens' rows of the
    table: `positions` (int32 or int64 [.., tokens], or all in one row), or the tokens' places in their sequence.  -> rotated q, rotated k."""
    return _rotary(q, k, table, positions, layout, 0)


def rotary_backward(dq: torch.Tensor, dk: Optional[torch.Tensor], table: torch.Tensor, positions: Optional[torch.Tensor] = None, *, layout: str = "half"):
    """Gradients of rotary_forward's inputs from those of its outputs."""
    return _rotary(dq, dk, table, positions, layout, 1)


# ------------------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------------------

def _heads(t: torch.Tensor, packed: bool) -> Tuple[torch.Tensor, B.ddp_heads]:
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        t = t.contiguous()
        s = t.stride()
    return t, B.ddp_heads(t.data_ptr() or None, 0, s[0], s[1]) if packed else B.ddp_heads(t.data_ptr() or None, s[0], s[1], s[2])


def _attention_shape(q, k, v, causal, scale, cu_q, cu_k) -> Tuple[B.ddp_attention, bool, torch.Size, tuple]:
    """-> the library's description, whether packed, q's shape and lse's."""
    dtype, packed = _typed(q), cu_q is not None
    _like("k", k, q.dtype, q)
    _like("v", v, q.dtype, q)
    of_q, of_k = q.shape, k.shape
    if not ((cu_k is not None) == packed and len(of_q) == (3 if packed else 4) and of_k == v.shape and len(of_k) == len(of_q) and of_k[-1] == of_q[-1] and
            (packed or of_k[0] == of_q[0])):
        _need((cu_q is None) == (cu_k is None), "cu_q and cu_k go together")
        _need(q.dim() == (3 if packed else 4), "q has to be [tokens, heads, dim] with cu_q and cu_k" if packed else "q has to be [batch, tokens, heads, dim] without cu_q and cu_k")
        _need(k.shape == v.shape and k.dim() == q.dim() and k.shape[-1] == q.shape[-1], "k and v have to be alike, and q but for tokens and heads")
        raise ValueError("q and k differ in the batch")
    if packed:
        for name, cu in (("cu_q", cu_q), ("cu_k", cu_k)):
            _need(cu.dim() == 1 and cu.numel() >= 1 and cu.numel() == cu_q.numel(), "cu_q and cu_k have to be [sequences + 1]")
            _plain(name, cu, cu.shape, torch.int32, q)
        q_tokens, heads, dim = of_q
        batch, k_tokens, k_heads, of_lse = cu_q.numel() - 1, of_k[0], of_k[1], (heads, q_tokens)
    else:
        batch, q_tokens, heads, dim = of_q
        k_tokens, k_heads, of_lse = of_k[1], of_k[2], (batch, heads, q_tokens)
    return B.ddp_attention(dtype, bool(causal), heads, k_heads, dim, batch, q_tokens, k_tokens, max(dim, 1) ** -0.5 if scale is None else scale, packed), packed, of_q, of_lse


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = True, scale: Optional[float] = None,
                      cu_q: Optional[torch.Tensor] = None, cu_k: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """softmax(scale q k^T) v per head.  q [batch, tokens, heads, dim], k and v [batch, tokens, key heads, dim] with key heads dividing
    heads; or packed [tokens, heads, dim] with the sequences' starts cu_q, cu_k (int32 [sequences + 1], on the GPU).  Causal: the
    last query of a sequence sees all its keys.  scale: dim ** -0.5.  -> o, lse [batch, heads, tokens] or [heads, tokens]."""
    shape, packed, _, of_lse = _attention_shape(q, k, v, causal, scale, cu_q, cu_k)
    (q, hq), (k, hk), (v, hv) = _heads(q, packed), _heads(k, packed), _heads(v, packed)
    o = _alike(q, q)
    lse = q.new_empty(of_lse, dtype=_F32)
    n = B.ddp_attention_forward_workspace(shape, hq, hk, hv)
    B.ddp_attention_forward(shape, hq, hk, hv, cu_q, cu_k, _heads(o, packed)[1], lse, _workspace(n, q), n)
    return o, lse


def attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor, *, causal: bool = True,
                       scale: Optional[float] = None, cu_q: Optional[torch.Tensor] = None,
                       cu_k: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """-> dq, dk, dv from the forward call's arguments and results; the probabilities are formed again."""
    shape, packed, of_q, of_lse = _attention_shape(q, k, v, causal, scale, cu_q, cu_k)
    if not (do.shape == of_q and o.shape == of_q):
        raise ValueError(f"do and o have to be {list(q.shape)}")
    _like("do", do, q.dtype, q)
    _like("o", o, q.dtype, q)
    _plain("lse", lse, of_lse, _F32, q)
    (q, hq), (k, hk), (v, hv), (o, ho), (do, hd) = _heads(q, packed), _heads(k, packed), _heads(v, packed), _heads(o, packed), _heads(do, packed)
    dq, dk, dv = _alike(q, q), _alike(k, k), _alike(v, v)
    n = B.ddp_attention_backward_workspace(shape, hd, hq, hk, hv)
    B.ddp_attention_backward(shape, hd, hq, hk, hv, ho, lse, cu_q, cu_k, _heads(dq, packed)[1], _heads(dk, packed)[1], _heads(dv, packed)[1],
                             _workspace(n, q), n)
    return dq, dk, dv


# ------------------------------------------------------------------------------------------------------------
# cross entropy of a language model's head
# ------------------------------------------------------------------------------------------------------------

def _head(x, weight, targets) -> Tuple[B.ddp_head, torch.Tensor, torch.Tensor, torch.Tensor]:
    dtype = _typed(x)
    _like("weight", weight, x.dtype, x)
    xr, rows, x_stride = _rows("x", x)
    of_x, of_w = x.shape, weight.shape
    hidden = of_x[-1]
    if not (len(of_w) == 2 and of_w[1] == hidden):
        raise ValueError("weight has to be [vocab, hidden]")
    wr, vocab, w_stride = _rows("weight", weight)
    if targets.shape != of_x[:-1]:
        raise ValueError(f"targets have to be {list(x.shape[:-1])}, not {list(targets.shape)}")
    _like("targets", targets, torch.int64, x)
    return B.ddp_head(dtype, rows, vocab, hidden, x_stride, w_stride, hidden, hidden), xr, wr, targets if targets.is_contiguous() else targets.contiguous()


def linear_cross_entropy_forward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """Per-token cross entropy of the logits x weight^T, which are never kept.  x [.., hidden], weight [vocab, hidden], targets
    int64 [..]; a target outside [0, vocab) has loss 0.  -> loss, log of the sum of exponentials; fp32 [..]."""
    head, xr, wr, t = _head(x, weight, targets)
    loss = x.new_empty(targets.shape, dtype=_F32)
    lse = torch.empty_like(loss)
    n = B.ddp_cross_entropy_forward_workspace(head, xr, wr)
    B.ddp_cross_entropy_forward(head, xr, wr, t, loss, lse, _workspace(n, x), n)
    return loss, lse


def linear_cross_entropy_backward(dloss: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, *, need_dx: bool = True,
                                  need_dweight: bool = True) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """-> dx, dweight from the gradient of the losses [..]; the logits are formed again, in pieces of the vocabulary."""
    head, xr, wr, t = _head(x, weight, targets)
    _plain("lse", lse, targets.shape, _F32, x)
    if dloss.shape != targets.shape:
        raise ValueError(f"dloss has to be {list(targets.shape)}, not {list(dloss.shape)}")
    dloss = dloss.contiguous()
    _plain("dloss", dloss, targets.shape, _F32, x)
    dx = _alike(x, xr) if need_dx else None
    dw = _alike(weight, wr) if need_dweight else None
    if dx is None and dw is None:
        return None, None
    n = B.ddp_cross_entropy_backward_workspace(head, xr, wr)
    B.ddp_cross_entropy_backward(head, dloss, xr, wr, t, lse, dx, dw, _workspace(n, x), n)
    return dx, dw


# ------------------------------------------------------------------------------------------------------------
# with gradients by autograd
# ------------------------------------------------------------------------------------------------------------

class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, kind, eps):
        y, mean, rstd = norm_forward(x, weight, bias, kind=kind, eps=eps)
        ctx.save_for_backward(x, weight, rstd, *(() if mean is None else (mean,)))
        ctx.kind, ctx.bias = kind, bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, rstd, *mean = ctx.saved_tensors
        dx, dw, db = norm_backward(dy, x, weight, mean[0] if mean else None, rstd, kind=ctx.kind, bias=ctx.bias)
        return dx, dw, db, None, None


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, table, positions, layout):
        ctx.save_for_backward(table, *(() if positions is None else (positions,)))
        ctx.layout = layout
        return rotary_forward(q, k, table, positions, layout=layout)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        table, *positions = ctx.saved_tensors
        dq, dk = rotary_backward(dq, dk, table, positions[0] if positions else None, layout=ctx.layout)
        return dq, dk, None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale, cu_q, cu_k):
        o, lse = attention_forward(q, k, v, causal=causal, scale=scale, cu_q=cu_q, cu_k=cu_k)
        ctx.save_for_backward(q, k, v, o, lse, *(() if cu_q is None else (cu_q, cu_k)))
        ctx.causal, ctx.scale = causal, scale
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, *cu = ctx.saved_tensors
        cu_q, cu_k = cu if cu else (None, None)
        return (*attention_backward(do, q, k, v, o, lse, causal=ctx.causal, scale=ctx.scale, cu_q=cu_q, cu_k=cu_k), None, None, None, None)


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets):
        loss, lse = linear_cross_entropy_forward(x, weight, targets)
        ctx.save_for_backward(x, weight, targets, lse)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        x, weight, targets, lse = ctx.saved_tensors
        dx, dw = linear_cross_entropy_backward(dloss, x, weight, targets, lse, need_dx=ctx.needs_input_grad[0], need_dweight=ctx.needs_input_grad[1])
        return dx, dw, None


def norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *, kind: str = "layer", eps: float = 1e-5) -> torch.Tensor:
    return _Norm.apply(x, weight, bias, kind, eps)


def rotary(q: torch.Tensor, k: torch.Tensor, table: torch.Tensor, positions: Optional[torch.Tensor] = None, *, layout: str = "half"):
    return _Rotary.apply(q, k, table, positions, layout)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, causal: bool = True, scale: Optional[float] = None, cu_q: Optional[torch.Tensor] = None,
              cu_k: Optional[torch.Tensor] = None) -> torch.Tensor:
    return _Attention.apply(q, k, v, causal, scale, cu_q, cu_k)


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, *, reduction: str = "mean") -> torch.Tensor:
    """reduction: "none" (per token), "sum", or "mean" over the tokens whose target is a word (0 if none is)."""
    if not (reduction in ("none", "sum", "mean")):
        raise ValueError(f"reduction has to be none, sum or mean, not {reduction!r}")
    loss = _LinearCrossEntropy.apply(x, weight, targets)
    if reduction == "none":
        return loss
    if reduction == "sum":
        return loss.sum()
    words = ((targets >= 0) & (targets < weight.shape[0])).sum()
    return loss.sum() / words.clamp(min=1)
