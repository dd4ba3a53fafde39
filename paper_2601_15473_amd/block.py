"""The operators of a transformer block that stand between its sketched layers, for PyTorch:

``attention``        softmax attention of packed heads, for training and for generation from a cache
``head_norm_rope``   RMS norm of every query and key head with the position rotation in the same pass
``embedding``        rows of a table by token, scaled
``dropout``          dropout by a counter-based generator whose mask is never stored, with a residual added
``layer_norm``       layer norm of rows, with a residual added first
``linear``           a layer that stays dense, with bias, activation and residual
``distillation_loss``  the loss of logits against a teacher's largest ones and against labels

Each has its gradients.  Everything that computes runs in libsk's HIP kernels (include/sk_block.h says what, in full);
PyTorch provides the tensors, the current stream and the autograd graph.  There is no CPU path: tensors that are not on a GPU raise.
Tensors are float32 or bfloat16, all floating ones of a call alike; sums are fp32 either way.
"""
from __future__ import annotations

import ctypes
import functools

import torch
from torch.autograd import forward_ad

from . import libsk as sk
from .nn import _DTYPES, _native, _on, _queueing, _stream, _workspace

_REFUSED = 2 ** 64 - 1


def _natively() -> bool:
    """Whether a call may try its native function (csrc/sk_torch_block.cpp), which computes the same for plain tensors outside of
    compilation, tracing and torch's modes and transforms, and gives None for anything else."""
    return _native is not None and not torch.compiler.is_compiling()


def _training(*tensors) -> bool:
    """Whether a call has to keep what its backward pass needs.  (A traced call does: the trace's own calls may want gradients.)

    Whatever the native functions leave goes through an operator's autograd function, gradients or not: a trace records that call, where it would see
    none of a kernel's launches, and a tangent, for which there is no rule, is refused there."""
    return torch.jit.is_tracing() or (torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors))


class _Underivable(torch.autograd.Function):
    """Results of ``compute`` that depend on something, with no rule for how."""

    @staticmethod
    def forward(ctx, anchor, compute):
        return compute()

    @staticmethod
    def backward(ctx, *unused):
        raise RuntimeError("libsk: a gradient of a gradient was asked for; these operators are differentiated once, not twice")


def _once(backward):
    """A backward pass whose gradients refuse to be differentiated, where a graph of it is made (create_graph): all of them do, also
    those that depend on nothing that has a gradient, so that a program is told the same whatever it differentiates."""
    @functools.wraps(backward)
    def wrapper(ctx, *grads):
        if not torch.is_grad_enabled():
            return backward(ctx, *grads)
        return _Underivable.apply(torch.empty(0, requires_grad=True), lambda: backward(ctx, *grads))
    return wrapper


def _checked(what: str, first: torch.Tensor, **tensors):
    """Refuses tensors that are not on ``first``'s GPU or not of its type."""
    if first.dtype not in _DTYPES:
        raise TypeError(f"{what}: dtype {first.dtype} is not supported (float32 or bfloat16)")
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise RuntimeError(f"{what}: {name} is on {t.device}; libsk runs on the GPU only (there is no CPU implementation)")
        if t.device != first.device:
            raise RuntimeError(f"{what}: {name} is on {t.device}, not on {first.device}")
        if t.dtype != first.dtype:
            raise TypeError(f"{what}: {name} has dtype {t.dtype}, not {first.dtype}")


def _integers(what: str, name: str, t: torch.Tensor, device: torch.device):
    if t.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"{what}: {name} has dtype {t.dtype}, not int32 or int64")
    if t.device != device:
        raise RuntimeError(f"{what}: {name} is on {t.device}, not on {device}")


def _dense(t: torch.Tensor) -> torch.Tensor:
    """t with dense rows from a 16-byte boundary on: itself where it is that already."""
    if t.is_contiguous() and t.data_ptr() % 16 == 0:
        return t
    return t.clone(memory_format=torch.contiguous_format)


def _strided(t: torch.Tensor, token: int) -> torch.Tensor:
    """t where the library takes its strides (the last dimension's values consecutive, the others whole multiples of 16 bytes,
    the dimension ``token`` less than 2^22 elements), else a dense copy."""
    unit = 16 // t.element_size()
    if t.data_ptr() % 16 == 0 and (t.stride(-1) == 1 or t.size(-1) == 1):
        for d in range(t.dim() - 1):
            if t.size(d) > 1 and (t.stride(d) % unit != 0 or t.stride(d) >= (1 << 22 if d == token else 1 << 40)):
                break
        else:
            return t
    return t.clone(memory_format=torch.contiguous_format)


def _apart(t: torch.Tensor) -> torch.Tensor:
    """Keys or values [batch, tokens, heads, head_dim] as the library takes them: copied too where tokens overlap in memory (expanded ones), since
    what a kernel reads past the last token is then that token again."""
    t = _strided(t, 1)
    return t if t.size(1) <= 1 or t.stride(1) >= t.size(3) else t.clone(memory_format=torch.contiguous_format)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

# (The library's structures are made in one call each: a compiler that looks at these functions takes an assignment to an array in one for one to its class.)
_2, _3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3


def _attention_shape(q, k, v, q_lengths, k_lengths, causal, scale):
    batch, q_len, heads, head_dim = q.shape
    return sk.AttentionShape(batch, q_len, k.shape[1], heads, k.shape[2], head_dim, int(causal), scale, _DTYPES[q.dtype],
                             _3(*q.stride()[:3]), _3(*k.stride()[:3]), _3(*v.stride()[:3]),
                             None if q_lengths is None else q_lengths.data_ptr(), None if k_lengths is None else k_lengths.data_ptr())


def _attention_workspace(shape, backward, device, stream):
    need = sk.sk_attention_workspace_bytes(shape, backward)
    if need == _REFUSED:
        raise sk.SkError(sk.SK_ERR_UNSUPPORTED)
    return _workspace(device, stream, need)


def _attention_forward(q, k, v, q_lengths, k_lengths, causal, scale, training):
    """o, and for a backward pass the rows' log of their sums and (bf16) what o's rounding left off."""
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device) if training else None
    rest = torch.empty_like(o) if training and q.dtype == torch.bfloat16 else None
    if q.numel() == 0 or k.numel() == 0:
        return o.zero_(), lse, rest
    shape = _attention_shape(q, k, v, q_lengths, k_lengths, causal, scale)
    with _on(q.device), _queueing:
        stream = _stream(q.device)
        ws = _attention_workspace(shape, 0, q.device, stream)
        sk.check(sk.sk_attention_fwd(shape, q, k, v, o, lse, rest, ws, ws.numel(), stream))
    return o, lse, rest


class AttentionFunction(torch.autograd.Function):
    """See ``attention``; keeps q, k, v, o (in bf16 with what its rounding left off) and a row's log of its sum of exponentials, and
    recomputes the probabilities."""

    @staticmethod
    def forward(ctx, q, k, v, q_lengths, k_lengths, causal, scale, training):
        qs, ks, vs = _strided(q, 1), _apart(k), _apart(v)
        o, lse, rest = _attention_forward(qs, ks, vs, q_lengths, k_lengths, causal, scale, training)
        ctx.save_for_backward(qs, ks, vs, o, lse, rest, q_lengths, k_lengths)
        ctx.causal, ctx.scale = causal, scale
        return o

    @staticmethod
    @_once
    def backward(ctx, do):
        q, k, v, o, lse, rest, q_lengths, k_lengths = ctx.saved_tensors
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        if q.numel() == 0 or k.numel() == 0:
            return dq.zero_(), dk.zero_(), dv.zero_(), None, None, None, None, None
        do = _dense(do)
        shape = _attention_shape(q, k, v, q_lengths, k_lengths, ctx.causal, ctx.scale)
        with _on(q.device), _queueing:
            stream = _stream(q.device)
            ws = _attention_workspace(shape, 1, q.device, stream)
            sk.check(sk.sk_attention_bwd(shape, q, k, v, o, lse, rest, do, dq, dk, dv, ws, ws.numel(), stream))
        return dq, dk, dv, None, None, None, None, None


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_lengths: torch.Tensor | None = None,
              k_lengths: torch.Tensor | None = None, *, causal: bool = False, scale: float | None = None) -> torch.Tensor:
    """Softmax attention: ``q [batch, q_len, heads, head_dim]`` on ``k``, ``v [batch, k_len, kv_heads, head_dim]``, where each of
    the kv_heads serves heads / kv_heads query heads in a row; the result is as q, dense.

    ``q_lengths``, ``k_lengths`` (integers [batch] on the GPU; int32 is taken as it is): how many queries and keys of each
    sequence count (a cache's filled part, a padded batch's sentences), clamped to what there is.  With ``causal`` the last query that
    counts stands at the last key that counts and every query sees the keys up to its own.  A query that sees no key gives
    zeros, and no gradient.  ``scale`` is head_dim ** -0.5 unless given.

    Strided views (slices of a projection's output, of a cache) are read in place.  head_dim: a multiple of 8 up to 128.
    """
    if _natively():
        o = _native.attention(q, k, v, q_lengths, k_lengths, causal, scale)
        if o is not None:
            return o
    _checked("attention", q, q=q, k=k, v=v)
    if q.dim() != 4 or k.dim() != 4 or k.shape != v.shape or q.shape[0] != k.shape[0] or q.shape[3] != k.shape[3]:
        raise ValueError("attention: shapes do not match (q [batch, q_len, heads, head_dim], k and v [batch, k_len, kv_heads, head_dim])")
    if k.shape[2] == 0 or q.shape[2] % k.shape[2] != 0:
        raise ValueError(f"attention: {q.shape[2]} query heads are not a multiple of {k.shape[2]} key heads")
    lengths = []
    for name, t, most in (("q_lengths", q_lengths, q.shape[1]), ("k_lengths", k_lengths, k.shape[1])):
        if t is not None:
            _integers("attention", name, t, q.device)
            if t.shape != (q.shape[0],):
                raise ValueError(f"attention: {name} has shape {tuple(t.shape)}, not [{q.shape[0]}]")
            t = (t if t.dtype == torch.int32 else t.clamp(0, most).to(torch.int32)).contiguous()   # (not the low halves of what does not fit)
        lengths.append(t)
    scale = float(q.shape[3]) ** -0.5 if scale is None else float(scale)
    return AttentionFunction.apply(q, k, v, *lengths, bool(causal), scale, _training(q, k, v))


# ---------------------------------------------------------------------------
# norms of queries and keys with the rotation
# ---------------------------------------------------------------------------

def _norm_rope_shape(q, k, cos, positions, eps, interleaved, q_out, k_out):
    tokens, heads, head_dim = q.shape
    return sk.NormRopeShape(tokens, heads, k.shape[1], head_dim, 2 * cos.shape[1], int(interleaved), positions.element_size(), cos.shape[0], eps, _DTYPES[q.dtype],
                            _2(*q.stride()[:2]), _2(*k.stride()[:2]), _2(*q_out.stride()[:2]), _2(*k_out.stride()[:2]))


def _norm_rope_forward(q, k, wq, wk, cos, sin, positions, eps, interleaved, out=None):
    q_out, k_out = out if out is not None else (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
    if q.shape[0] > 0:
        shape = _norm_rope_shape(q, k, cos, positions, eps, interleaved, q_out, k_out)
        with _on(q.device):
            sk.check(sk.sk_norm_rope_fwd(shape, q, k, wq, wk, cos, sin, positions, q_out, k_out, _stream(q.device)))
    return q_out, k_out


class NormRopeFunction(torch.autograd.Function):
    """See ``head_norm_rope``, on q and k [tokens, heads, head_dim]; keeps its inputs and recomputes the norms."""

    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, eps, interleaved):
        q, k, wq, wk = _strided(q, -1), _strided(k, -1), _dense(wq), _dense(wk)
        ctx.save_for_backward(q, k, wq, wk, cos, sin, positions)
        ctx.eps, ctx.interleaved = eps, interleaved
        return _norm_rope_forward(q, k, wq, wk, cos, sin, positions, eps, interleaved)

    @staticmethod
    @_once
    def backward(ctx, dq_out, dk_out):
        q, k, wq, wk, cos, sin, positions = ctx.saved_tensors
        dq, dk, dwq, dwk = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, wq, wk))
        if q.shape[0] == 0:
            return dq, dk, dwq.zero_(), dwk.zero_(), None, None, None, None, None
        shape = _norm_rope_shape(q, k, cos, positions, ctx.eps, ctx.interleaved, q, k)
        dq_out, dk_out = _dense(dq_out), _dense(dk_out)
        with _on(q.device), _queueing:
            stream = _stream(q.device)
            ws = _workspace(q.device, stream, sk.sk_norm_rope_workspace_bytes(shape))
            sk.check(sk.sk_norm_rope_bwd(shape, q, k, wq, wk, cos, sin, positions, dq_out, dk_out, dq, dk, dwq, dwk, ws, ws.numel(), stream))
        if k.shape[1] == 0:
            dwk.zero_()
        return dq, dk, dwq, dwk, None, None, None, None, None


def head_norm_rope(q: torch.Tensor, k: torch.Tensor, q_weight: torch.Tensor, k_weight: torch.Tensor, cos: torch.Tensor,
                   sin: torch.Tensor, positions: torch.Tensor, *, eps: float = 1e-6, interleaved: bool = False, out=None):
    """RMS norm of every head of ``q [..., heads, head_dim]`` and ``k [..., kv_heads, head_dim]`` with weights ``[head_dim]``, then
    the rotation of its first features by the token's position: row ``positions[...]`` of the fp32 tables ``cos`` and ``sin
    [rows, rotated / 2]`` (positions outside the tables take their first or last row; the tables get no gradient).  Pairs are a feature and the one
    rotated / 2 further, or with ``interleaved`` neighbours.  Returns the two results, dense; outside of
    autograd they go into ``out = (q_out, k_out)`` if given (a cache's slots, or q and k themselves).

    Strided views are read in place.  head_dim: a multiple of 8 up to 256; the number of rotated features is a multiple of 8.
    """
    if out is None and _natively():
        if q.dim() == 3:
            both = _native.head_norm_rope(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved)
            if both is not None:
                return both
        elif q.dim() > 3 and positions.shape == q.shape[:-2] == k.shape[:-2]:
            both = _native.head_norm_rope(q.flatten(0, -3), k.flatten(0, -3), q_weight, k_weight, cos, sin, positions.reshape(-1), eps, interleaved)
            if both is not None:
                return both[0].view(q.shape), both[1].view(k.shape)
    _checked("head_norm_rope", q, q=q, k=k, q_weight=q_weight, k_weight=k_weight)
    D = q.shape[-1]
    if q.dim() < 3 or q.dim() != k.dim() or q.shape[:-2] != k.shape[:-2] or k.shape[-1] != D or q_weight.shape != (D,) or k_weight.shape != (D,):
        raise ValueError("head_norm_rope: shapes do not match (q [..., heads, head_dim], k [..., kv_heads, head_dim], weights [head_dim])")
    for name, t in (("cos", cos), ("sin", sin)):
        if t.dtype != torch.float32:
            raise TypeError(f"head_norm_rope: {name} has dtype {t.dtype}, not float32")
        if t.device != q.device:
            raise RuntimeError(f"head_norm_rope: {name} is on {t.device}, not on {q.device}")
        if torch.is_grad_enabled() and t.requires_grad:
            raise RuntimeError(f"head_norm_rope: {name} gets no gradient; pass it detached")
    if cos.dim() != 2 or cos.shape != sin.shape or 2 * cos.shape[1] > D or (cos.shape[0] == 0 and cos.shape[1] > 0):
        raise ValueError("head_norm_rope: cos and sin are [rows, rotated / 2], of one row at least")
    _integers("head_norm_rope", "positions", positions, q.device)
    if positions.shape != q.shape[:-2]:
        raise ValueError(f"head_norm_rope: positions have shape {tuple(positions.shape)}, not {tuple(q.shape[:-2])}")
    lead = q.shape[:-2]
    q3, k3 = (t if t.dim() == 3 else t.flatten(0, -3) for t in (q, k))
    args = (_dense(cos), _dense(sin), _dense(positions.reshape(-1)), float(eps), bool(interleaved))
    if out is not None:
        floating = (q, k, q_weight, k_weight)
        if torch.is_grad_enabled() and any(t.requires_grad for t in (*floating, *out)):
            raise RuntimeError("head_norm_rope: out is for calls without gradients")
        for t, like, name in zip(out, (q, k), ("q_out", "k_out")):
            _checked("head_norm_rope", q, **{name: t})
            if t.shape != like.shape:
                raise ValueError(f"head_norm_rope: {name} has shape {tuple(t.shape)}, not {tuple(like.shape)}")
        views = tuple(t if t.dim() == 3 else t.view(-1, *t.shape[-2:]) for t in out)
        if any(_strided(t, -1) is not t for t in views):
            raise ValueError("head_norm_rope: out needs heads of consecutive values at 16-byte boundaries")
        if torch.jit.is_tracing() or any(forward_ad.unpack_dual(t).tangent is not None for t in (*floating, cos, sin)):   # (as _training says)
            for t, result in zip(views, NormRopeFunction.apply(q3, k3, q_weight, k_weight, *args)):
                t.copy_(result)
        else:
            _norm_rope_forward(_strided(q3, -1), _strided(k3, -1), _dense(q_weight), _dense(k_weight), *args, views)
            torch.autograd.graph.increment_version([t for t in out if not t.is_inference()])   # (as a change in place: who has saved them finds out)
        return tuple(out)
    q_out, k_out = NormRopeFunction.apply(q3, k3, q_weight, k_weight, *args)
    return (q_out, k_out) if len(lead) == 1 else (q_out.view(q.shape), k_out.view(k.shape))


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------

def _embedding_forward(ids, table, scale):
    y = torch.empty((*ids.shape, table.shape[1]), dtype=table.dtype, device=table.device)
    if y.numel() > 0:
        with _on(table.device):
            sk.check(sk.sk_embedding_fwd(ids, ids.element_size(), table, y, ids.numel(), table.shape[0], table.shape[1], scale,
                                         _DTYPES[table.dtype], _stream(table.device)))
    return y


class EmbeddingFunction(torch.autograd.Function):
    """See ``embedding``; keeps the tokens only."""

    @staticmethod
    def forward(ctx, ids, table, scale):
        ctx.save_for_backward(ids)
        ctx.shape, ctx.scale = table.shape, scale
        return _embedding_forward(ids, _dense(table), scale)

    @staticmethod
    @_once
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        rows, width = ctx.shape
        dtable = torch.empty(ctx.shape, dtype=dy.dtype, device=dy.device)
        if ids.numel() == 0:
            return None, dtable.zero_(), None
        dy = _dense(dy)
        args = (ids.numel(), rows, width)
        with _on(dy.device), _queueing:
            stream, dt = _stream(dy.device), _DTYPES[dy.dtype]
            need = sk.sk_embedding_workspace_bytes(*args, dt)
            if need == _REFUSED:
                raise sk.SkError(sk.SK_ERR_UNSUPPORTED)
            ws = _workspace(dy.device, stream, need)
            sk.check(sk.sk_embedding_bwd(ids, ids.element_size(), dy, dtable, *args, ctx.scale, dt, ws, ws.numel(), stream))
        return None, dtable, None


def embedding(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """``scale * table[ids]``: ids int32 or int64 of any shape, table ``[rows, width]``, width a multiple of 8.  An id
    outside the table (a padding token's, say) gives zeros and no gradient.  The table's gradient is dense, added up in fp32 by
    sorted tokens, the same from run to run."""
    if _natively():
        y = _native.embedding(ids, table, scale)
        if y is not None:
            return y
    _checked("embedding", table, table=table)
    _integers("embedding", "ids", ids, table.device)
    if table.dim() != 2 or table.shape[0] == 0 or table.shape[1] == 0:
        raise ValueError("embedding: the table is [rows, width]")
    return EmbeddingFunction.apply(_dense(ids), table, float(scale))


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------

def _dropout(x, p, seed, offset, residual):
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if y.numel() > 0:
        with _on(x.device):
            sk.check(sk.sk_dropout(x, residual, y, x.numel(), p, seed, offset, _DTYPES[x.dtype], _stream(x.device)))
    return y


class DropoutFunction(torch.autograd.Function):
    """See ``dropout``; keeps nothing but the seed and the offset."""

    @staticmethod
    def forward(ctx, x, residual, p, seed, offset):
        ctx.args = p, seed, offset
        return _dropout(_dense(x), p, seed, offset, None if residual is None else _dense(residual))

    @staticmethod
    def backward(ctx, dy):
        dx = None
        if ctx.needs_input_grad[0]:
            dx = dropout(dy, *ctx.args)
        return dx, dy if ctx.needs_input_grad[1] else None, None, None, None


def dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, residual: torch.Tensor | None = None) -> torch.Tensor:
    """``x`` with each value dropped at rate ``p`` (to the nearest 2^-16) and the others scaled by 1 / (1 - p), plus ``residual``.

    What is dropped is a function of (seed, offset) and a value's place in x alone: the gradient draws it again.  Calls that are to
    differ take other offsets (or seeds), 64-bit unsigned numbers both; a graph that replays a call replays its numbers."""
    if _natively():
        y = _native.dropout(x, p, seed, offset, residual)
        if y is not None:
            return y
    _checked("dropout", x, x=x, residual=residual)
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"dropout: a rate of {p} is not between 0 and 1")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("dropout: seed and offset are 64-bit unsigned numbers")
    if residual is not None and residual.shape != x.shape:
        raise ValueError(f"dropout: residual has shape {tuple(residual.shape)}, not {tuple(x.shape)}")
    return DropoutFunction.apply(x, residual, float(p), int(seed), int(offset))


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------

def _rows_of(t: torch.Tensor, least: int = 0, most: int = 1 << 40) -> torch.Tensor:
    """t as a matrix of its rows, in place where they lie a stride of ``least`` to ``most`` elements apart that the library takes."""
    t = t.reshape(-1, t.shape[-1])
    if _strided(t, -1) is not t or (t.shape[0] > 1 and not least <= t.stride(0) <= most):
        return t.clone(memory_format=torch.contiguous_format)
    return t


def _row_stride(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _saved(t: torch.Tensor | None) -> torch.Tensor | None:
    """What was saved dense: hooks may have laid it out differently."""
    return None if t is None else _dense(t)


def _layer_norm_shape(x, residual, eps):
    return sk.LayerNormShape(x.shape[0], x.shape[1], eps, _DTYPES[x.dtype], _row_stride(x), x.shape[1] if residual is None else _row_stride(residual))


class LayerNormFunction(torch.autograd.Function):
    """See ``layer_norm``, on rows; keeps what was normed, each row's mean and deviation, and for the gradient of a weight what a sum's rounding to bf16 left off."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, eps, training):
        x2 = _rows_of(x)
        r2 = None if residual is None else _rows_of(residual)
        w, b = (None if t is None else _dense(t) for t in (weight, bias))
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        total = None if residual is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty((x2.shape[0], 2), dtype=torch.float32, device=x.device) if training else None
        rest = None
        if training and total is not None and weight is not None and weight.requires_grad and x.dtype == torch.bfloat16:
            rest = torch.empty((x2.shape[0], x2.shape[1] // 8), dtype=torch.int32, device=x.device)
        if x.numel() > 0:
            with _on(x.device):
                sk.check(sk.sk_layer_norm_fwd(_layer_norm_shape(x2, r2, eps), x2, r2, w, b, y, total, stats, _stream(x.device), rest))
        ctx.save_for_backward(x2 if total is None else total, w, stats, rest)
        ctx.shape, ctx.bias = x.shape, bias is not None
        ctx.set_materialize_grads(False)
        return y if total is None else (y, total)

    @staticmethod
    @_once
    def backward(ctx, dy, ds=None):
        x, *saved = ctx.saved_tensors
        x, (w, stats, rest) = _rows_of(x), map(_saved, saved)
        dx = torch.empty(ctx.shape, dtype=x.dtype, device=x.device)
        dw, db = (torch.empty(ctx.shape[-1], dtype=x.dtype, device=x.device) if there else None for there in (w is not None, ctx.bias))
        if x.numel() == 0:
            for t in (dw, db):
                if t is not None:
                    t.zero_()
            return dx, dw, db, dx if ctx.needs_input_grad[3] else None, None, None
        dy = torch.zeros_like(dx) if dy is None else _dense(dy)
        ds = None if ds is None else _dense(ds)
        shape = _layer_norm_shape(x, None, 0.0)
        with _on(x.device), _queueing:
            stream = _stream(x.device)
            ws = _workspace(x.device, stream, sk.sk_layer_norm_workspace_bytes(shape))
            sk.check(sk.sk_layer_norm_bwd(shape, x, w, stats, dy, ds, dx, dw, db, ws, ws.numel(), stream, rest))
        return dx, dw, db, dx if ctx.needs_input_grad[3] else None, None, None


def _vector(what: str, name: str, t: torch.Tensor | None, n: int):
    if t is not None and t.shape != (n,):
        raise ValueError(f"{what}: {name} has shape {tuple(t.shape)}, not [{n}]")


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, residual: torch.Tensor | None = None, *,
               eps: float = 1e-5):
    """Layer norm over the last dimension of ``x [..., width]``, times ``weight`` and plus ``bias [width]`` where they are given.

    With a ``residual`` (as x) the norm is of ``x + residual``, and the sum comes back too: ``(y, sum)``, the stream that a block goes on with.  What is
    normed is the sum before it is rounded.  (In bf16 its gradients are too, to four bits behind the rounding, where ``weight`` wants one; with a frozen weight they are
    those at the rounded sum.)  Rows of a strided matrix are read in place.  width: a multiple of 8 up to 32768.
    """
    if _natively():
        out = _native.layer_norm(x, weight, bias, residual, eps)
        if out is not None:
            return out
    _checked("layer_norm", x, x=x, weight=weight, bias=bias, residual=residual)
    if x.dim() == 0 or x.shape[-1] == 0:
        raise ValueError("layer_norm: x is [..., width]")
    for name, t in (("weight", weight), ("bias", bias)):
        _vector("layer_norm", name, t, x.shape[-1])
    if residual is not None and residual.shape != x.shape:
        raise ValueError(f"layer_norm: residual has shape {tuple(residual.shape)}, not {tuple(x.shape)}")
    return LayerNormFunction.apply(x, weight, bias, residual, float(eps), _training(x, weight, bias, residual))


# ---------------------------------------------------------------------------
# dense layers
# ---------------------------------------------------------------------------

_ACTIVATIONS = {None: sk.SK_ACT_NONE, "relu": sk.SK_ACT_RELU, "gelu": sk.SK_ACT_GELU, "gelu_tanh": sk.SK_ACT_GELU_TANH, "silu": sk.SK_ACT_SILU}


def _dense_shape(x, weight, residual, activation):
    return sk.DenseShape(x.shape[0], weight.shape[1], weight.shape[0], activation, _DTYPES[x.dtype], _row_stride(x),
                         weight.shape[0] if residual is None else _row_stride(residual))


def _dense_workspace(shape, backward, device, stream):
    need = sk.sk_dense_workspace_bytes(shape, backward)
    if need == _REFUSED:
        raise sk.SkError(sk.SK_ERR_UNSUPPORTED)
    return _workspace(device, stream, need)


class LinearFunction(torch.autograd.Function):
    """See ``linear``; keeps x, the weight, and with an activation what goes into it."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, activation, training):
        x2, w = _rows_of(x, x.shape[-1], 1 << 20), _dense(weight)
        b = None if bias is None else _dense(bias)
        r2 = None if residual is None else _rows_of(residual, residual.shape[-1], 1 << 20)
        y = torch.empty((*x.shape[:-1], w.shape[0]), dtype=x.dtype, device=x.device)
        z = torch.empty((x2.shape[0], w.shape[0]), dtype=x.dtype, device=x.device) if training and activation != sk.SK_ACT_NONE else None
        if y.numel() > 0:
            shape = _dense_shape(x2, w, r2, activation)
            with _on(x.device), _queueing:
                stream = _stream(x.device)
                ws = _dense_workspace(shape, 0, x.device, stream)
                sk.check(sk.sk_dense_fwd(shape, x2, w, b, r2, y, z, ws, ws.numel(), stream))
        ctx.save_for_backward(x2, w, z)
        ctx.shape, ctx.activation, ctx.bias = x.shape, activation, bias is not None
        return y

    @staticmethod
    @_once
    def backward(ctx, dy):
        x, w, z = ctx.saved_tensors
        x, w, z = _rows_of(x, x.shape[-1], 1 << 20), _saved(w), _saved(z)
        wanted = ctx.needs_input_grad
        dx = torch.empty(ctx.shape, dtype=x.dtype, device=x.device) if wanted[0] else None
        dw = torch.empty(w.shape, dtype=x.dtype, device=x.device) if wanted[1] else None
        db = torch.empty(w.shape[0], dtype=x.dtype, device=x.device) if wanted[2] else None
        if x.numel() == 0:
            for t in (dw, db):
                if t is not None:
                    t.zero_()
        elif any(wanted[:3]):
            d = _dense(dy)
            shape = _dense_shape(x, w, None, ctx.activation)
            with _on(x.device), _queueing:
                stream = _stream(x.device)
                ws = _dense_workspace(shape, 1, x.device, stream)
                sk.check(sk.sk_dense_bwd(shape, x, w, z, d, dx, dw, db, ws, ws.numel(), stream))
        return dx, dw, db, dy if wanted[3] else None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, residual: torch.Tensor | None = None, *,
           activation: str | None = None) -> torch.Tensor:
    """``activation(x @ weight.t() + bias) + residual``: a layer that stays dense, ``x [..., in]``, ``weight [out, in]`` and ``bias [out]`` as
    ``torch.nn.Linear`` has them, ``residual [..., out]``.

    ``activation``: None, "relu", "gelu" (z Phi(z)), "gelu_tanh" (its approximation by tanh) or "silu".  A backward pass has what goes into
    it, in the tensors' type.  Rows of strided matrices x and residual are read in place, of other layouts that are not dense from a copy.  in and out: multiples of 8.
    """
    if activation not in _ACTIVATIONS:
        raise ValueError(f"linear: no activation {activation!r}; there are {', '.join(map(repr, _ACTIVATIONS))}")
    act = _ACTIVATIONS[activation]
    if _natively():
        y = _native.dense_layer(x, weight, bias, residual, act)
        if y is not None:
            return y
    _checked("linear", x, x=x, weight=weight, bias=bias, residual=residual)
    if x.dim() == 0 or weight.dim() != 2 or weight.numel() == 0 or x.shape[-1] != weight.shape[1]:
        raise ValueError("linear: shapes do not match (x [..., in], weight [out, in])")
    _vector("linear", "bias", bias, weight.shape[0])
    if residual is not None and residual.shape != (*x.shape[:-1], weight.shape[0]):
        raise ValueError(f"linear: residual has shape {tuple(residual.shape)}, not {(*x.shape[:-1], weight.shape[0])}")
    return LinearFunction.apply(x, weight, bias, residual, act, _training(x, weight, bias, residual))


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

def _distill_shape(z, ids, labels, temperature, label_weight):
    return sk.DistillShape(z.shape[0], z.shape[1], _row_stride(z), ids.shape[-1], ids.element_size(), 8 if labels is None else labels.element_size(),
                           temperature, label_weight, _DTYPES[z.dtype])


def _logit_rows(z: torch.Tensor) -> torch.Tensor:
    return z if z.stride(1) == 1 and z.stride(0) <= 1 << 40 else z.clone(memory_format=torch.contiguous_format)


class DistillationFunction(torch.autograd.Function):
    """See ``distillation_loss``; keeps its inputs and each row's largest logit and sums."""

    @staticmethod
    def forward(ctx, logits, teacher_logits, teacher_ids, labels, temperature, label_weight, training):
        z = logits.reshape(-1, logits.shape[-1])
        z = _logit_rows(z)
        loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
        stats = torch.empty((z.shape[0], 8), dtype=torch.float32, device=logits.device) if training else None
        if z.shape[0] > 0:
            shape = _distill_shape(z, teacher_ids, labels, temperature, label_weight)
            with _on(logits.device):
                sk.check(sk.sk_distill_fwd(shape, z, teacher_logits, teacher_ids, labels, loss, stats, _stream(logits.device)))
        ctx.save_for_backward(z, teacher_logits, teacher_ids, labels, stats)
        ctx.shape, ctx.args = logits.shape, (temperature, label_weight)
        return loss

    @staticmethod
    @_once
    def backward(ctx, dloss):
        z, *rest = ctx.saved_tensors
        z, (t, ids, labels, stats) = _logit_rows(z), map(_saved, rest)
        dz = torch.empty(ctx.shape, dtype=z.dtype, device=z.device)
        if z.shape[0] > 0:
            with _on(z.device):
                sk.check(sk.sk_distill_bwd(_distill_shape(z, ids, labels, *ctx.args), z, t, ids, labels, stats, _dense(dloss), dz, _stream(z.device)))
        return dz, None, None, None, None, None, None


def distillation_loss(logits: torch.Tensor, teacher_logits: torch.Tensor, teacher_ids: torch.Tensor, labels: torch.Tensor | None = None, *,
                      temperature: float = 1.0, label_weight: float = 0.0) -> torch.Tensor:
    """The loss of every row of ``logits [..., vocabulary]`` (fp32 ``[...]``; sum or average it as the program does) against a teacher's largest
    logits ``teacher_logits [..., top]`` at the places ``teacher_ids [..., top]``, and against ``labels [...]``:

        (1 - label_weight) temperature^2 KL(p || q) + label_weight (log sum exp z - z_label)

    with p the softmax of the teacher's entries over the temperature and q that of all of a row's logits.  An entry whose id is outside the vocabulary or
    whose logit is -infinity is not there (a list that ends early), an id that is named twice has both entries; a row without an entry has no first
    term, one whose label is outside the vocabulary no second.  The logits alone get a gradient.  Ids and labels are int32 or int64.  Any size of
    vocabulary.  Dense logits and the rows of a strided matrix are read in place; others (a part of the positions of each of many sequences, ``logits[:, a:b]``)
    are copied first, and the copy is kept for the backward pass.  Made for lists of up to some hundred entries: past about a thousand the gradient's time
    grows with the square of ``top``.
    """
    if _natively():
        loss = _native.distillation_loss(logits, teacher_logits, teacher_ids, labels, temperature, label_weight)
        if loss is not None:
            return loss
    what = "distillation_loss"
    _checked(what, logits, logits=logits, teacher_logits=teacher_logits)
    if logits.dim() == 0 or logits.shape[-1] == 0 or teacher_logits.dim() != logits.dim() or teacher_logits.shape[:-1] != logits.shape[:-1]:
        raise ValueError(f"{what}: shapes do not match (logits [..., vocabulary], teacher_logits [..., top])")
    if torch.is_grad_enabled() and teacher_logits.requires_grad:
        raise RuntimeError(f"{what}: teacher_logits get no gradient; pass them detached")
    _integers(what, "teacher_ids", teacher_ids, logits.device)
    if teacher_ids.shape != teacher_logits.shape:
        raise ValueError(f"{what}: teacher_ids have shape {tuple(teacher_ids.shape)}, not {tuple(teacher_logits.shape)}")
    if labels is not None:
        _integers(what, "labels", labels, logits.device)
        if labels.shape != logits.shape[:-1]:
            raise ValueError(f"{what}: labels have shape {tuple(labels.shape)}, not {tuple(logits.shape[:-1])}")
        labels = _dense(labels)
    if not 0.0 < temperature < float("inf"):
        raise ValueError(f"{what}: a temperature of {temperature}")
    if not 0.0 <= label_weight <= 1.0:
        raise ValueError(f"{what}: a label_weight of {label_weight} is not between 0 and 1")
    return DistillationFunction.apply(logits, _dense(teacher_logits), _dense(teacher_ids), labels, float(temperature), float(label_weight), _training(logits))
