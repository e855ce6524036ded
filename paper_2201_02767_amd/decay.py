"""Linear attention with a decay for each head (``qta_decay_attn*`` of ``include/qta.h``).

Argument marshalling only, like ``dense.py``, whose layouts hold here too: sequences ``[B, N, heads, d]``, or maps
``[B, H, W, heads, d]`` read row by row, fp32 or bf16, channels of a head contiguous, tensors that start on 16 bytes with strides
that are multiples of 16 bytes.
"""
from __future__ import annotations

import ctypes

import torch

from .dense import _call, _new, _no_tangents, _int32, _tokens, _workspace
from .qta import _DTYPES, _SIGS, _dtype_code, _scale

_P, _I, _F, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_int64


class DecayAttnArgs(ctypes.Structure):
    _fields_ = [("q", _P), ("k", _P), ("v", _P), ("log_decay", _P), ("state", _P), ("B", _I), ("heads", _I), ("N", _I),
                ("dk", _I), ("dv", _I), ("dtype", _I), ("q_batch", _L), ("q_token", _L), ("q_head", _L), ("k_batch", _L),
                ("k_token", _L), ("k_head", _L), ("v_batch", _L), ("v_token", _L), ("v_head", _L), ("lens", _P),
                ("scale", _F)]


_SIGS.update({
    "qta_decay_attn_workspace_bytes": ([_P], ctypes.c_size_t),
    "qta_decay_attn": ([_P, _P, _P, _P, ctypes.c_size_t, _P], _I),
    "qta_decay_attn_backward_workspace_bytes": ([_P], ctypes.c_size_t),
    "qta_decay_attn_backward": ([_P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P], _I),
})


def _state(t, name, like, shape):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dtype is not torch.float32 or t.device != like.device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous torch.float32 {tuple(shape)} on {like.device}")
    return t.data_ptr()


def _decay_args(q, k, v, log_decay, scale, lens, state):
    """The library's arguments, and the shapes of the output and of a state."""
    B, N, heads, dk, qb, qn, qh = _tokens(q, "q")
    *ks, kb, kn, kh = _tokens(k, "k", q)
    *vs, dv, vb, vn, vh = _tokens(v, "v", q)
    code = _DTYPES.get(q.dtype)
    if code is None:
        _dtype_code(q)
    if ks != [B, N, heads, dk] or vs != [B, N, heads] or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    if not isinstance(log_decay, torch.Tensor):
        raise TypeError("log_decay must be a tensor")
    if log_decay.dtype is not torch.float32 or log_decay.device != q.device or log_decay.shape != (heads,) \
            or not log_decay.is_contiguous():
        raise ValueError(f"log_decay must be contiguous torch.float32 {(heads,)} on {q.device}")
    if scale is not None and not 2.0 ** -64 <= scale <= 2.0 ** 64:        # (zero and below mean 1/sqrt(dk) to the library)
        raise ValueError(f"scale must be positive, from 2^-64 to 2^64, got {scale}")
    shape = (B, heads, dk, dv)
    args = DecayAttnArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
                         None if state is None else _state(state, "state", q, shape), B, heads, N, dk, dv, code,
                         qb, qn, qh, kb, kn, kh, vb, vn, vh, None if lens is None else _int32(lens, "lens", q, (B,)),
                         _scale(scale))
    return args, (*q.shape[:-1], dv), shape


def _decay_forward(args, shape, q, state, state_out):
    out = q.new_empty(shape)
    if out.numel() == 0 or args.dk == 0:
        out.zero_()
        if state_out is not None and state_out is not state:
            state_out.copy_(state) if state is not None else state_out.zero_()
        return out
    ws, nbytes = _workspace("qta_decay_attn_workspace_bytes", args, q)
    _call("qta_decay_attn", q, ctypes.byref(args), out.data_ptr(), None if state_out is None else state_out.data_ptr(),
          None if ws is None else ws.data_ptr(), nbytes)
    return out


def _decay_backward(args, q, k, v, dout, dstate_out, dstate):
    grads = [_new(t) for t in (q, k, v)]
    if dout.numel() == 0 or args.dk == 0:
        if dstate is not None:
            dstate.copy_(dstate_out) if dstate_out is not None else dstate.zero_()
        return tuple(g.zero_() for g in grads)
    ws, nbytes = _workspace("qta_decay_attn_backward_workspace_bytes", args, q)
    _call("qta_decay_attn_backward", q, ctypes.byref(args), dout.data_ptr(),
          None if dstate_out is None else dstate_out.data_ptr(), *[g.data_ptr() for g in grads],
          None if dstate is None else dstate.data_ptr(), None if ws is None else ws.data_ptr(), nbytes)
    return tuple(grads)


def decay_attn(q, k, v, log_decay, *, scale=None, lens=None, state=None, return_state=False, state_out=None):
    """Linear attention with a decay for each head: with g = ``log_decay[head]``,

        S_t = exp(g) S_{t-1} + k_t v_t^T,    out_t = scale * S_t^T q_t.

    q, k ``[B, N, heads, dk]``, v ``[B, N, heads, dv]`` (or maps ``[B, H, W, ..]``, row by row), dk and dv 32, 64 or 128;
    ``log_decay`` fp32 ``[heads]``, at most 0 (a positive one grows, and is right while exp(g N) stays far from fp32's largest: g N below
    80). Returns ``[B, N, heads, dv]``; with ``return_state`` or ``state_out`` a pair of
    it and the state behind the last token, fp32 ``[B, heads, dk, dv]``.

    ``state``: the state before the first token (None: zeros), so that a call goes on where another one ended: prompts
    in pieces, then single tokens, which are read and written through the state alone. ``state_out``: where the new state goes;
    may be ``state`` itself. ``lens`` (int32 ``[B]``): tokens of each batch element; what lies behind them is never used, and gives
    zeros. ``scale``: positive, or None for 1/sqrt(dk).

    Tokens before the lengths and the state have to be finite: in calls of more than 16 tokens a NaN or an infinity makes NaNs of up to 31
    *earlier* results of its head as well."""
    _no_tangents(q, k, v, log_decay, state)
    args, shape, sshape = _decay_args(q, k, v, log_decay, scale, lens, state)
    given = state_out is not None
    if given:
        _state(state_out, "state_out", q, sshape)
        if state_out.requires_grad and torch.is_grad_enabled():
            raise ValueError("state_out requires gradients: decay_attention has them")
        if state_out is not state and state is not None and state_out.numel() and state_out.data_ptr() != state.data_ptr() \
                and abs(state_out.data_ptr() - state.data_ptr()) < 4 * state.numel():
            raise ValueError("state_out must be state itself or lie apart from it")
    elif return_state:
        state_out = torch.empty(sshape, dtype=torch.float32, device=q.device)
    out = _decay_forward(args, shape, q, state, state_out)
    if given:
        torch.autograd.graph.increment_version((state_out,))    # (for what autograd may have kept of it)
    return out if state_out is None else (out, state_out)


def decay_attn_backward(q, k, v, log_decay, dout, *, scale=None, lens=None, state=None, dstate_out=None):
    """Gradients (dq, dk, dv, dstate) of ``decay_attn`` for the upstream gradients ``dout`` and ``dstate_out`` (of the state behind
    the last token; None: zeros), the other arguments the same. ``dstate`` is None without a ``state``."""
    args, shape, sshape = _decay_args(q, k, v, log_decay, scale, lens, state)
    if dout.dtype is not q.dtype or dout.device != q.device or dout.shape != shape or not dout.is_contiguous():
        raise ValueError(f"dout must be contiguous {q.dtype} {tuple(shape)} on {q.device}")
    if dstate_out is not None:
        _state(dstate_out, "dstate_out", q, sshape)
    dstate = None if state is None else torch.empty_like(state)
    return (*_decay_backward(args, q, k, v, dout, dstate_out, dstate), dstate)


def _once(backward):
    """A Function's backward whose results are not to be differentiated again. (The decorator for that takes 7 us a call: only where
    a graph of the backward is asked for.)"""
    guarded = torch.autograd.function.once_differentiable(backward)
    return staticmethod(lambda ctx, *grads: guarded(ctx, *grads) if torch.is_grad_enabled() else backward(ctx, *grads))


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, state, log_decay, scale, lens, return_state):
        ctx.set_materialize_grads(False)
        ctx.args, ctx.shape, sshape = _decay_args(q, k, v, log_decay, scale, lens, state)
        last = torch.empty(sshape, dtype=torch.float32, device=q.device) if return_state else None
        out = _decay_forward(ctx.args, ctx.shape, q, state, last)
        ctx.strides, ctx.scale = (q.stride(), k.stride(), v.stride()), scale
        ctx.save_for_backward(q, k, v, state, log_decay, lens)
        return (out, last) if return_state else out

    @_once
    def backward(ctx, dout, dstate_out=None):
        q, k, v, state, log_decay, lens = ctx.saved_tensors
        if dout is None and dstate_out is None:
            return (None,) * 8
        dout = torch.zeros(ctx.shape, dtype=q.dtype, device=q.device) if dout is None else dout.contiguous()
        dout = dout.clone() if dout.data_ptr() % 16 else dout
        if dstate_out is not None:
            dstate_out = dstate_out.contiguous()
            dstate_out = dstate_out.clone() if dstate_out.data_ptr() % 16 else dstate_out
        dstate = torch.empty_like(state) if state is not None and ctx.needs_input_grad[3] else None
        # the forward's checks hold as long as what was kept came back as it was laid out, at whatever address
        if (q.stride(), k.stride(), v.stride()) == ctx.strides and (state is None or state.is_contiguous()):
            args = DecayAttnArgs.from_buffer_copy(ctx.args)
            args.q, args.k, args.v, args.log_decay = q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr()
            args.state = None if state is None else state.data_ptr()
            args.lens = None if lens is None else lens.data_ptr()
        else:
            args = _decay_args(q, k, v, log_decay, ctx.scale, lens, state)[0]
        return (*_decay_backward(args, q, k, v, dout, dstate_out, dstate), dstate, None, None, None, None)


def decay_attention(q, k, v, log_decay, *, scale=None, lens=None, state=None, return_state=False):
    """Differentiable ``decay_attn`` (reverse mode): gradients of q, k, v and state, from those of the output and of the returned
    state. ``log_decay`` that requires gradients is refused. Upstream gradients have to be finite like the tokens: what is not reaches
    up to 31 gradients on the other side of its token too."""
    _no_tangents(q, k, v, log_decay, state)
    if not (torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in (q, k, v, log_decay, state))):
        return decay_attn(q, k, v, log_decay, scale=scale, lens=lens, state=state, return_state=return_state)
    if getattr(log_decay, "requires_grad", False):
        raise ValueError("log_decay gets no gradient: detach it")
    return _DecayAttention.apply(q, k, v, state, log_decay, scale, lens, bool(return_state))
