"""Group norm with an activation, channels last (``qta_group_norm*`` of ``include/qta.h``). Argument marshalling only."""
from __future__ import annotations

import ctypes

import torch

from .decay import _once
from .dense import _call, _new, _no_tangents, _tokens, _workspace
from .qta import _DTYPES, _SIGS, _dtype_code

_P, _I, _F, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_int64
_ACTS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}


class GroupNormArgs(ctypes.Structure):
    _fields_ = [("x", _P), ("weight", _P), ("bias", _P), ("B", _I), ("N", _I), ("C", _I), ("groups", _I), ("dtype", _I),
                ("param_dtype", _I), ("x_batch", _L), ("x_token", _L), ("per_token", _I), ("act", _I), ("eps", _F)]


_SIGS.update({
    "qta_group_norm_workspace_bytes": ([_P], ctypes.c_size_t),
    "qta_group_norm": ([_P, _P, _P, _P, ctypes.c_size_t, _P], _I),
    "qta_group_norm_backward_workspace_bytes": ([_P], ctypes.c_size_t),
    "qta_group_norm_backward": ([_P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P], _I),
})


def _norm_args(x, groups, weight, bias, eps, act, per_token):
    if not isinstance(x, torch.Tensor):
        raise TypeError("x must be a tensor")
    if x.dim() not in (3, 4):
        raise ValueError(f"x must be [B, N, C] or [B, H, W, C], got shape {tuple(x.shape)}")
    B, N, _, C, xb, xn, _ = _tokens(x.unsqueeze(-2), "x")
    code = _DTYPES.get(x.dtype)
    if code is None:
        _dtype_code(x)
    if not isinstance(groups, int) or isinstance(groups, bool) or groups <= 0 or C % groups:
        raise ValueError(f"groups must be a positive divisor of {C} channels, got {groups}")
    if act not in _ACTS:
        raise ValueError(f"act must be one of 'none', 'relu', 'silu' and 'gelu', got {act!r}")
    if not 0.0 <= eps < float("inf"):
        raise ValueError(f"eps must be at least 0, got {eps}")
    params = [t for t in (weight, bias) if t is not None]
    for t in params:
        if not isinstance(t, torch.Tensor):
            raise TypeError("weight and bias must be tensors")
        if t.dtype not in (torch.float32, x.dtype) or t.dtype is not params[0].dtype or t.device != x.device or t.shape != (C,) \
                or not t.is_contiguous():
            raise ValueError(f"weight and bias must be contiguous {(C,)}, both torch.float32 or {x.dtype}, on {x.device}")
    return GroupNormArgs(x.data_ptr(), None if weight is None else weight.data_ptr(), None if bias is None else bias.data_ptr(),
                         B, N, C, groups, code, _DTYPES[params[0].dtype] if params else 0, xb, xn, bool(per_token), _ACTS[act],
                         eps)


def _norm_forward(args, x, keep):
    y = _new(x)
    stats = torch.empty((args.B, args.groups, 2), dtype=torch.float32, device=x.device) if keep and not args.per_token else None
    if y.numel():
        ws, nbytes = (None, 0) if args.per_token else _workspace("qta_group_norm_workspace_bytes", args, x)
        _call("qta_group_norm", x, ctypes.byref(args), y.data_ptr(), None if stats is None else stats.data_ptr(),
              None if ws is None else ws.data_ptr(), nbytes)
    return y, stats


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act, per_token):
        ctx.args = _norm_args(x, groups, weight, bias, eps, act, per_token)
        ctx.how, ctx.stride = (groups, eps, act, per_token), x.stride()
        y, stats = _norm_forward(ctx.args, x, True)
        ctx.save_for_backward(x, weight, bias, stats)
        return y

    @_once
    def backward(ctx, dy):
        x, weight, bias, stats = ctx.saved_tensors
        dy = dy.contiguous()
        groups, eps, act, per_token = ctx.how
        # the forward's checks hold as long as what was kept came back as it was laid out, at whatever address
        if x.stride() == ctx.stride:
            args = GroupNormArgs.from_buffer_copy(ctx.args)
            args.x = x.data_ptr()
            args.weight = None if weight is None else weight.data_ptr()
            args.bias = None if bias is None else bias.data_ptr()
        else:
            args = _norm_args(x, groups, weight, bias, eps, act, per_token)
        dx = torch.empty_like(dy)
        dw = torch.empty_like(weight) if weight is not None and ctx.needs_input_grad[1] else None
        db = torch.empty_like(bias) if bias is not None and ctx.needs_input_grad[2] else None
        if dx.numel():
            ws, n = None, 0
            if not per_token or dw is not None or db is not None:
                ws, n = _workspace("qta_group_norm_backward_workspace_bytes", args, x)
            _call("qta_group_norm_backward", x, ctypes.byref(args), None if stats is None else stats.data_ptr(), dy.data_ptr(),
                  dx.data_ptr(), None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                  None if ws is None else ws.data_ptr(), n)
        else:
            for t in (dw, db):
                if t is not None:
                    t.zero_()
        return dx, dw, db, None, None, None, None


def group_norm(x, groups, weight=None, bias=None, *, eps=1e-5, act="none", per_token=False):
    """Group norm with an activation, channels last: ``act(weight * (x - mean) / sqrt(var + eps) + bias)``. x ``[B, N, C]`` or a map
    ``[B, H, W, C]``, fp32 or bf16; mean and variance are those of each of the ``groups`` groups of C / groups neighbouring channels
    over the tokens of a batch element, or with ``per_token`` over one token (which causal models need, and the heads of an
    attention's output ``out.flatten(-2)`` with a group for each). ``weight``, ``bias``: ``[C]``, fp32 or x's type, or None.
    ``act``: "none", "relu", "silu" or "gelu" (by the error function). Differentiable in x, weight and bias (reverse mode).

    A NaN or an infinity makes NaNs of its group's results (with ``per_token`` of its token's group), and reaches no other group."""
    _no_tangents(x, weight, bias)
    if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in (x, weight, bias)):
        return _GroupNorm.apply(x, weight, bias, groups, eps, act, per_token)
    return _norm_forward(_norm_args(x, groups, weight, bias, eps, act, per_token), x, False)[0]
