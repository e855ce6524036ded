"""Rotary positions and differential attention (``qta_rotary`` and ``qta_diff_attn*`` of ``include/qta.h``).

Argument marshalling only, like ``qta.py``. Tokens come as sequences ``[B, N, heads, d]`` or as maps
``[B, H, W, heads, d]`` (fp32 or bf16, on a GPU); views are taken as they are as long as the channels of a head are
contiguous and, on a map, its rows follow each other at one distance. Attention also needs tensors that start on 16 bytes
with all strides multiples of 16 bytes; rotary positions take any.
"""
from __future__ import annotations

import ctypes
import math

import torch
from torch.autograd import forward_ad

from .qta import _DTYPES, _SIGS, _check, _dtype_code, _scale, lib

_INT_MAX = 2 ** 31 - 1

_P, _I, _F, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_int64


class RotaryTensor(ctypes.Structure):
    _fields_ = [("x", _P), ("y", _P), ("heads", _I), ("x_batch", _L), ("x_token", _L), ("x_head", _L),
                ("y_batch", _L), ("y_token", _L), ("y_head", _L)]


class DiffAttnArgs(ctypes.Structure):
    _fields_ = [("q", _P), ("k", _P), ("v", _P), ("lam", _P), ("B", _I), ("heads", _I), ("kv_heads", _I), ("Nq", _I),
                ("Nk", _I), ("d", _I), ("dtype", _I), ("lam_dtype", _I), ("q_batch", _L), ("q_token", _L),
                ("q_head", _L), ("k_batch", _L), ("k_token", _L), ("k_head", _L), ("v_batch", _L), ("v_token", _L),
                ("v_head", _L), ("lam_batch", _L), ("lam_token", _L), ("lam_head", _L), ("lens", _P), ("q_pos", _P),
                ("causal", _I), ("scale", _F)]


_SIGS.update({
    "qta_rotary": ([_P, _I, _I, _I, _I, _I, _I, _I, _I, _I, _I, _P, _P, _L, _I, _F, _P], _I),
    "qta_diff_attn_workspace_bytes": ([_P], ctypes.c_size_t),
    "qta_diff_attn": ([_P, _P, _P, _P, _P, ctypes.c_size_t, _P], _I),
    "qta_diff_attn_backward_workspace_bytes": ([_P], ctypes.c_size_t),
    "qta_diff_attn_backward": ([_P, _P, _P, _P, _P, _P, _P, _P, _I, _P, ctypes.c_size_t, _P], _I),
})


def _tokens(t, name, like=None):
    """(B, N, heads, channels, and the strides of the first three) of a sequence or a map."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU")
    if like is not None and (t.dtype is not like.dtype or t.device != like.device):
        raise ValueError(f"{name} must be {like.dtype} on {like.device}, got {t.dtype} on {t.device}")
    shape, st = t.shape, t.stride()
    if len(shape) not in (4, 5):
        raise ValueError(f"{name} must be [B, N, heads, d] or [B, H, W, heads, d], got shape {tuple(shape)}")
    if shape[-1] > 1 and st[-1] != 1:
        raise ValueError(f"the channels of {name} must be contiguous")
    if len(shape) == 4:
        N, token = shape[1], st[1]
    else:
        N, token = shape[1] * shape[2], st[2] if shape[2] > 1 else st[1]
        if shape[1] > 1 and shape[2] > 1 and st[1] != shape[2] * st[2]:
            raise ValueError(f"the rows of the map {name} must follow each other at one distance")
    if t.numel() > _INT_MAX and max(shape[0], N, *shape[-2:]) > _INT_MAX:       # (ctypes would wrap them)
        raise ValueError(f"{name} has shape {tuple(shape)}: sizes are below 2^31")
    # (the stride of an axis of one entry is never taken, and may be anything)
    return (shape[0], N, shape[-2], shape[-1], st[0] if shape[0] > 1 else 0, token if N > 1 else 0,
            st[-2] if shape[-2] > 1 else 0)


def _int32(t, name, like, *shapes):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dtype is not torch.int32 or t.device != like.device or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous torch.int32 on {like.device}")
    if t.shape not in shapes:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {' or '.join(str(s) for s in shapes)}")
    return t.data_ptr()


def _raw_stream(dev):
    """The current stream (torch.cuda.current_stream: 2 us a call). A torch without GPUs does not have the name."""
    return torch._C._cuda_getCurrentRawStream(dev)


def _call(name, t, *args):
    """The library's function on t's device, which is made current for it, and on torch's current stream there."""
    dev = t.get_device()
    if dev == torch.cuda.current_device():
        status = getattr(lib(), name)(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            status = getattr(lib(), name)(*args, _raw_stream(dev))
    if status:
        _check(name, status)


def _no_tangents(*tensors):
    """Refuses dual tensors, whose derivative a result of the library's would not carry on."""
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(      # (outside every dual level none is dual: 0.1 us a call)
            isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError("rotary positions and differential attention have no forward-mode derivatives")


def _new(t):
    """A contiguous tensor like t."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


# ------------------------------------------------------------------------------------------------
# rotary positions
# ------------------------------------------------------------------------------------------------

def rotary_freqs(rot, *, theta=10000.0, axes=1, factor=1.0, trained=None, low=1.0, high=32.0, device=None):
    """Frequencies for ``rotary``: fp64 ``[rot/2]``, theta^(-j/n) for the n = rot/2/axes pairs of each axis.

    ``factor`` > 1 stretches the positions to a longer context: every frequency divided by it, or, with ``trained``
    (the context length in training), only those that turn less than ``low`` times in that length; those that turn
    more than ``high`` times stay, and between the two the change is blended linearly in the number of turns."""
    if rot <= 0 or axes not in (1, 2) or rot % (2 * axes) != 0:
        raise ValueError(f"rot must be a positive multiple of {2 * axes} for {axes} axes, got {rot}")
    if theta <= 0 or factor < 1.0 or high <= low:
        raise ValueError("theta > 0, factor >= 1 and high > low are needed")
    n = rot // 2 // axes
    f = float(theta) ** (-torch.arange(n, dtype=torch.float64) / n)
    if trained is not None:
        keep = ((f * float(trained) / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    else:
        f = f / factor
    return f.repeat(axes).to(device) if device is not None else f.repeat(axes)


def _rotary_args(xs, freqs, pos, axes, interleaved, scale, start):
    """A call's arguments, checked: sizes and strides of the tensors, and the rest but for pointers and the direction."""
    x = xs[0]
    if not -_INT_MAX <= start <= _INT_MAX:              # (and start + N as well: the library's check)
        raise ValueError(f"start must be below 2^31, got {start}")
    shapes = [_tokens(t, n, x) for t, n in zip(xs, ("x", "k"))]
    B, N, _, d = shapes[0][:4]
    for t, s in zip(xs[1:], shapes[1:]):
        if t.shape[:-2] != x.shape[:-2] or s[3] != d:
            raise ValueError(f"k has shape {tuple(t.shape)}, x {tuple(x.shape)}: only the heads may differ")
    code = _DTYPES.get(x.dtype)
    if code is None:
        _dtype_code(x)
    axes = (2 if x.dim() == 5 else 1) if axes is None else axes
    if not isinstance(freqs, torch.Tensor):
        raise TypeError("freqs must be a tensor")
    if freqs.dtype is not torch.float64 or freqs.device != x.device or freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError(f"freqs must be a contiguous torch.float64 vector on {x.device}")
    pos_batch = 0
    if pos is not None:
        if start != 0:
            raise ValueError("start goes with positions that are counted, not with given ones")
        _int32(pos, "pos", x, *(((N,), (B, N)) if axes == 1 else ((N, 2), (B, N, 2))))
        pos_batch = N * axes if pos.dim() > axes else 0
    elif axes == 2:
        if x.dim() != 5:
            raise ValueError("two axes need a map or given positions")
        if start != 0:
            raise ValueError("start goes with the positions of a sequence, not with rows and columns")
    return shapes, (B, N, d, 2 * freqs.numel(), axes, x.shape[2] if x.dim() == 5 else 0, interleaved), code, \
        (pos_batch, start, scale)


def _turn(xs, ys, freqs, pos, args, inverse, x_dense=False, y_dense=True):
    """The launch. ``x_dense``, ``y_dense``: xs or ys are contiguous, whatever strides the checked tensors had."""
    shapes, sizes, code, rest = args
    B, N, d = sizes[:3]
    if B == 0 or N == 0 or d == 0:
        return
    table = (RotaryTensor * len(xs))()
    for e, t, y, (_, _, heads, _, *st) in zip(table, xs, ys, shapes):
        dense = (N * heads * d, heads * d, d)
        e.__init__(t.data_ptr(), y.data_ptr(), heads, *(dense if x_dense else st), *(dense if y_dense else st))
    _call("qta_rotary", xs[0], ctypes.addressof(table), len(xs), *sizes, inverse, code, freqs.data_ptr(),
          None if pos is None else pos.data_ptr(), *rest)


def _extent(axes, run):
    """Elements from the first to behind the last of runs that lie at the axes (stride, entries), where no two runs meet as
    each axis steps over all that is inside it; None where an axis does not."""
    for stride, n in sorted(axes):
        if stride < run:
            return None
        run += stride * (n - 1)
    return run


def _apart(xs, shapes):
    """Whether no two heads of the tokens of one or two tensors (and their ``_tokens``) share an element. (In place each is
    read and written by threads of its own.)"""
    size, at = xs[0].element_size(), [t.data_ptr() for t in xs]
    lo, hi = (0, 1) if at[0] <= at[-1] else (1, 0)
    gap = (at[-1] - at[0]) * (hi - lo)
    # tokens, and heads within them, one after the other: the usual layouts, quickly
    spans = []
    for B, N, heads, d, b, n, h in shapes:
        token = (heads - 1) * h + d
        row = (N - 1) * n + token
        if (heads > 1 and h < d) or (N > 1 and n < token) or (B > 1 and b < row):
            break
        spans.append((token, (B - 1) * b + row))
    else:
        if len(xs) == 1 or gap >= spans[lo][1] * size:
            return True
        B, N, _, _, b, n, _ = shapes[0]
        both = gap + spans[hi][0] * size                # a token of both, side by side
        if (b, n) == shapes[1][4:6] and gap >= spans[lo][0] * size and (N == 1 or n * size >= both) \
                and (B == 1 or b * size >= (N - 1) * n * size + both):
            return True
    if any(0 in s[:4] for s in shapes):                 # (no element, or a call that is refused)
        return True
    return _apart_anyhow(at, [[a for a in zip(s[4:], s[:3]) if a[1] > 1] for s in shapes], shapes[0][3], size)


def _apart_anyhow(at, axes, d, size):
    """The same from addresses, axes (stride, entries) and the length of a head, for strides of any order."""
    if any(s == 0 for a in axes for s, _ in a):
        return False
    spans = [_extent(a, d) for a in axes]
    if None not in spans:
        if len(at) == 1:
            return True
        lo, hi = (0, 1) if at[0] <= at[1] else (1, 0)
        gap = at[hi] - at[lo]
        if gap >= spans[lo] * size:
            return True
        # side by side inside the axes on which both step alike
        alike = sorted((a for a in axes[0] if a in axes[1]), reverse=True)
        for n in range(1, len(alike) + 1):
            inside = [_extent([a for a in x if a not in alike[:n]], d) for x in axes]
            if gap >= inside[lo] * size and _extent(alike[:n], -(-gap // size) + inside[hi]) is not None:
                return True
    # every head's place
    places = []
    for p, x in zip(at, axes):
        p = torch.full((1,), p, dtype=torch.int64, device="cpu")
        for s, n in x:
            p = (p[:, None] + torch.arange(n, dtype=torch.int64, device="cpu") * (s * size)).flatten()
        places.append(p)
    return bool((torch.cat(places).sort().values.diff() >= d * size).all())


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, freqs, pos, how, *xs):
        ctx.args = _rotary_args(xs, freqs, pos, *how)
        ctx.save_for_backward(freqs, pos)
        ys = tuple(_new(t) for t in xs)
        _turn(xs, ys, freqs, pos, ctx.args, False)
        return ys

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *dys):
        # autograd's thread runs Python two to three times slower than the caller's: no checks here, the engine has
        # brought the gradients to the shapes, type and device of the outputs
        freqs, pos = ctx.saved_tensors
        dys = [dy.contiguous() for dy in dys]
        dxs = [torch.empty_like(dy) for dy in dys]
        _turn(dys, dxs, freqs, pos, ctx.args, True, x_dense=True)
        return (None, None, None, *dxs)


def rotary(x, freqs, *, k=None, pos=None, axes=None, interleaved=False, scale=1.0, start=0, inverse=False, inplace=False):
    """Rotary positions: the first ``rot = 2 * len(freqs)`` channels of every head turned pair by pair by
    position * freqs (fp64, radians; see ``rotary_freqs``), times ``scale``; the other channels are copied. Returns a new
    tensor, or with ``k`` (the same tokens, its own number of heads) a pair of them from one launch. Differentiable in x and k
    (reverse mode); frequencies that require gradients are refused.

    ``axes``: 1, or 2 for row and column positions, the first half of the turned channels going by the row and the rest by
    the column (the default for maps, ``[B, H, W, heads, d]``). ``pos``: int32 positions ``[N]`` or ``[B, N]``
    (``[.., N, 2]`` for two axes, N = H*W on a map); None: ``start`` + 0, 1, .. (below 2^31) along the tokens for one axis,
    the coordinates of a map for two.
    ``interleaved``: pairs are neighbouring channels instead of the two halves of an axis. ``inverse``: turn back.
    ``inplace``: overwrite x and k, which must not overlap, and return them; not differentiable."""
    xs = (x,) if k is None else (x, k)
    how = (axes, bool(interleaved), float(scale), int(start))
    _no_tangents(x, k, freqs)
    grad = torch.is_grad_enabled()
    if grad and getattr(freqs, "requires_grad", False):
        raise ValueError("freqs gets no gradient: detach it")
    if grad and (getattr(x, "requires_grad", False) or getattr(k, "requires_grad", False)):
        if inplace:
            raise ValueError("in-place rotation of a tensor that requires gradients")
        if inverse:
            raise ValueError("inverse is for tensors that do not require gradients")
        ys = _Rotary.apply(freqs, pos, how, *xs)
    else:
        args = _rotary_args(xs, freqs, pos, *how)
        if inplace and not _apart(xs, args[0]):
            raise ValueError("in place, no two heads may share memory: a broadcast or overlapping tensor, or x and k that overlap")
        ys = xs if inplace else [_new(t) for t in xs]
        _turn(xs, ys, freqs, pos, args, bool(inverse), y_dense=not inplace)
        if inplace:
            torch.autograd.graph.increment_version(xs)      # (for what autograd may have kept of them)
    return ys[0] if k is None else (ys[0], ys[1])


# ------------------------------------------------------------------------------------------------
# differential attention
# ------------------------------------------------------------------------------------------------

def _diff_args(q, k, v, lam, scale, causal, lens, q_pos):
    """The library's arguments, and the shape of the output."""
    B, Nq, h2, d, qb, qn, qh = _tokens(q, "q")
    Bk, Nk, k2, dk, kb, kn, kh = _tokens(k, "k", q)
    Bv, Nv, kv, dv, vb, vn, vh = _tokens(v, "v", q)
    code = _DTYPES.get(q.dtype)
    if code is None:
        _dtype_code(q)
    if h2 % 2 or k2 != 2 * kv or kv == 0 or (h2 // 2) % kv:
        raise ValueError(f"q has {h2} and k {k2} heads and v {kv}: two for each head, and a multiple of v's, are needed")
    if (Bk, Bv, Nv, dk, dv) != (B, B, Nk, d, 2 * d):
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    heads = h2 // 2
    if not isinstance(lam, torch.Tensor):
        raise TypeError("lam must be a tensor")
    if lam.dtype not in (torch.float32, q.dtype) or lam.device != q.device:
        raise ValueError(f"lam must be torch.float32 or {q.dtype} on {q.device}")
    if lam.shape == (heads,):
        lb, ln, lh = 0, 0, lam.stride(0)
    elif lam.shape == (*q.shape[:-2], heads):
        lb, ln, lh = _tokens(lam.unsqueeze(-1), "lam")[4:]
    else:
        raise ValueError(f"lam has shape {tuple(lam.shape)}, expected {(heads,)} or {(*q.shape[:-2], heads)}")
    if q_pos is not None and not causal:
        raise ValueError("q_pos goes with causal=True")
    if scale is not None and not 2.0 ** -96 <= scale <= 2.0 ** 96:         # (zero and below mean 1/sqrt(d) to the library)
        raise ValueError(f"scale must be positive, from 2^-96 to 2^96, got {scale}")
    args = DiffAttnArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), lam.data_ptr(), B, heads, kv, Nq, Nk, d, code,
                        _DTYPES[lam.dtype], qb, qn, qh, kb, kn, kh, vb, vn, vh, lb, ln, lh,
                        None if lens is None else _int32(lens, "lens", q, (B,)),
                        None if q_pos is None else _int32(q_pos, "q_pos", q, (B,)), bool(causal), _scale(scale))
    return args, (*q.shape[:-2], heads, 2 * d)


def _workspace(name, args, like):
    """Device memory for a call, or nothing where the library needs none (it then asks for 256 bytes)."""
    dev = like.get_device()
    if dev == torch.cuda.current_device():
        n = getattr(lib(), name)(ctypes.byref(args))
    else:
        with torch.cuda.device(dev):
            n = getattr(lib(), name)(ctypes.byref(args))
    return (torch.empty(n, dtype=torch.uint8, device=like.device), n) if n > 256 else (None, 0)


def _diff_forward(args, shape, q, keep):
    out = torch.empty(shape, dtype=q.dtype, device=q.device)
    maps = lse = None
    if keep:
        maps = torch.empty((*shape[:-1], 2, shape[-1]), dtype=torch.float32, device=q.device)
        lse = torch.empty((args.B, args.heads, 2, args.Nq), dtype=torch.float32, device=q.device)
    if args.Nk == 0 or out.numel() == 0:
        out.zero_()
        if keep:
            maps.zero_()
            lse.fill_(-math.inf)
    else:
        ws, nbytes = _workspace("qta_diff_attn_workspace_bytes", args, q)
        _call("qta_diff_attn", q, ctypes.byref(args), out.data_ptr(), maps.data_ptr() if keep else None,
              lse.data_ptr() if keep else None, None if ws is None else ws.data_ptr(), nbytes)
    return out, maps, lse


def _diff_backward(args, q, k, v, lam, maps, lse, dout):
    grads = [_new(t) for t in (q, k, v, lam)]
    if args.Nk == 0 or dout.numel() == 0:
        return tuple(g.zero_() for g in grads)
    ws, nbytes = _workspace("qta_diff_attn_backward_workspace_bytes", args, q)
    _call("qta_diff_attn_backward", q, ctypes.byref(args), maps.data_ptr(), lse.data_ptr(), dout.data_ptr(),
          *[g.data_ptr() for g in grads], lam.dim() == 1, None if ws is None else ws.data_ptr(), nbytes)
    return tuple(grads)


def diff_attn(q, k, v, lam, *, scale=None, causal=False, lens=None, q_pos=None, keep=False):
    """Differential attention, ``softmax(scale q0 k0^T) v - lam softmax(scale q1 k1^T) v`` for every head, the maps of
    head i being q's heads 2i and 2i + 1. q ``[B, Nq, 2*heads, d]``, k ``[B, Nk, 2*kv_heads, d]``, v
    ``[B, Nk, kv_heads, 2*d]`` (or maps ``[B, H, W, ..]``), d 32 or 64, heads a multiple of kv_heads; ``lam`` ``[heads]``
    or one for every token ``[B, Nq, heads]``, fp32 or q's type. Returns ``[B, Nq, heads, 2*d]``.

    ``lens`` (int32 ``[B]``): keys of each batch element; what lies behind them is never used, so k and v may be the
    whole of a cache. ``causal``: query i sees the keys up to position ``q_pos[b] + i`` (int32 ``[B]``; None: the
    queries are the last Nq of Nk tokens). A row that sees no key gives 0, whatever it holds. ``scale``: positive, or None
    for 1/sqrt(d). ``keep``: also return what ``diff_attn_backward`` needs."""
    args, shape = _diff_args(q, k, v, lam, scale, causal, lens, q_pos)
    out, maps, lse = _diff_forward(args, shape, q, keep)
    return (out, (maps, lse)) if keep else out


def diff_attn_backward(q, k, v, lam, kept, dout, *, scale=None, causal=False, lens=None, q_pos=None):
    """Gradients (dq, dk, dv, dlam) of ``diff_attn(.., keep=True)`` for the upstream gradient ``dout``, each in the
    shape and type of its input; ``kept`` is what that call returned, the other arguments the same."""
    args, shape = _diff_args(q, k, v, lam, scale, causal, lens, q_pos)
    maps, lse = kept
    for t, n, dtype, s in ((maps, "kept", torch.float32, (*shape[:-1], 2, shape[-1])),
                           (lse, "kept", torch.float32, (args.B, args.heads, 2, args.Nq)), (dout, "dout", q.dtype, shape)):
        if t.dtype is not dtype or t.device != q.device or t.shape != s or not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous {dtype} {tuple(s)} on {q.device}")
    return _diff_backward(args, q, k, v, lam, maps, lse, dout)


class _DiffAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, lam, scale, causal, lens, q_pos):
        ctx.args, shape = _diff_args(q, k, v, lam, scale, causal, lens, q_pos)
        out, maps, lse = _diff_forward(ctx.args, shape, q, True)
        ctx.strides, ctx.how = (q.stride(), k.stride(), v.stride(), lam.stride()), (scale, causal)
        ctx.save_for_backward(q, k, v, lam, maps, lse, lens, q_pos)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, lam, maps, lse, lens, q_pos = ctx.saved_tensors
        dout = dout.contiguous()
        if dout.data_ptr() % 16:
            dout = dout.clone()
        # the forward's checks hold as long as what was kept came back as it was laid out, at whatever address
        if (q.stride(), k.stride(), v.stride(), lam.stride()) == ctx.strides:
            args = DiffAttnArgs.from_buffer_copy(ctx.args)
            args.q, args.k, args.v, args.lam = q.data_ptr(), k.data_ptr(), v.data_ptr(), lam.data_ptr()
            args.lens = None if lens is None else lens.data_ptr()
            args.q_pos = None if q_pos is None else q_pos.data_ptr()
        else:
            args, _ = _diff_args(q, k, v, lam, *ctx.how, lens, q_pos)
        return (*_diff_backward(args, q, k, v, lam, maps, lse, dout), None, None, None, None)


def diff_attention(q, k, v, lam, *, scale=None, causal=False, lens=None, q_pos=None):
    """Differentiable ``diff_attn`` (reverse mode): gradients of q, k, v and lam."""
    _no_tangents(q, k, v, lam)
    if not (torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in (q, k, v, lam))):
        return diff_attn(q, k, v, lam, scale=scale, causal=causal, lens=lens, q_pos=q_pos)
    return _DiffAttention.apply(q, k, v, lam, scale, causal, lens, q_pos)
