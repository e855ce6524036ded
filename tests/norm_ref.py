"""Group norm with an activation in 64 bits, each result with a bound on what a kernel may be off.

f = 2^-24, u is half a step of the storage type relative to the value (bf16 2^-8, fp32 2^-24), M the largest |x| of a group, N its tokens
(at most N of them follow each other in one sum; joining rows, channels and slabs takes at most 300 more steps):
  - a running mean moves by a rounded part of a difference three times a step: dm = 3 (N + 300) f M;
  - a difference x - mean is off by e = f (|x| + |mean|) + dm, the variance by 2 mean(|x - mean| e) + e^2 + 3 (N + 300) f var, and r by
    half of that relative to var + eps, and 4 f;
  - n = (x - mean) r by r e + |n| (dr / r + 2 f); z = w n + b by |w| dn + 2 f (|w n| + |b|);
  - activations have slopes of at most 1.13, and their slopes of at most 1 (ReLU's jumps: where |z| is below dz, by 1); their own functions
    are off by 8 f (1 + |z|);
  - sums over N tokens by (N + 300) f of the terms' magnitudes, and what the terms are off; results are rounded once.
"""
import math

import torch

F = 2.0 ** -24


def _act(z, act):
    phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    s = torch.sigmoid(z)
    return {"none": (z, torch.ones_like(z)), "relu": (z.clamp(min=0), (z > 0).double()), "silu": (z * s, s * (1 + z * (1 - s))),
            "gelu": (z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))}[act]


def group_norm(x, groups, weight=None, bias=None, *, eps=1e-5, act="none", per_token=False, dy=None):
    """{name: (value, bound)} of y, and with dy of dx, dweight and dbias (as of weights of 1 and 0 where there are none)."""
    u = torch.finfo(x.dtype).eps / 2
    uw = torch.finfo(weight.dtype if weight is not None else bias.dtype if bias is not None else torch.float32).eps / 2
    shape, C = x.shape, x.shape[-1]
    X = x.double().reshape(shape[0], -1, C)
    Y = dy.double().reshape(X.shape) if dy is not None else None
    tokens = X.shape[0] * X.shape[1]
    if per_token:
        X = X.reshape(-1, 1, C)
        Y = Y.reshape(X.shape) if dy is not None else None
    B, N, _ = X.shape
    split = lambda t: t.reshape(*t.shape[:-1], groups, C // groups)
    over = lambda t: split(t).mean((1, 3), keepdim=True).expand(-1, N, -1, C // groups).reshape(B, N, C)
    top = lambda t: split(t).amax((1, 3), keepdim=True).expand(-1, N, -1, C // groups).reshape(B, N, C)
    one = torch.ones(C, dtype=torch.float64, device=x.device)
    w = weight.double() if weight is not None else one
    b = bias.double() if bias is not None else 0 * one
    steps = (N + 300) * F
    mean = over(X)
    d = X - mean
    var = over(d * d)
    r = 1 / torch.sqrt(var + eps)
    n = d * r
    e = F * (X.abs() + mean.abs()) + 3 * steps * top(X.abs())
    dvar = 2 * over(d.abs() * e) + top(e) ** 2 + 3 * steps * var
    dr = 0.5 * dvar / (var + eps) + 4 * F
    en = r * e + n.abs() * (dr + 2 * F)
    z = w * n + b
    ez = w.abs() * en + 2 * F * ((w * n).abs() + b.abs())
    y, s = _act(z, act)
    out = {"y": (y.reshape(shape), (1.13 * ez + 8 * F * (1 + z.abs()) + u * y.abs()).reshape(shape))}
    if dy is None:
        return out
    dz = Y * s
    edz = Y.abs() * (ez + 8 * F * (1 + z.abs()))
    if act == "relu":
        edz = edz + Y.abs() * (z.abs() <= ez)
    dn, edn = w * dz, w.abs() * edz + F * (w * dz).abs()
    s0, s1 = over(dn), over(dn * n)
    es0 = over(edn) + steps * over(dn.abs())
    es1 = over(edn * n.abs() + dn.abs() * en) + steps * over((dn * n).abs())
    dx = r * (dn - s0 - n * s1)
    edx = r * (edn + es0 + n.abs() * es1 + en * s1.abs() + 4 * F * (dn.abs() + s0.abs() + (n * s1).abs())) + dx.abs() * (dr + u)
    total = (tokens + 300) * F
    dw, db = (dz * n).sum((0, 1)), dz.sum((0, 1))
    edw = (edz * n.abs() + dz.abs() * en + total * (dz * n).abs()).sum((0, 1)) + uw * dw.abs()
    edb = (edz + total * dz.abs()).sum((0, 1)) + uw * db.abs()
    out.update(dx=(dx.reshape(shape), edx.reshape(shape)), dweight=(dw, edw), dbias=(db, edb))
    return out
