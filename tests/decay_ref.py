"""Linear attention with a decay in 64 bits, each result with a bound on what a kernel may be off.

Written as the sum over pairs, out_i = scale (sum over j <= i of W_ij (q_i . k_j) v_j + W_i S^T q_i), W_ij = exp(g (i - j)). The
bounds are sums of the terms' magnitudes times what each may be off, in units of f = 2^-24 (u is half a step of the storage type
relative to the value, bf16 2^-8, fp32 2^-24):
  - a weight is a product of powers exp2(g2 n), one for each chunk of at least 32 tokens that it crosses and up to three within
    its own: each is off by its function's and product's rounding, 4 f, and its exponent by 2 f |g2 n| (g2 and the product round)
    and thus the power by as much: (N / 8 + 12) f + 4 |g| (i - j) f in all;
  - a score of d channels by d f; what is summed over N tokens by N f, and the sum over the state's d rows by d f;
  - with bf16 inputs weighted scores and states are operands of two terms: 2^-16 = 256 f; what is added to a state has three
    terms, 2^-24;
  - results are rounded to the storage type: u of the value (states: fp32).
"""
import math

import torch

F = 2.0 ** -24


def _mix(q, k, v, g, state, first, bf16):
    """(out, state behind the last token), each (value, magnitude times f): out_i = sum over j <= i of exp(g (i - j))
    (q_i . k_j) v_j + exp(g (i + first)) state^T q_i; the state sums exp(g (n - first - j)) k_j v_j^T and exp(g n) state."""
    n, d = q.shape
    i = torch.arange(n, dtype=torch.float64, device=q.device)
    apart = (i[:, None] - i[None, :]).clamp(min=0.0)
    w = torch.exp(g * apart) * (i[:, None] >= i[None, :])
    c = n + n / 8 + 2 * d + 32 + (256 if bf16 else 0)
    ag = abs(g) if math.isfinite(g) else 0.0
    s, a = q @ k.T, q.abs() @ k.abs().T
    out, mag = (s * w) @ v, (a * w * (c + 4 * ag * apart)) @ v.abs()
    wi, ws = torch.exp(g * (i + first))[:, None], torch.exp(g * (n - first - i))[:, None]
    if math.isinf(g):                                              # (0 times infinity: one token keeps a weight of one)
        w.copy_(torch.eye(n, device=q.device))
        out, mag = (s * w) @ v, (a * w * c) @ v.abs()
        wi, ws = ((i + first) == 0).double()[:, None], ((n - first - i) == 0).double()[:, None]
    last = (k * ws).T @ v
    lmag = (k.abs() * ws * (c + 4 * ag * (n - first - i).clamp(min=0.0))[:, None]).T @ v.abs()
    if state is not None:
        out = out + wi * (q @ state)
        mag = mag + (wi * (c + 4 * ag * (i + first))[:, None]) * (q.abs() @ state.abs())
        e = math.exp(g * n) if n and math.isfinite(g) else float(n == 0)
        last = last + e * state
        lmag = lmag + e * (c + 4 * ag * n) * state.abs()
    return out, mag * F, last, lmag * F


def decay_attention(q, k, v, log_decay, *, scale=None, lens=None, state=None, dout=None, dstate_out=None):
    """{name: (value, bound)} of out and state, and with dout of dq, dk, dv and dstate. Sequences [B, N, heads, .] in their storage
    type."""
    u = torch.finfo(q.dtype).eps / 2
    bf16 = q.dtype is torch.bfloat16
    B, N, heads, dk = q.shape
    dv = v.shape[-1]
    sc = 1.0 / math.sqrt(dk) if scale is None else scale
    z = lambda *s: [torch.zeros(*s, dtype=torch.float64, device=q.device) for _ in range(2)]
    res = {"out": z(B, N, heads, dv), "state": z(B, heads, dk, dv)}
    if dout is not None:
        res.update(dq=z(*q.shape), dk=z(*k.shape), dv=z(*v.shape), dstate=z(B, heads, dk, dv))

    def put(name, at, value, bound, unit):
        res[name][0][at], res[name][1][at] = value, bound + unit * value.abs()

    for b in range(B):
        n = N if lens is None else max(0, min(N, int(lens[b])))
        for h in range(heads):
            g = float(log_decay[h])
            x, y, w = (t[b, :n, h].double() for t in (q, k, v))
            S = None if state is None else state[b, h].double()
            o, e, last, le = _mix(x * sc, y, w, g, S, 1, bf16)
            put("out", (b, slice(0, n), h), o, e, u)
            put("state", (b, h), last, le, F)
            if dout is None:
                continue
            do = dout[b, :n, h].double()
            R = None if dstate_out is None else dstate_out[b, h].double()
            o, e, _, _ = _mix(do, w, y, g, None if S is None else S.T, 1, bf16)
            put("dq", (b, slice(0, n), h), o * sc, e * sc, u)
            rx, ry, rw, rd = (t.flip(0) for t in (x * sc, y, w, do))
            o, e, first, fe = _mix(ry, rx, rd, g, R, 0, bf16)
            put("dv", (b, slice(0, n), h), o.flip(0), e.flip(0), u)
            put("dstate", (b, h), first, fe, F)
            o, e, _, _ = _mix(rw, rd, rx, g, None if R is None else R.T, 0, bf16)
            put("dk", (b, slice(0, n), h), o.flip(0), e.flip(0), u)
    return {n: tuple(x) for n, x in res.items()}
