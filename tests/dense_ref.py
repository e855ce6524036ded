"""Rotary positions and differential attention in 64 bits, each result with a bound on what a kernel may be off.

The bounds are sums over what the kernels round. u is half a step of the storage type relative to the value (bf16 2^-8,
fp32 2^-24), f = 2^-24. For differential attention, with L the largest scale * sum_c |q_c k_c| and N keys:
  - a weight P is off by at most w = (2 L (d + 4) + 2 N + 16) f relatively: the logit's d products and sums and its
    exponent's rounding (twice, in the weight and in the sum of weights), and N summands;
  - for a product with V or dO weights are rounded to the storage type: u more. So O_m is off by (u + w) A_m with
    A_m = P_m |V|, and O, rounded once more, by u |O| + (u + w) (A_0 + |lam| A_1) =: E;
  - D = dO V^T is off by 2 d f |dO| |V|^T;
  - t_m = dO . O_m is taken from the fp32 O_m that the forward keeps, off by (u + w + 2 f) A_m, and the dot product by
    (2 d + 2) f |dO| . |O_m|; dlam is made exact again by the sum of P_1 (D - t_1) over the Nk keys, whose terms are off by
    w P_1 |D - t_1| + P_1 dD and whose sum by Nk f (and 2 f for what it corrects);
  - dS_m = (lam) P_m (D - t_m) is off by its factors' errors, (w + 4 f) |dS_m| + P_m (dD + dt_m), and u |dS_m| when it is
    rounded for the products with K and Q; dK, dQ and dV are sums of such terms (n f more for n summands), rounded once.
"""
import math

import torch

F = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def visible(Nq, Nk, dev, length=None, causal=False, start=None):
    """[Nq, Nk] of what one batch element's queries see."""
    keys = torch.arange(Nk, device=dev)
    see = torch.ones(Nq, Nk, dtype=torch.bool, device=dev)
    if length is not None:
        see &= keys < length
    if causal:
        see &= keys <= torch.arange(Nq, device=dev)[:, None] + (Nk - Nq if start is None else start)
    return see


def diff_attention(q, k, v, lam, *, scale=None, causal=False, lens=None, q_pos=None, dout=None):
    """{name: (value, bound)} of out, and with dout of dq, dk, dv, dlam (in the shape of lam). Sequences
    [B, N, heads, d]; inputs in their storage type. Keys behind an element's length count as zero."""
    u = half_step(q.dtype)
    ul = half_step(lam.dtype)
    B, Nq, heads, d = q.shape[0], q.shape[1], q.shape[2] // 2, q.shape[3]
    Nk, kv = k.shape[1], v.shape[2]
    G = heads // kv
    sc = 1.0 / math.sqrt(d) if scale is None else scale
    Q, K, V = (t.double().clone() for t in (q, k, v))
    lamf = lam.double().expand(B, Nq, heads)
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=q.device)
    res = {"out": [z(B, Nq, heads, 2 * d), z(B, Nq, heads, 2 * d)]}
    if dout is not None:
        for n, t in (("dq", Q), ("dk", K), ("dv", V), ("dlam", lamf)):
            res[n] = [z(*t.shape), z(*t.shape)]
    for b in range(B):
        length = None if lens is None else max(0, min(Nk, int(lens[b])))
        see = visible(Nq, Nk, q.device, length, causal, None if q_pos is None else int(q_pos[b]))
        unused = ~see.any(0)
        K[b, unused] = 0.0
        V[b, unused] = 0.0
        if length is not None:
            K[b, length:] = 0.0
            V[b, length:] = 0.0
        for h in range(heads):
            g, l = h // G, lamf[b, :, h, None]
            x = [Q[b, :, 2 * h + m] for m in (0, 1)]
            y = [K[b, :, 2 * g + m] for m in (0, 1)]
            W = V[b, :, g]
            P, w = [], 0.0
            for m in (0, 1):
                s = (x[m] @ y[m].T.contiguous()) * sc
                big = float((x[m].abs() @ y[m].abs().T.contiguous()).max()) * sc if Nk else 0.0
                w = max(w, (2 * big * (d + 4) + 2 * Nk + 16) * F)
                s = s.masked_fill(~see, -math.inf)
                top = s.max(-1, keepdim=True).values.clamp(min=-1e300)
                e = (s - top).exp() * see
                P.append(e / e.sum(-1, keepdim=True).clamp(min=1e-300))
            O = [p @ W for p in P]
            A = [p @ W.abs() for p in P]
            out = O[0] - l * O[1]
            E = u * out.abs() + (u + w) * (A[0] + l.abs() * A[1])
            res["out"][0][b, :, h], res["out"][1][b, :, h] = out, E
            if dout is None:
                continue
            do = dout[b, :, h].double()
            ado = do.abs()
            D = do @ W.T.contiguous()
            eD = 2 * d * F * (ado @ W.abs().T.contiguous())
            dot = lambda a_, b_: (a_ * b_).sum(-1, keepdim=True)
            t = [dot(do, O[0]), dot(do, O[1])]
            et = [(u + w + 2 * F) * dot(ado, A[m]) + (2 * d + 2) * F * dot(ado, O[m].abs()) for m in (0, 1)]
            el = dot(P[1], (w + (Nk + 4) * F) * ((D - t[1]).abs() + et[1]) + eD) + 2 * F * (dot(ado, O[1].abs()) + et[1])
            res["dlam"][0][b, :, h], res["dlam"][1][b, :, h] = -t[1][:, 0], el[:, 0]
            for m in (0, 1):
                f = -l if m else 1.0
                dS = f * P[m] * (D - t[m])
                eS = (w + 4 * F + u) * dS.abs() + (P[m] * (l.abs() if m else 1.0)) * (eD + et[m])
                n = F * (Nk + Nq)
                dq, eq = dS @ y[m] * sc, (eS + n * dS.abs()) @ y[m].abs() * sc
                dk, ek = dS.T @ x[m] * sc, (eS + G * n * dS.abs()).T @ x[m].abs() * sc
                res["dq"][0][b, :, 2 * h + m], res["dq"][1][b, :, 2 * h + m] = dq, eq + u * dq.abs()
                res["dk"][0][b, :, 2 * g + m] += dk
                res["dk"][1][b, :, 2 * g + m] += ek
            Pd = P[0] - l * P[1]
            ap = P[0] + l.abs() * P[1]
            res["dv"][0][b, :, g] += Pd.T @ do
            res["dv"][1][b, :, g] += ((u * Pd.abs() + (w + 4 * F + G * F * Nq) * ap).T @ ado)
    if dout is not None:
        for n in ("dk", "dv"):
            res[n][1] += u * res[n][0].abs()
        if lam.dim() == 1:
            rows = B * Nq
            v_, e_ = res["dlam"]
            res["dlam"] = [v_.sum((0, 1)), e_.sum((0, 1)) + rows * F * v_.abs().sum((0, 1))]
        res["dlam"][1] = res["dlam"][1] + ul * res["dlam"][0].abs()
    return {n: tuple(x) for n, x in res.items()}


def rotary(x, freqs, pos, *, interleaved=False, scale=1.0, inverse=False):
    """(value, bound) for x [B, N, heads, d] and positions [B or 1, N, axes]. The angle is a fraction of half a turn
    rounded to fp32 (pi f), its sine and cosine are within 2 steps (4 f), and two products, a sum and the factor round
    once each: 12 f (|x1| + |x2|) |scale|, and the result's own rounding."""
    u = half_step(x.dtype)
    axes = pos.shape[-1]
    n = freqs.numel()
    per = n // axes
    j = torch.arange(n, device=x.device)
    sec, r = j // per, j % per
    first = 2 * per * sec + (2 * r if interleaved else r)
    second = first + (1 if interleaved else per)
    ang = pos.double()[..., sec] * freqs
    c, s = ang.cos()[..., None, :], ang.sin()[..., None, :] * (-1.0 if inverse else 1.0)
    X = x.double()
    a, b = X[..., first], X[..., second]
    y, e = X.clone(), torch.zeros_like(X)
    y[..., first], y[..., second] = scale * (a * c - b * s), scale * (b * c + a * s)
    far = float(pos.double().abs().max()) if pos.numel() else 0.0
    err = (12 * F + 4 * far * 2.0 ** -52) * abs(scale) * (a.abs() + b.abs())
    e[..., first] = err + u * y[..., first].abs()
    e[..., second] = err + u * y[..., second].abs()
    return y, e
