"""What the speed of linear attention with a decay and of group norm is measured on.

A case is a dict of plain values. Its ``kind`` names the call a user's program makes:

  decay        linear attention with a decay for each head, inference: prompts, drafts and single tokens, with or without
               a state that is carried on
  decay_train  the same and its gradients, for given upstream gradients
  norm         group norm with an activation, channels last, inference
  norm_train   the same and its gradients, for a given upstream gradient

``own`` false computes the operators in plain torch in 32 bits, true makes the framework's calls.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 128                                                       # tokens that the plain form takes at a time


def _decay(name, kind, B, N, heads, dk, dv, dtype, ragged=False, carried=False):
    """``ragged``: every batch element has its own number of tokens; ``carried``: a state goes in and comes out (and
    in training their gradients)."""
    case = dict(kind=kind, B=B, N=N, heads=heads, dk=dk, dv=dv, dtype=dtype, ragged=ragged, carried=carried)
    if name:
        case["name"] = name
    return case


def _norm(name, kind, B, H, W, C, groups, dtype, act="none", affine=True, per_token=False):
    """Maps of H x W tokens, or with H = 0 sequences of W; ``per_token``: every token has its own statistics."""
    case = dict(kind=kind, B=B, H=H, W=W, C=C, groups=groups, dtype=dtype, act=act, affine=affine, per_token=per_token)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # serving, one new token for each of 8 requests: latency is all there is
        _decay("step_few_bf16", "decay", 8, 1, 16, 64, 64, "bf16", carried=True),
        # serving a large batch, one new token each: the states are read and written
        _decay("step_batch_bf16", "decay", 64, 1, 32, 128, 128, "bf16", carried=True),
        # five drafted tokens at once over states that are kept for going back, fp32
        _decay("draft_f32", "decay", 8, 5, 16, 32, 64, "f32", carried=True),
        # the next piece of prompts of different lengths, behind what was read before
        _decay("prompt_ragged_bf16", "decay", 3, 1031, 8, 32, 64, "bf16", ragged=True, carried=True),
        # one long prompt, values twice as wide as keys
        _decay("prompt_long_bf16", "decay", 1, 65536, 16, 64, 128, "bf16", carried=True),
        # training in fp32 on pieces of documents of odd length, the state and its gradient passed on
        _decay("ragged_f32_train", "decay_train", 2, 997, 8, 32, 32, "f32", ragged=True, carried=True),
        # training in bf16
        _decay("long_bf16_train", "decay_train", 2, 8192, 16, 128, 128, "bf16"),
        # the output of 16 heads for 8 new tokens, each head of each token normalised
        _norm("norm_token_bf16", "norm", 8, 0, 1, 2048, 16, "bf16", affine=False, per_token=True),
        # the values' map of a stereo pair (640x480 at 1/4), convolution - norm - activation
        _norm("norm_map_bf16", "norm", 2, 120, 160, 256, 32, "bf16", act="silu"),
        # a training step of the heads' norm behind a long sequence
        _norm("norm_heads_bf16_train", "norm_train", 2, 0, 8192, 2048, 16, "bf16", per_token=True),
        # a training step on an odd fp32 map with few channels
        _norm("norm_odd_f32_train", "norm_train", 3, 61, 83, 90, 6, "f32", act="gelu"),
        # a training step on the maps of a dense-prediction backbone
        _norm("norm_map_bf16_train", "norm_train", 8, 200, 336, 256, 32, "bf16", act="silu"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    kind = rng.choice(["step", "step", "decay", "decay", "decay_train", "decay_train", "norm", "norm", "norm_train", "norm_train"])
    if kind.startswith("norm"):
        groups = rng.choice([1, 2, 3, 6, 8, 12, 16, 32, 32])
        C = groups * rng.choice([1, 3, 4, 5, 8, 8, 16, 24, 32, 64, 128])
        # from one token to the tensors of the largest listed case
        top = 275_000_000 // size // C // (2 if dtype == "f32" else 1)
        tokens = _log_int(rng, 1, top)
        B = min(tokens, _log_int(rng, 1, 32))
        H, W = 0, tokens // B
        if W >= 64 and rng.random() < 0.6:
            H = max(4, int(math.sqrt(W) * math.exp(rng.uniform(-0.5, 0.3))))
            W = W // H
        acts = ["none", "silu", "silu", "gelu"] + (["relu"] if kind == "norm" else [])
        return _norm(None, kind, B, H, W, C, groups, dtype, rng.choice(acts), rng.random() < 0.8, rng.random() < 0.3)
    heads = rng.choice([1, 2, 3, 4, 8, 12, 16, 32])
    dk, dv = rng.choice([32, 64, 64, 128]), rng.choice([32, 64, 64, 128])
    if kind == "step":
        top = 268_000_000 // (8 * heads * dk * dv)
        return _decay(None, "decay", _log_int(rng, 1, max(1, min(256, top))), rng.choice([1, 1, 1, 2, 3, 5, 8]), heads, dk, dv,
                      dtype, carried=True)
    train = kind == "decay_train"
    # the bytes of the largest listed pass, the products of which fp32 has the longer time for
    room = (500_000_000 if train else 800_000_000) // size // (2 * (dk + dv)) // (4 if dtype == "f32" else 1) // (2 if train else 1)
    N = _log_int(rng, 2, max(2, min(65536, room // heads)))
    B = _log_int(rng, 1, max(1, min(16, room // (heads * N))))
    return _decay(None, kind, B, N, heads, dk, dv, dtype, rng.random() < 0.4, rng.random() < 0.6)


# --------------------------------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------------------------------

def _device():
    return torch.device("cuda", torch.cuda.current_device()) if torch.cuda.is_available() else torch.device("cpu")


def _inputs(case, seed):
    dev = _device()
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device=dev)
    dt = DTYPES[case["dtype"]]
    B, train = case["B"], case["kind"].endswith("train")
    if case["kind"].startswith("norm"):
        C = case["C"]
        lead = (B, case["H"], case["W"]) if case["H"] else (B, case["W"])
        # channels have means and widths of their own
        s = {"x": (rand(*lead, C) * (0.5 + rand(C).abs()) + rand(C)).to(dt), "weight": None, "bias": None}
        if case["affine"]:
            s["weight"], s["bias"] = (1.0 + 0.2 * rand(C)).to(dt), (0.2 * rand(C)).to(dt)
        if train:
            s["dy"] = rand(*lead, C).to(dt)
        return s
    N, heads, dk, dv = case["N"], case["heads"], case["dk"], case["dv"]
    s = {"q": rand(B, N, heads, dk).to(dt), "k": rand(B, N, heads, dk).to(dt), "v": rand(B, N, heads, dv).to(dt),
         "lens": None, "lengths": [N] * B, "state": None}
    # heads remember from two tokens to some five hundred
    s["log_decay"] = -(2.0 ** (-1.0 - 8.0 * (torch.arange(heads, device=dev) + 0.5) / heads))
    if case["ragged"]:
        lens = torch.randint((N + 1) // 2, N + 1, (B,), generator=g, device=dev)
        s["lens"], s["lengths"] = lens.to(torch.int32), lens.tolist()
    if case["carried"]:
        s["state"] = 2.0 * rand(B, heads, dk, dv)
    if train:
        s["dout"] = rand(B, N, heads, dv).to(dt)
        s["dstate"] = rand(B, heads, dk, dv) if case["carried"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "decay" and case["N"] <= 8:
        s["next"] = torch.empty_like(s["state"])                  # the other of a program's two sets of states
    if own and case["kind"].endswith("train"):
        for n in ("q", "k", "v", "state", "x", "weight", "bias"):
            if s.get(n) is not None:
                s[n].requires_grad_(True)
    return s


# --------------------------------------------------------------------------------------------------
# the calls
# --------------------------------------------------------------------------------------------------

def run(state):
    if not own:
        return _plain(state)
    import paper_2201_02767_amd as qta

    s, case = state, state["case"]
    if case["kind"].startswith("norm"):
        y = qta.group_norm(s["x"], case["groups"], s["weight"], s["bias"], act=case["act"], per_token=case["per_token"])
        if case["kind"] == "norm":
            return y
        leaves = (s["x"], s["weight"], s["bias"]) if case["affine"] else (s["x"],)
        return (y.detach(), *torch.autograd.grad(y, leaves, s["dy"]))
    args = (s["q"], s["k"], s["v"], s["log_decay"])
    if case["kind"] == "decay":
        if "next" in s:
            return qta.decay_attn(*args, lens=s["lens"], state=s["state"], state_out=s["next"])
        return qta.decay_attn(*args, lens=s["lens"], state=s["state"], return_state=case["carried"])
    if not case["carried"]:
        out = qta.decay_attention(*args, lens=s["lens"])
        return (out.detach(), *torch.autograd.grad(out, args[:3], s["dout"]))
    out, last = qta.decay_attention(*args, lens=s["lens"], state=s["state"], return_state=True)
    return (out.detach(), last.detach(), *torch.autograd.grad((out, last), (*args[:3], s["state"]), (s["dout"], s["dstate"])))


# ---- plain forms, in 32 bits ----

def _mix(q, k, v, g, state, first):
    """out_i = sum over j <= i of exp(g (i - j)) (q_i . k_j) v_j + exp(g (i + first)) q_i state, and the state behind the last
    token, sum over j of exp(g (n - first - j)) k_j v_j + exp(g n) state. [B, n, heads, .] in fp32, g [heads]."""
    B, n, heads, dk = q.shape
    dv = v.shape[-1]
    c = min(CHUNK, n)
    m = (n + c - 1) // c
    if state is None:
        state = torch.zeros(B, heads, dk, dv, device=q.device)

    def chunks(t):
        t = torch.cat((t, t.new_zeros(B, m * c - n, heads, t.shape[-1])), 1) if m * c > n else t
        return t.reshape(B, m, c, heads, -1).permute(1, 0, 3, 2, 4).contiguous()      # [m, B, heads, c, .]

    q, k, v = chunks(q), chunks(k), chunks(v)
    i = torch.arange(c, device=g.device)
    apart = (i[:, None] - i[None, :]).float()
    w = torch.where(apart >= 0, torch.exp(g[:, None, None] * apart.clamp(min=0.0)), 0.0)          # [heads, c, c]
    out = torch.matmul(torch.matmul(q, k.transpose(-1, -2).contiguous()) * w, v)
    come = torch.exp(g[:, None] * (i + first).float())[..., None]                                  # [heads, c, 1]
    for x in range(m):
        size = min(c, n - x * c)
        out[x] += torch.matmul(q[x], state) * come
        keep = torch.exp(g[:, None] * (size - first - i).clamp(min=0).float())[..., None]
        # (what lies behind the last token is zero)
        state = state * torch.exp(g * size)[:, None, None] + torch.matmul((k[x] * keep).transpose(-1, -2).contiguous(), v[x])
    return out.permute(1, 0, 3, 2, 4).reshape(B, m * c, heads, dv)[:, :n], state


def _plain_decay(s):
    case, g = s["case"], s["log_decay"]
    q, k, v = s["q"], s["k"], s["v"]
    B, N = q.shape[:2]
    scale = 1.0 / math.sqrt(case["dk"])
    train, carried = case["kind"] == "decay_train", case["carried"]
    out = torch.zeros_like(v)
    last = torch.empty(B, case["heads"], case["dk"], case["dv"], device=q.device) if carried else None
    grads = [torch.zeros_like(t) for t in (q, k, v)] + ([torch.empty_like(last)] if carried else []) if train else []
    # batch elements of one length at a time
    for n, which in ([(N, slice(None))] if not case["ragged"] else [(n, slice(b, b + 1)) for b, n in enumerate(s["lengths"])]):
        x, y, z = (t[which, :n].float() for t in (q, k, v))
        before = s["state"][which] if carried else None
        o, after = _mix(x * scale, y, z, g, before, 1)
        out[which, :n] = o.to(out.dtype)
        if carried:
            last[which] = after
        if not train:
            continue
        do = s["dout"][which, :n].float()
        turned = None if before is None else before.transpose(-1, -2).contiguous()
        dq, _ = _mix(do, z, y, g, turned, 1)
        # what reaches a key and a value comes from later tokens: the same with time running back
        back = s["dstate"][which] if carried else None
        rx, ry, rz, rdo = (t.flip(1) for t in (x * scale, y, z, do))
        dv, dstate = _mix(ry, rx, rdo, g, back, 0)
        dk, _ = _mix(rz, rdo, rx, g, None if back is None else back.transpose(-1, -2).contiguous(), 0)
        for t, new in zip(grads, (dq * scale, dk.flip(1), dv.flip(1))):
            t[which, :n] = new.to(t.dtype)
        if carried:
            grads[3][which] = dstate
    if not train:
        return (out, last) if carried else out
    return (out, last, *grads) if carried else (out, *grads)


def _activation(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z.clamp(min=0.0) if act == "relu" else z


def _slope(z, act):
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _plain_norm(s):
    case = s["case"]
    C, groups = case["C"], case["groups"]
    n = case["B"] * max(case["H"], 1) * case["W"]
    units = n if case["per_token"] else case["B"]
    split = (units, n // units, groups, C // groups)
    x = s["x"].float().reshape(split)
    x = x - x.mean((1, 3), keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean((1, 3), keepdim=True) + 1e-5)
    x = x * r
    w = s["weight"].float().reshape(groups, -1) if case["affine"] else 1.0
    z = x * w + s["bias"].float().reshape(groups, -1) if case["affine"] else x
    y = _activation(z, case["act"]).to(s["x"].dtype).reshape(s["x"].shape)
    if case["kind"] == "norm":
        return y
    dz = s["dy"].float().reshape(split) * _slope(z, case["act"])
    dn = dz * w
    dx = r * (dn - dn.mean((1, 3), keepdim=True) - x * (dn * x).mean((1, 3), keepdim=True))
    dx = dx.to(s["x"].dtype).reshape(s["x"].shape)
    if not case["affine"]:
        return y, dx
    return y, dx, (dz * x).sum((0, 1)).reshape(C).to(s["weight"].dtype), dz.sum((0, 1)).reshape(C).to(s["bias"].dtype)


def _plain(s):
    return _plain_norm(s) if s["case"]["kind"].startswith("norm") else _plain_decay(s)


# --------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------

def work(case):
    tb = 2.0 if case["dtype"] == "bf16" else 4.0
    if case["kind"].startswith("norm"):
        elems = float(case["B"] * max(case["H"], 1) * case["W"] * case["C"])
        weights = 2.0 * case["C"] * tb if case["affine"] else 0.0
        if case["kind"] == "norm":
            return {"bytes": 2 * elems * tb + weights, "flops": 10.0 * elems}
        # x and dy in, y and dx out
        return {"bytes": 4 * elems * tb + 2 * weights, "flops": 30.0 * elems}
    # ragged lengths lie between a half and the whole: three quarters on average
    tokens = case["B"] * case["heads"] * case["N"] * (0.75 if case["ragged"] else 1.0)
    rows = float(case["B"] * case["heads"] * case["N"])
    dk, dv = case["dk"], case["dv"]
    states = float(case["B"] * case["heads"] * dk * dv * 4) if case["carried"] else 0.0
    # the recurrence: a product into the state and one out of it for each token
    if case["kind"] == "decay":
        return {"bytes": (tokens * (2 * dk + dv) + rows * dv) * tb + 2 * states, "flops": 4.0 * dk * dv * tokens}
    # q, k, v and dout in, out and the three gradients out; two recurrences, and three products out of them
    return {"bytes": (tokens + rows) * (2 * dk + 2 * dv) * tb + 4 * states, "flops": 14.0 * dk * dv * tokens}


# --------------------------------------------------------------------------------------------------
# the same in 64 bits: token by token, as the state is defined, and the norm's moments
# --------------------------------------------------------------------------------------------------

def _exact_decay(case, s):
    B, N, heads, dk, dv = case["B"], case["N"], case["heads"], case["dk"], case["dv"]
    train, carried = case["kind"] == "decay_train", case["carried"]
    # about 40 us a token and pass over it
    if N * max(1.0, B * heads * dk * dv / 2e6) * (4 if train else 1) > 400_000:
        return None
    f = torch.exp(s["log_decay"].double())[:, None, None]
    scale = 1.0 / math.sqrt(dk)
    alive = [[n > t for n in s["lengths"]] for t in range(N)] if case["ragged"] else None
    first = lambda t: t.double().permute(1, 0, 2, 3).contiguous()                # [N, B, heads, .]
    q, k, v = first(s["q"]), first(s["k"]), first(s["v"])
    out = torch.zeros(N, B, heads, dv, dtype=torch.float64, device=q.device)
    S = s["state"].double() if carried else torch.zeros(B, heads, dk, dv, dtype=torch.float64, device=q.device)
    if case["ragged"]:
        on = torch.tensor(alive, device=q.device)[:, :, None, None, None]        # [N, B, 1, 1, 1]
    if train:
        do = first(s["dout"])
        dq, dk_, dv_ = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for t in range(N):
        new = S * f + k[t, ..., :, None] * v[t, ..., None, :]
        S = torch.where(on[t], new, S) if case["ragged"] else new
        out[t] = scale * (q[t, ..., :, None] * S).sum(-2)
        if train:
            dq[t] = scale * (S * do[t, ..., None, :]).sum(-1)
    if train:
        # G: the loss's gradient with respect to the state behind token t
        G = s["dstate"].double() if carried else torch.zeros_like(S)
        for t in range(N - 1, -1, -1):
            here = G + scale * q[t, ..., :, None] * do[t, ..., None, :]
            if case["ragged"]:
                here = torch.where(on[t], here, G)
            dk_[t] = (here * v[t, ..., None, :]).sum(-1)
            dv_[t] = (here * k[t, ..., :, None]).sum(-2)
            G = torch.where(on[t], here * f, G) if case["ragged"] else here * f
    result = [out] + ([dq, dk_, dv_] if train else [])
    if case["ragged"]:
        result = [torch.where(on[..., 0], t, 0.0) for t in result]
    result = [t.permute(1, 0, 2, 3) for t in result]
    if carried:
        result.insert(1, S)
        if train:
            result.append(G)
    return tuple(result) if len(result) > 1 else result[0]


def _exact_norm(case, s):
    C, groups, act = case["C"], case["groups"], case["act"]
    x = s["x"].double().flatten(0 if case["per_token"] else 1, -2)               # [tokens, C] or [B, N, C]
    if case["per_token"]:
        x = x[:, None]
    shape = x.shape
    x = x.unflatten(-1, (groups, C // groups))
    var, mean = torch.var_mean(x, dim=(1, 3), correction=0, keepdim=True)
    sigma = (var + 1e-5).sqrt()
    n = ((x - mean) / sigma).reshape(shape)
    del x
    one = torch.ones(C, dtype=torch.float64, device=n.device)
    w, b = (s["weight"].double(), s["bias"].double()) if case["affine"] else (one, 0.0 * one)
    z = n * w + b
    phi = lambda t: 0.5 * torch.special.erfc(-t / math.sqrt(2.0))
    y = {"none": lambda: z, "relu": lambda: z.relu(), "silu": lambda: z * z.sigmoid(), "gelu": lambda: z * phi(z)}[act]()
    y = y.reshape(s["x"].shape)
    if case["kind"] == "norm":
        return y
    if act == "silu":
        d = z.sigmoid() * (1.0 + z * (-z).sigmoid())
    elif act == "gelu":
        d = phi(z) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    else:
        d = torch.ones_like(z)
    del z
    dz = s["dy"].double().reshape(shape) * d
    del d
    dw, db = (dz * n).sum((0, 1)), dz.sum((0, 1))
    dn = (dz * w).unflatten(-1, (groups, C // groups))
    n = n.unflatten(-1, (groups, C // groups))
    count = dn.shape[1] * dn.shape[3]
    m0, m1 = dn.sum((1, 3), keepdim=True) / count, (dn * n).sum((1, 3), keepdim=True) / count
    dx = ((dn - m0 - n * m1) / sigma).reshape(s["x"].shape)
    return (y, dx, dw, db) if case["affine"] else (y, dx)


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_norm(case, s) if case["kind"].startswith("norm") else _exact_decay(case, s)
