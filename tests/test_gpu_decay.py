"""Linear attention with a decay on the GPU against tests/decay_ref.py's 64-bit values and its bounds (element by element:
|gpu - ref| <= bound)."""
import math

import pytest
import torch

import paper_2201_02767_amd as P
from tests import decay_ref as R
from tests.test_gpu_dense import DT, announce, dev, gen, i32, within       # noqa: F401

pytestmark = pytest.mark.gpu


def make(dev, B, N, heads, dk, dv, dtype, seed=0, state=True):
    r = gen(seed, dev)
    dt = DT[dtype]
    q, k, v = r(B, N, heads, dk).to(dt), r(B, N, heads, dk).to(dt), r(B, N, heads, dv).to(dt)
    g = -torch.logspace(-0.3, -3.0, heads, device=dev)
    s = 2 * r(B, heads, dk, dv) if state else None
    return (q, k, v, g, s), (r(B, N, heads, dv).to(dt), r(B, heads, dk, dv))


def check(args, ups, *, label="", grads=True, ref=None, **how):
    q, k, v, g, s = args
    announce(f"decay_attn {label} q {tuple(q.shape)} v {tuple(v.shape)} {q.dtype} state {s is not None} {how}")
    how = {n: (i32(x, q.device) if n == "lens" else x) for n, x in how.items()}
    dout, dlast = ups
    rq, rk, rv, rd = ref or (q, k, v, dout)
    want = R.decay_attention(rq, rk, rv, g, state=s, dout=rd if grads else None, dstate_out=dlast, **how)
    out, last = P.decay_attn(q, k, v, g, state=s, return_state=True, **how)
    torch.cuda.synchronize()
    within("out", out, want["out"])
    within("state", last, want["state"])
    if not grads:
        return out, last
    got = P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast, **how)
    torch.cuda.synchronize()
    for n, t in zip(("dq", "dk", "dv", "dstate"), got):
        if t is not None:
            within(n, t, want[n])
    return out, last


SIZES = [(1, 1, 1), (2, 2, 3), (1, 16, 2), (1, 17, 1), (2, 31, 2), (1, 32, 1), (1, 33, 2), (2, 64, 1), (1, 65, 3), (1, 95, 1),
         (1, 129, 2), (3, 300, 2), (1, 1025, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 64), (128, 128), (32, 128), (128, 64), (64, 32)])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(dev, size, dk, dv, dtype):
    check(*make(dev, *size, dk, dv, dtype, seed=sum(size)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_a_state(dev, dtype):
    for N in (1, 7, 100, 600):
        args, (dout, _) = make(dev, 2, N, 3, 64, 32, dtype, seed=N, state=False)
        check(args, (dout, None))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [9, 150, 700])
def test_lengths(dev, N, dtype):
    """Lengths of zero, one, on and beside the borders of chunks and segments, all, beyond and below (clamped); what lies behind
    them may be anything and is not used."""
    lens = [0, 1, 31, 32, 33, 64, 65, 128, N - 1, N, N + 7, -3]
    args, ups = make(dev, len(lens), N, 2, 32, 64, dtype, seed=N)
    q, k, v, g, s = args
    ref = [t.clone() for t in (q, k, v, ups[0])]
    for b, n in enumerate(lens):
        for t in (q, k, v, ups[0]):
            t[b, max(n, 0):] = math.nan
    out, _ = check(args, ups, lens=lens, ref=ref)
    for b, n in enumerate(lens):
        assert bool((out[b, max(n, 0):] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [3, 40, 300])
def test_views(dev, N, dtype):
    """Parts of one projection, heads that share keys by a zero stride, a transposed batch, a map."""
    r = gen(5, dev)
    x = r(2, N, 4, 128).to(DT[dtype])
    q, k, v = x[..., :32], x[..., 32:64], x[..., 64:]
    (_, _, _, g, s), _ = make(dev, 2, 1, 4, 32, 64, dtype, seed=N)
    dout, dlast = r(2, N, 4, 64).to(DT[dtype]), r(2, 4, 32, 64)
    check((q, k, v, g, s), (dout, dlast), label="views")
    one = r(N, 2, 1, 64).to(DT[dtype]).transpose(0, 1)
    check((q, one[..., :32].expand(2, N, 4, 32), one.expand(2, N, 4, 64), g, s), (dout, dlast), label="shared")
    args = [t.reshape(2, N // 3 if N % 3 == 0 else 1, -1, *t.shape[2:]) for t in (q, k, v)]
    out = P.decay_attn(*[t.contiguous() for t in args], g, state=s)
    assert out.shape == (*args[0].shape[:-1], 64)
    assert torch.equal(out.reshape(2, N, 4, 64), P.decay_attn(q, k, v, g, state=s))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [2, 16, 70, 400])
def test_decays(dev, N, dtype):
    """Nothing forgotten, nothing remembered, in between, and growth."""
    (q, k, v, _, s), ups = make(dev, 1, N, 8, 32, 32, dtype, seed=N)
    g = torch.tensor([0.0, -math.inf, -1e-7, -0.01, -1.0, -30.0, -3000.0, 0.005], device=dev)
    check((q, k, v, g, s), ups, label="decays")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** -64, 0.3, 2.0 ** 20])
def test_scales(dev, scale, dtype):
    args, ups = make(dev, 1, 150, 2, 64, 32, dtype, seed=1)
    check(args, ups, scale=scale, label="scale") if scale < 1 else check(args, (ups[0], None), scale=scale, label="scale")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_states_in_place(dev, dtype):
    """A state may be overwritten by the call that reads it: the same results."""
    for N in (1, 16, 17, 40, 2000):
        (q, k, v, g, s), _ = make(dev, 2, N, 2, 64, 64, dtype, seed=N)
        out, last = P.decay_attn(q, k, v, g, state=s, return_state=True)
        t = s.clone()
        out2, same = P.decay_attn(q, k, v, g, state=t, state_out=t)
        assert same is t and torch.equal(out, out2) and torch.equal(last, t)
        other = torch.full_like(s, math.nan)
        P.decay_attn(q, k, v, g, state=s, state_out=other)
        assert torch.equal(last, other)


def test_runs_are_identical(dev):
    args, (dout, dlast) = make(dev, 2, 3000, 3, 64, 128, "bf16", seed=2)
    q, k, v, g, s = args
    first = (*P.decay_attn(q, k, v, g, state=s, return_state=True), *P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast))
    for _ in range(3):
        again = (*P.decay_attn(q, k, v, g, state=s, return_state=True), *P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_prompt_in_pieces_then_tokens(dev, dtype):
    """The state carries on: pieces of any length, then token by token, against one call's 64-bit values."""
    (q, k, v, g, s), _ = make(dev, 2, 350, 2, 64, 32, dtype, seed=8)
    want = R.decay_attention(q, k, v, g, state=s)
    state, at, outs = s.clone(), 0, []
    for n in (100, 1, 37, 200, 1, 1, 2, 5, 3):
        o, _ = P.decay_attn(*[t[:, at:at + n] for t in (q, k, v)], g, state=state, state_out=state)
        outs.append(o)
        at += n
    assert at == 350
    within("out", torch.cat(outs, 1), want["out"])
    # (each of nine pieces starts from a rounded state)
    value, bound = want["state"]
    within("state", state, (value, bound + 9 * R.F * value.abs().max()))


def test_empty_calls(dev):
    z = lambda *s: torch.zeros(*s, device=dev)
    g, s = z(2), torch.randn(3, 2, 32, 64, device=dev)
    out, last = P.decay_attn(z(3, 0, 2, 32), z(3, 0, 2, 32), z(3, 0, 2, 64), g, state=s, return_state=True)
    assert out.shape == (3, 0, 2, 64) and torch.equal(last, s)
    out, last = P.decay_attn(z(0, 5, 2, 32), z(0, 5, 2, 32), z(0, 5, 2, 64), g, return_state=True)
    assert out.shape == (0, 5, 2, 64) and last.shape == (0, 2, 32, 64)
    q, k, v = (t.requires_grad_() for t in (z(3, 0, 2, 32), z(3, 0, 2, 32), z(3, 0, 2, 64)))
    s.requires_grad_()
    out, last = P.decay_attention(q, k, v, g, state=s, return_state=True)
    (last * 2).sum().backward()
    assert torch.equal(s.grad, torch.full_like(s, 2.0)) and q.grad.shape == q.shape


def test_autograd(dev):
    """Gradients through either result alone and both; views of what comes back; what is refused."""
    (q, k, v, g, s), (dout, dlast) = make(dev, 2, 90, 2, 32, 64, "f32", seed=4)
    for use in ("out", "state", "both"):
        leaves = [t.detach().clone().requires_grad_() for t in (q, k, v, s)]
        out, last = P.decay_attention(*leaves[:3], g, state=leaves[3], return_state=True)
        ups = [(out, dout)] * (use != "state") + [(last, dlast)] * (use != "out")
        torch.autograd.backward([a for a, _ in ups], [b for _, b in ups])
        want = R.decay_attention(q, k, v, g, state=s, dout=dout * (use != "state"), dstate_out=dlast * (use != "out"))
        for n, t in zip(("dq", "dk", "dv", "dstate"), leaves):
            within(f"{use} {n}", t.grad, want[n])
    # an upstream gradient that is a broadcast view; a leaf without a gradient
    a = q.detach().requires_grad_()
    (P.decay_attention(a, k, v, g).sum() * 2).backward()
    within("dq", a.grad, R.decay_attention(q, k, v, g, dout=torch.full_like(dout, 2.0))["dq"])
    # a second derivative is refused, not left out
    a = q.detach().requires_grad_()
    d, = torch.autograd.grad(P.decay_attention(a, k, v, g), a, dout, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()
    with pytest.raises(ValueError, match="log_decay"):
        P.decay_attention(q, k, v, g.clone().requires_grad_())
    # what autograd keeps is not overwritten unseen
    a, st = q.detach().requires_grad_(), s.clone()
    out = P.decay_attention(a, k, v, g, state=st)
    P.decay_attn(q, k, v, g, state=st, state_out=st)
    with pytest.raises(RuntimeError, match="inplace"):
        out.backward(dout)


def test_gradients_against_differences(dev):
    (q, k, v, g, s), (dout, dlast) = make(dev, 1, 45, 1, 32, 32, "f32", seed=6)
    dq, dk, dv, ds = P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast)
    args = dict(q=q, k=k, v=v, state=s)
    r = gen(9, dev)
    for n, grad in (("q", dq), ("k", dk), ("v", dv), ("state", ds)):
        e = r(*args[n].shape)
        f = []
        for h in (0.5, -0.5):                                      # (the results are linear in each of the four)
            x = {**args, n: args[n] + h * e}
            out, last = P.decay_attn(x["q"], x["k"], x["v"], g, state=x["state"], return_state=True)
            f.append(float((out.double() * dout).sum() + (last.double() * dlast).sum()))
        slope, size = f[0] - f[1], abs(f[0]) + abs(f[1])
        # some 10^4 fp32 values, each within about 400 steps of its magnitude, whose signs differ
        assert abs(slope - float((grad.double() * e).sum())) <= 400 * R.F * 100 * (size + float((grad.double() * e).norm())), n


@pytest.mark.parametrize("N", [1, 300])
def test_streams_and_graphs(dev, N):
    """On another stream, and captured: replays read what is in the tensors then, between eager calls on the same tensors."""
    (q, k, v, g, s), (dout, dlast) = make(dev, 2, N, 2, 64, 64, "bf16", seed=N)
    side = torch.cuda.Stream()
    want = P.decay_attn(q, k, v, g, state=s, return_state=True)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = P.decay_attn(q, k, v, g, state=s, return_state=True)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    last = torch.empty_like(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, _ = P.decay_attn(q, k, v, g, state=s, state_out=last)
        grads = P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast)
    r = gen(77, dev)
    for _ in range(4):
        for t in (q, k, v, dout, s):
            t.copy_(r(*t.shape))
        graph.replay()
        eager = (*P.decay_attn(q, k, v, g, state=s, return_state=True), *P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, last, *grads), eager))


def test_two_streams_at_once(dev):
    args = [make(dev, 1, 5000, 4, 64, 64, "bf16", seed=i)[0] for i in range(2)]
    want = [P.decay_attn(*a[:4], state=a[4], return_state=True) for a in args]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in args], [[], []]
    for _ in range(5):
        for st, a, res in zip(streams, args, got):
            with torch.cuda.stream(st):
                res.append(P.decay_attn(*a[:4], state=a[4], return_state=True))
    torch.cuda.synchronize()
    for w, res in zip(want, got):
        assert all(torch.equal(x, y) for r in res for x, y in zip(w, r))


def test_offsets_past_32_bits(dev):
    """2^31 elements and more in v and out; with a decay that forgets, the last tokens are those of a short call."""
    N, heads, dv = (1 << 19) + 70, 32, 128
    q = torch.randn(1, N, 1, 32, device=dev).to(torch.bfloat16).expand(1, N, heads, 32)
    v = torch.empty(1, N, heads, dv, device=dev, dtype=torch.bfloat16).normal_()
    g = torch.full((heads,), -2.0, device=dev)
    announce("decay_attn past 2^31 elements")
    out, last = P.decay_attn(q, q, v, g, return_state=True)
    n = 100
    tail = [t[:, -n:].contiguous() for t in (q, q, v)]
    want = R.decay_attention(*tail, g)
    value, bound = want["out"]
    within("out", out[:, -50:], (value[:, -50:], bound[:, -50:] + 1e-12))
    within("state", last, (want["state"][0], want["state"][1] + 1e-12))
    del out, last
    dout = torch.empty_like(v).normal_()
    dq, dk, dv_, _ = P.decay_attn_backward(q, q, v, g, dout)
    del dq, dk
    want = R.decay_attention(*tail, g, dout=dout[:, -n:].contiguous())
    within("dv", dv_[:, -50:], tuple(t[:, -50:] for t in want["dv"]))


def test_refusals(dev):
    z = lambda *s, t=torch.float32: torch.zeros(*s, device=dev, dtype=t)
    q, k, v, g, s = z(2, 5, 2, 32), z(2, 5, 2, 32), z(2, 5, 2, 64), z(2), z(2, 2, 32, 64)
    ok = lambda **kw: P.decay_attn(**{**dict(q=q, k=k, v=v, log_decay=g), **kw})
    ok(state=s)
    for kw in (dict(k=z(2, 6, 2, 32)), dict(k=z(2, 5, 2, 64)), dict(v=z(2, 5, 3, 64)), dict(v=z(2, 5, 2, 64, t=torch.bfloat16)),
               dict(log_decay=z(3)), dict(log_decay=z(2, t=torch.float64)), dict(log_decay=g.cpu()), dict(state=z(2, 2, 64, 32)),
               dict(state=s.to(torch.bfloat16)), dict(state=s.transpose(2, 3).contiguous().transpose(2, 3)),
               dict(lens=z(2)), dict(lens=z(3, t=torch.int32)), dict(scale=0.0), dict(scale=-1.0), dict(scale=1e30),
               dict(state_out=z(2, 2, 64, 32)), dict(q=q.cpu()), dict(q=q.double(), k=k.double(), v=v.double())):
        with pytest.raises(ValueError):
            ok(**kw)
    with pytest.raises(TypeError):
        ok(q=[1.0])
    both = z(2 * s.numel() - 4)
    with pytest.raises(ValueError, match="apart"):
        ok(state=both[:s.numel()].view_as(s), state_out=both[s.numel() - 4:].view_as(s))
    with pytest.raises(P.QtaError):
        P.decay_attn(z(2, 5, 2, 48), z(2, 5, 2, 48), v, g)
    with pytest.raises(P.QtaError):
        P.decay_attn(z(2, 5, 2, 33)[..., :32], k, v, g)
    with pytest.raises(NotImplementedError, match="forward-mode"):
        from torch.autograd import forward_ad
        with forward_ad.dual_level():
            P.decay_attention(forward_ad.make_dual(q, q), k, v, g)


def test_a_layer_of_them(dev):
    """Positions, decay attention and the heads' norm: a causal layer, whose prompt and single tokens agree, and its gradients."""
    r = gen(12, dev)
    B, N, heads, d = 2, 60, 4, 64
    qkv = [r(B, N, heads, d) for _ in range(3)]
    g = -torch.tensor([0.5, 0.1, 0.02, 0.004], device=dev)
    w = (1 + 0.1 * r(heads * d)).requires_grad_()
    freqs = P.rotary_freqs(d, device=dev)

    def layer(q, k, v, start=0, state=None, train=False):
        q, k = P.rotary(q, freqs, k=k, start=start)
        if train:
            o, state = P.decay_attention(q, k, v, g, return_state=True)
        else:
            o, state = P.decay_attn(q, k, v, g, state=state, return_state=True)
        return P.group_norm(o.flatten(-2), heads, w if train else w.detach(), act="silu", per_token=True), state

    def plain(q, k, v, weight):
        at = torch.arange(N, device=dev)[:, None] * freqs
        c, s = at.cos()[:, None], at.sin()[:, None]
        turn = lambda x: torch.cat((x[..., :d // 2] * c - x[..., d // 2:] * s, x[..., d // 2:] * c + x[..., :d // 2] * s), -1)
        q, k = turn(q), turn(k)
        i = torch.arange(N, device=dev).double()
        m = torch.exp(g.double()[:, None, None] * (i[:, None] - i).clamp(min=0)) * (i[:, None] >= i)
        sc = torch.stack([torch.stack([q[b, :, h] @ k[b, :, h].T for h in range(heads)]) for b in range(B)]) * m / math.sqrt(d)
        o = torch.stack([torch.stack([sc[b, h] @ v[b, :, h] for h in range(heads)], 1) for b in range(B)])
        o = (o - o.mean(-1, keepdim=True)) / torch.sqrt(o.var(-1, keepdim=True, correction=0) + 1e-5)
        z = o.flatten(-2) * weight
        return z * torch.sigmoid(z)

    leaves = [t.clone().requires_grad_() for t in qkv]
    y, _ = layer(*leaves, train=True)
    up = r(*y.shape)
    got = torch.autograd.grad(y, (*leaves, w), up)
    dbl = [t.double().requires_grad_() for t in (*qkv, w.detach())]
    ref = plain(*dbl)
    want = torch.autograd.grad(ref, dbl, up.double())
    # errors of some hundred steps of the operators before pass through a norm that divides by a head's width: 2^-24 * 2000 of the size
    for a, b in zip((y, *got), (ref, *want)):
        assert float((a.double() - b).detach().abs().max()) <= 2000 * R.F * float(b.detach().abs().max())
    out, state = layer(*[t[:, :50] for t in qkv])
    rows = [out]
    for n in range(50, N):
        o, state = layer(*[t[:, n:n + 1] for t in qkv], start=n, state=state)
        rows.append(o)
    assert float((torch.cat(rows, 1).double() - ref).detach().abs().max()) <= 2000 * R.F * float(ref.detach().abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(128, 32), (64, 128), (32, 64)])
def test_other_widths(dev, dk, dv, dtype):
    """The pairs of widths that the sizes leave out, in one and in several segments."""
    for N in (5, 75, 500):
        check(*make(dev, 2, N, 2, dk, dv, dtype, seed=N + dk))
        args, ups = make(dev, 2, N, 2, dk, dv, dtype, seed=N)
        check(args, ups, lens=[N - 3, N // 2])


@pytest.mark.parametrize("N", [6, 200])
def test_broadcast_batches_and_tokens(dev, N):
    """Zero strides along the batch and along the tokens."""
    r = gen(21, dev)
    q, k, v = r(1, N, 2, 32).expand(3, N, 2, 32), r(3, 1, 2, 32).expand(3, N, 2, 32), r(1, 1, 2, 64).expand(3, N, 2, 64)
    (_, _, _, g, s), _ = make(dev, 3, 1, 2, 32, 64, "f32", seed=N)
    check((q, k, v, g, s), (r(3, N, 2, 64), r(3, 2, 32, 64)), label="broadcast")


def test_a_captured_training_step(dev):
    """Forward and backward captured together, replayed on new inputs, against eager steps."""
    (q, k, v, g, _), (dout, _) = make(dev, 1, 150, 2, 32, 32, "f32", seed=3, state=False)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]

    def step(xs):
        y = P.decay_attention(*xs, g)
        y = P.group_norm(y.flatten(-2), 2, per_token=True).unflatten(-1, (2, 32))
        return torch.autograd.grad(y, xs, dout)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step(leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = step(leaves)
    r = gen(5, dev)
    for _ in range(3):
        with torch.no_grad():
            for t in leaves:
                t.copy_(r(*t.shape))
        graph.replay()
        eager = step([t.detach().clone().requires_grad_() for t in leaves])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(grads, eager))
