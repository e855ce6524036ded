"""Group norm on the GPU against tests/norm_ref.py's 64-bit values and its bounds (element by element: |gpu - ref| <= bound)."""
import math

import pytest
import torch

import paper_2201_02767_amd as P
from tests import norm_ref as R
from tests.test_gpu_dense import DT, announce, dev, gen, within            # noqa: F401

pytestmark = pytest.mark.gpu


def make(dev, shape, dtype, seed=0, affine=True, params=None):
    r = gen(seed, dev)
    C = shape[-1]
    x = (r(*shape) * (0.5 + r(C).abs()) + r(C)).to(DT[dtype])
    w, b = ((1 + 0.3 * r(C)).to(params or DT[dtype]), (0.3 * r(C)).to(params or DT[dtype])) if affine else (None, None)
    return x, w, b, r(*shape).to(DT[dtype])


def check(x, groups, w, b, dy, **how):
    announce(f"group_norm x {tuple(x.shape)} {x.stride()} {x.dtype} groups {groups} params {None if w is None else w.dtype} {how}")
    want = R.group_norm(x, groups, w, b, dy=dy, **how)
    y = P.group_norm(x, groups, w, b, **how)
    torch.cuda.synchronize()
    within("y", y, want["y"])
    leaves = [t.detach().requires_grad_() if t is not None else None for t in (x, w, b)]
    y2 = P.group_norm(leaves[0], groups, *leaves[1:], **how)
    given = [t for t in leaves if t is not None]
    grads = torch.autograd.grad(y2, given, dy)
    torch.cuda.synchronize()
    assert torch.equal(y2, y)
    for n, t in zip([n for n, t in zip(("dx", "dweight", "dbias"), leaves) if t is not None], grads):
        within(n, t, want[n])
    return y


SHAPES = [  # shape, groups
    ((1, 1, 1), 1), ((1, 1, 8), 1), ((2, 3, 6), 3), ((1, 5, 90), 6), ((2, 7, 9, 32), 4), ((3, 130, 15), 5), ((1, 1000, 24), 24),
    ((2, 31, 33, 64), 32), ((1, 700, 160), 32), ((1, 50, 2048), 16), ((2, 20, 5000), 5), ((1, 9, 4104), 1), ((1, 4, 9000), 3),
    ((1, 3, 8192), 2), ((40, 2, 16), 2), ((1, 3, 1001), 1), ((1, 5, 5005), 5),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("shape,groups", SHAPES, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_sizes(dev, shape, groups, per_token, dtype):
    check(*(lambda x, w, b, dy: (x, groups, w, b, dy))(*make(dev, shape, dtype, seed=sum(shape))), per_token=per_token, act="silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("per_token", [False, True])
def test_activations_and_weights(dev, act, per_token, dtype):
    for params in (torch.float32, DT[dtype]):
        x, w, b, dy = make(dev, (2, 100, 96), dtype, seed=1, params=params)
        check(x, 12, w, b, dy, act=act, per_token=per_token)
        check(x, 12, w, None, dy, act=act, per_token=per_token)
        check(x, 12, None, b, dy, act=act, per_token=per_token)
    check(x, 12, None, None, dy, act=act, per_token=per_token, eps=0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
def test_views(dev, per_token, dtype):
    """Channels of a wider tensor, every alignment of their start, a transposed batch, a broadcast one."""
    r = gen(3, dev)
    wide = r(3, 50, 200).to(DT[dtype])
    dy = r(3, 50, 48).to(DT[dtype])
    for start in (0, 1, 2, 4, 8):
        check(wide[..., start:start + 48], 6, None, None, dy, per_token=per_token, act="silu")
    check(wide.transpose(0, 1)[:, :, :48], 6, None, None, r(50, 3, 48).to(DT[dtype]), per_token=per_token)
    check(wide[:1, :, :48].expand(3, 50, 48), 6, None, None, dy, per_token=per_token)
    odd = r(3, 50, 49).to(DT[dtype])
    check(odd[..., :48], 6, None, None, dy, per_token=per_token)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_hard_statistics(dev, dtype):
    """Means far from zero, a first token unlike the others, equal values, many slabs, large values."""
    r = gen(4, dev)
    x, w, b, dy = make(dev, (2, 900, 32), dtype, seed=5)
    check((x.float() + 300).to(DT[dtype]), 4, w, b, dy, act="silu")
    y = x.clone()
    y[:, :1] += 1000
    check(y, 4, w, b, dy)
    check(y, 4, w, b, dy, per_token=True)
    check(torch.full_like(x, 3.25), 4, w, b, dy, act="gelu")
    check((x.float() * 1e15).to(DT[dtype]), 4, w, b, dy)
    x, w, b, dy = make(dev, (1, 20000, 16), dtype, seed=6)
    check(x, 2, w, b, dy, act="silu")


def test_runs_are_identical_and_streams_and_graphs(dev):
    x, w, b, dy = make(dev, (2, 3000, 64), "bf16", seed=7)
    for per_token in (False, True):
        run = lambda x, w, b: P.group_norm(x, 8, w, b, act="silu", per_token=per_token)
        leaves = [t.detach().clone().requires_grad_() for t in (x, w, b)]
        step = lambda: (lambda y: (y.detach(), *torch.autograd.grad(y, leaves, dy)))(run(*leaves))
        first = step()
        for _ in range(3):
            assert all(torch.equal(p, q) for p, q in zip(first, step()))
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = run(x, w, b)
        side.synchronize()
        assert torch.equal(got, first[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run(x, w, b)
        r = gen(8, dev)
        for _ in range(4):
            x.copy_(r(*x.shape))
            graph.replay()
            eager = run(x, w, b)
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
        x.copy_(leaves[0].detach())


def test_two_streams_at_once(dev):
    xs = [make(dev, (2, 20000, 64), "bf16", seed=i)[0] for i in range(2)]
    want = [P.group_norm(x, 8, act="silu") for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], [[], []]
    for _ in range(5):
        for st, x, res in zip(streams, xs, got):
            with torch.cuda.stream(st):
                res.append(P.group_norm(x, 8, act="silu"))
    torch.cuda.synchronize()
    assert all(torch.equal(w, y) for w, res in zip(want, got) for y in res)


def test_empty_calls(dev):
    for shape in ((0, 5, 8), (3, 0, 8), (2, 0, 4, 8)):
        for per_token in (False, True):
            x, w, b = torch.zeros(shape, device=dev).requires_grad_(), torch.ones(8, device=dev).requires_grad_(), torch.ones(8, device=dev).requires_grad_()
            y = P.group_norm(x, 2, w, b, per_token=per_token)
            y.sum().backward()
            assert y.shape == shape and x.grad.shape == shape and not w.grad.any() and not b.grad.any()


def test_autograd(dev):
    x, w, b, dy = make(dev, (2, 30, 32), "f32", seed=9)
    want = R.group_norm(x, 4, w, b, dy=dy, act="gelu")
    for use in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 0)):
        for per_token in (False, True):
            want = R.group_norm(x, 4, w, b, dy=dy, act="gelu", per_token=per_token)
            leaves = [t.detach().clone().requires_grad_(bool(u)) for t, u in zip((x, w, b), use)]
            P.group_norm(leaves[0], 4, *leaves[1:], act="gelu", per_token=per_token).backward(dy)
            for n, t, u in zip(("dx", "dweight", "dbias"), leaves, use):
                assert (t.grad is not None) == bool(u)
                if u:
                    within(n, t.grad, want[n])
    a = x.detach().requires_grad_()
    (P.group_norm(a, 4).sum() * 2).backward()
    within("dx", a.grad, R.group_norm(x, 4, dy=torch.full_like(x, 2.0))["dx"])
    d, = torch.autograd.grad(P.group_norm(a, 4), a, dy, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()


def test_gradients_against_differences(dev):
    x, w, b, dy = make(dev, (2, 40, 24), "f32", seed=10)
    leaves = [t.detach().clone().requires_grad_() for t in (x, w, b)]
    for per_token in (False, True):
        grads = torch.autograd.grad(P.group_norm(leaves[0], 3, *leaves[1:], act="silu", per_token=per_token), leaves, dy)
        r = gen(11, dev)
        for i, grad in enumerate(grads):
            e, f, h = r(*leaves[i].shape), [], 2.0 ** -7
            for sign in (h, -h):
                t = [p.detach().clone() for p in leaves]
                t[i] += sign * e
                f.append(float((P.group_norm(t[0], 3, t[1], t[2], act="silu", per_token=per_token).double() * dy).sum()))
            slope, got = (f[0] - f[1]) / (2 * h), float((grad.double() * e).sum())
            # 1920 results in two sums, each up to 40 f off, over the step, and the third derivative's h^2 of as many terms of about one
            assert abs(slope - got) <= 2 * 1920 * 40 * R.F / (2 * h) + h * h * 1920, (i, slope, got)


def test_offsets_past_32_bits(dev):
    """2^31 elements and more: the last tokens' results, per token and over the last of two batch elements."""
    C = 2048
    announce("group_norm past 2^31 elements")
    x = torch.empty(2, (1 << 19) + 40, C, device=dev, dtype=torch.bfloat16).normal_()
    y = P.group_norm(x, 16, per_token=True)
    within("y", y[1, -30:], tuple(t[0] for t in R.group_norm(x[1:, -30:], 16, per_token=True)["y"]))
    del y
    y = P.group_norm(x, 16)
    xs = x[1].view(-1, 16, 128)[:, 3].double()
    mean, var = float(xs.mean()), float(xs.var(correction=0))
    n = (xs[-30:] - mean) / math.sqrt(var + 1e-5)
    off = (y[1, -30:].view(30, 16, 128)[:, 3].double() - n).abs()
    # a mean and variance of 2^26 values in slabs of 2^11 tokens, 2^6 of them after each other in a sum, and 2^-8 for the result
    assert bool((off <= 2.0 ** -8 * n.abs() + 2.0 ** -12).all())


def test_refusals(dev):
    z = lambda *s, t=torch.float32: torch.zeros(*s, device=dev, dtype=t)
    x, w = z(2, 6, 8), z(8)
    for kw in (dict(groups=3), dict(groups=0), dict(groups=2.0), dict(act="tanh"), dict(eps=-1.0), dict(eps=math.nan), dict(x=z(2, 8)),
               dict(x=x.cpu()), dict(x=x.double()), dict(x=z(2, 8, 6).transpose(1, 2)), dict(weight=z(7)), dict(weight=z(8).cpu()),
               dict(weight=z(8, t=torch.bfloat16)), dict(weight=z(16)[::2]), dict(x=z(2, 5, 8, 8)[:, :, :3])):
        with pytest.raises(ValueError):
            P.group_norm(**{**dict(x=x, groups=2, weight=w), **kw})
    with pytest.raises(ValueError):
        P.group_norm(x.to(torch.bfloat16), 2, w, z(8, t=torch.bfloat16))
    with pytest.raises(TypeError):
        P.group_norm([1.0], 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("shape,groups", [((2, 3, 600), 300), ((1, 2, 1200), 1200), ((1, 6, 8200), 1), ((1, 5, 2501), 1), ((2, 40, 9), 9),
                                          ((1, 70, 4400), 1100), ((3, 1, 2048), 16)],
                         ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_many_and_wide_groups(dev, shape, groups, per_token, dtype):
    """More groups than a workgroup has lanes for, and groups wider than a workgroup."""
    x, w, b, dy = make(dev, shape, dtype, seed=sum(shape))
    check(x, groups, w, b, dy, per_token=per_token, act="gelu")
