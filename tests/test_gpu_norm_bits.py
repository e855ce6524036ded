"""Group norm over maps on the GPU where statistics lose bits, against tests/norm_bits.py's bounds."""
import math
import sys

import pytest
import torch

import paper_2201_02767_amd as P
from tests import norm_bits as R
from tests import norm_ref as Ref
from tests.test_gpu_dense import announce, dev, gen, within                # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [0.0, 30.0, 1000.0, -1e5])
@pytest.mark.parametrize("C,groups", [(16, 2), (16, 16), (64, 1)])
def test_a_slab_unlike_the_others(dev, C, groups, apart):
    """256 slabs of 1024 tokens (C = 64: 4096), of which the first, or another one, lies apart."""
    N = 256 * 16 * 1024 // C * (4 if C == 64 else 1)
    r = gen(41, dev)
    announce(f"group_norm, {N} tokens of {C} channels, {groups} groups, a slab {apart} apart")
    for at in (0, 77):
        x = r(1, N, C)
        x[:, at * N // 256:(at + 1) * N // 256] += apart
        within("y", P.group_norm(x, groups), R.group_norm(x, groups, N * C // 256 // 4096, N // 256))


EQUAL = [((1, 5000, 90), 6), ((2, 700, 64), 8), ((1, 9, 4104), 1), ((1, 6, 20000), 1), ((3, 40, 96), 1), ((1, 30000, 5), 5)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("shape,groups", EQUAL, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_equal_values_are_the_bias(dev, shape, groups, per_token, dtype):
    """A group of equal values far from zero, which 1 / sqrt(eps) makes of any rounding of its mean: over maps the mean is exact. Per token
    distances from the first mean, 100 f of it at most (as many values at most follow each other in a sum), are corrected by their mean, 100 f
    of them off: (100 f)^2 |x| r. Their mean square, less that of their mean, is 200 f (100 f x)^2 off nothing."""
    r = gen(43, dev)
    C = shape[-1]
    b = r(C).to(dtype)
    announce(f"group_norm of equal values {shape} {groups} {per_token} {dtype}")
    for value in (1000.1, -1e4 / 3, 2.0 ** -10 / 3):
        x = torch.full(shape, value, device=dev, dtype=dtype)
        w, value = (1 + 0.3 * r(C)).to(dtype), float(x[0, 0, 0])
        y = P.group_norm(x, groups, w, b, per_token=per_token)
        if per_token:
            off = (100 * R.F) ** 2 * abs(value) / 1e-5 ** 0.5 * w.double().abs()
            u = torch.finfo(dtype).eps / 2
            assert bool(((y.double() - b.double()).abs() <= off + u * (b.double().abs() + off)).all()), value
        else:
            assert torch.equal(y, b.expand(shape)), value
        # and dx is r (dn - mean dn): the group's gradients without their mean
        x.requires_grad_()
        dy = r(*shape).to(dtype)
        dx, = torch.autograd.grad(P.group_norm(x, groups, w, b, per_token=per_token), x, dy)
        dn = (dy.double() * w.double()).unflatten(-1, (groups, -1))
        over = (3,) if per_token else (1, 3)
        want = ((dn - dn.mean(over, keepdim=True)) / 1e-5 ** 0.5).flatten(-2)
        # (r by 4 f and eps as a float; the sum of dn by a step for each of its terms in a row, at most 100 here)
        dr = 8 * R.F + per_token * 100 * R.F * (100 * R.F * value) ** 2 / 1e-5
        bound = (torch.finfo(dtype).eps / 2 + dr) * want.abs() + 108 * R.F * (dn.abs() + dn.abs().mean(over, keepdim=True)).flatten(-2) / 1e-5 ** 0.5
        within("dx", dx, (want, bound))


@pytest.mark.parametrize("shift", [0.0, 300.0, -5000.0])
def test_means_far_from_zero(dev, shift):
    r = gen(44, dev)
    announce(f"group_norm, means of {shift}")
    x = r(1, 262144, 16) + shift
    within("y", P.group_norm(x, 2), R.group_norm(x, 2, 4, 1024))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("shape,groups", [((2, 900, 32), 4), ((2, 50, 90), 6), ((2, 7, 9000), 2)],
                         ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_what_is_not_finite_stays_in_its_group(dev, shape, groups, per_token, value, dtype):
    r = gen(45, dev)
    C = shape[-1]
    x, w, b, dy = r(*shape).to(dtype), r(C).to(dtype), r(C).to(dtype), r(*shape).to(dtype)
    announce(f"group_norm with {value} in a group {shape} {groups} {per_token} {dtype}")
    split = lambda t: t.detach().unflatten(-1, (groups, -1))
    for act in ("none", "relu", "silu", "gelu"):
        both = []
        for bad in (False, True):
            leaves = [t.clone() for t in (x, w, b)]
            if bad:
                leaves[0][1, 3, C // groups + 1] = value
            leaves = [t.requires_grad_() for t in leaves]
            y = P.group_norm(leaves[0], groups, *leaves[1:], act=act, per_token=per_token)
            both.append([split(t) for t in (y, *torch.autograd.grad(y, leaves, dy))])
        clean, got = both
        hit = torch.zeros(*shape[:-1], groups, dtype=torch.bool, device=dev)
        hit[1, 3 if per_token else slice(None), 1] = True
        for n in (0, 1):
            assert bool(got[n][hit].isnan().all()) and torch.equal(got[n][~hit], clean[n][~hit]), (act, n)
        group = torch.arange(groups, device=dev) == 1
        assert bool(got[2][group].isnan().all()) and all(torch.equal(got[n][~group], clean[n][~group]) for n in (2, 3)), act


@pytest.mark.parametrize("shape", [(1, 300, 16), (1, 9000, 6), (2, 3, 5000)], ids=str)
@pytest.mark.parametrize("power,mean", [(70, 0.0), (70, 3.0), (100, 3.0), (100, -1.7)])
def test_squares_that_overflow(dev, power, mean, shape):
    """Distances of 2^70 and 2^100: an infinite variance, the bias, and no gradient of x."""
    r = gen(47, dev)
    announce(f"group_norm, values of 2^{power}, {mean} {shape}")
    x = ((r(*shape) + mean) * 2.0 ** power).requires_grad_()
    b = r(shape[-1])
    for per_token in (False, True):
        y = P.group_norm(x, 2 if shape[-1] < 5000 else 1, None, b, per_token=per_token)
        assert torch.equal(y, b.expand(shape))
        assert not bool(torch.autograd.grad(y, x, r(*shape))[0].any())


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("shape,groups", [((3, 5063, 90), 6), ((2, 40, 2048), 2), ((1, 60, 5000), 1), ((1, 40000, 32), 4)],
                         ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else str(s))
def test_fp32_keeps_its_bits(dev, shape, groups, per_token, act):
    """The root mean square of the errors, relative to the values'. f = 2^-24, independent roundings of 0.4 f: x - mean and what the mean is off,
    0.7 f; r, 1 f; n, z and the products around them five roundings, 0.9 f; an activation or its slope, 2 f. So y within 2.5 f; dz and dn, and the sums that
    dx takes from them (whose terms' errors differ in sign), 3 f; the weights' gradients, with the 40 additions at most that a value passes,
    4 f. Twice that are the limits. Statistics of 16 bits, or a mean that keeps 2^-20 of a group's width, are off by more than 16."""
    r = gen(46, dev)
    C = shape[-1]
    x, w, b, dy = r(*shape) * (0.5 + r(C).abs()) + r(C), 1 + 0.2 * r(C), 0.2 * r(C), r(*shape)
    announce(f"group_norm, fp32 bits {shape} {groups} {per_token} {act}")
    want = Ref.group_norm(x, groups, w, b, act=act, per_token=per_token, dy=dy)
    leaves = [t.requires_grad_() for t in (x, w, b)]
    y = P.group_norm(x, groups, w, b, act=act, per_token=per_token)
    for (n, t), limit in zip(zip(("y", "dx", "dweight", "dbias"), (y.detach(), *torch.autograd.grad(y, leaves, dy))), (5.0, 6.0, 8.0, 8.0)):
        off = float((t.double() - want[n][0]).square().mean().sqrt() / want[n][0].square().mean().sqrt()) / R.F
        print(f"{n}: {off:.2f} f", file=sys.stderr)
        assert off <= limit, (n, off)
