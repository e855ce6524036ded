"""Group norm on the GPU against tests/norm_ref.py's 64-bit values and its bounds (element by element: |gpu - ref| <= bound)."""
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
