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
    g = -torch.rand(heads, device=dev, generator=None) * 0 - torch.logspace(-0.3, -3.0, heads, device=dev)
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
