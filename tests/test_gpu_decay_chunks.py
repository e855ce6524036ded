"""Linear attention with a decay on the GPU: its bits, and its chunks and segments where they are many."""
import math

import pytest
import torch

import paper_2201_02767_amd as P
from tests import decay_ref as R
from tests.test_gpu_decay import check, make
from tests.test_gpu_dense import announce, dev, gen, within       # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(32, 64), (128, 128)])
@pytest.mark.parametrize("N", [5, 40, 130, 600, 3000])
def test_results_are_the_same_with_and_without_a_state(dev, N, dk, dv, dtype):
    """The bits of a result do not depend on whether the state, or its gradient, is asked for."""
    (q, k, v, g, s), (dout, dlast) = make(dev, 2, N, 2, dk, dv, dtype, seed=N)
    announce(f"decay_attn with and without the state {N} {dk} {dv} {dtype}")
    assert torch.equal(P.decay_attn(q, k, v, g, state=s), P.decay_attn(q, k, v, g, state=s, return_state=True)[0])
    zero = torch.zeros_like(s)
    assert torch.equal(P.decay_attn(q, k, v, g), P.decay_attn(q, k, v, g, state=zero, return_state=True)[0])
    without = P.decay_attn_backward(q, k, v, g, dout, dstate_out=dlast)
    assert without[3] is None
    given = P.decay_attn_backward(q, k, v, g, dout, state=zero, dstate_out=dlast)
    assert all(torch.equal(a, b) for a, b in zip(without[:3], given[:3]))


@pytest.mark.parametrize("N,d", [(1, 128), (17, 32)])
def test_as_many_heads_as_the_header_names(dev, N, d):
    """2^22 (batch, head) pairs, forward and backward, on a sample of the batch elements."""
    B, heads = 1 << 18, 16
    announce(f"decay_attn {B} x {heads} heads of {d}, {N} tokens")
    q, k, v, dout = (torch.empty(B, N, heads, d, device=dev, dtype=torch.bfloat16).normal_() for _ in range(4))
    g = -torch.logspace(-0.3, -3.0, heads, device=dev)
    out = P.decay_attn(q, k, v, g)
    grads = P.decay_attn_backward(q, k, v, g, dout)
    torch.cuda.synchronize()
    for b in (0, 99_999, B - 1):
        some = [t[b:b + 1] for t in (q, k, v)]
        want = R.decay_attention(*some, g, dout=dout[b:b + 1])
        for n, t in zip(("out", "dq", "dk", "dv"), (out, *grads)):
            within(n, t[b:b + 1], want[n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("N", [16, 200, 3000])
def test_what_is_not_finite_stays_near_its_token(dev, N, value, dtype):
    """A NaN or an infinity in one token reaches what depends on it, and in calls of more than 16 tokens the rest of its chunk of 32; other heads and
    batch elements, and earlier chunks, keep their bits."""
    (q, k, v, g, s), (dout, _) = make(dev, 2, N, 2, 32, 64, dtype, seed=N)
    announce(f"decay_attn with {value} in a token of {N} {dtype}")
    clean, last = P.decay_attn(q, k, v, g, state=s, return_state=True)
    t = N - 7
    first = t if N <= 16 else t // 32 * 32
    for x in (q, k, v):
        old = x[1, t, 0, 5].clone()
        x[1, t, 0, 5] = value
        out, state = P.decay_attn(q, k, v, g, state=s, return_state=True)
        assert torch.equal(out[0], clean[0]) and torch.equal(out[1, :, 1], clean[1, :, 1]) and torch.equal(out[1, :first], clean[1, :first])
        assert not bool(torch.isfinite(out[1, t, 0]).all())
        assert torch.equal(state[0], last[0]) and torch.equal(state[1, 1], last[1, 1])
        x[1, t, 0, 5] = old
    grads = P.decay_attn_backward(q, k, v, g, dout, state=s)
    dout[1, t, 0, 5] = value
    for a, b in zip(P.decay_attn_backward(q, k, v, g, dout, state=s)[:3], grads):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1, :, 1], b[1, :, 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [30, 4000])
def test_growth(dev, N, dtype):
    """A positive log decay of 70 / N: e^70 over the call, which multiplies zeros (no state, and no token before the last quarter) and numbers. In one
    segment and in many."""
    (q, k, v, _, _), (dout, _) = make(dev, 1, N, 3, 32, 32, dtype, seed=N, state=False)
    g = torch.tensor([70.0 / N, 35.0 / N, 0.0], device=dev)
    check((q, k, v, g, None), (dout, None), label="growth")
    for t in (k, v):
        t[:, :3 * N // 4] = 0
    check((q, k, v, g, None), (dout, None), label="growth of zeros")
