"""Linear attention with a decay on the GPU: its bits, and its chunks and segments where they are many."""
import ctypes
import math
import sys

import pytest
import torch

import paper_2201_02767_amd as P
from paper_2201_02767_amd.decay import _decay_args
from tests import decay_bits as Bits
from tests import decay_ref as R
from tests.test_gpu_decay import check, make
from tests.test_gpu_dense import DT, announce, dev, gen, i32, within       # noqa: F401

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


def chunks(args, back):
    """(segments, chunks of 32 tokens in a segment) of a call, from the states that its workspace has room for."""
    q, k, v, g, _ = args
    a, _, (B, heads, dk, dv) = _decay_args(q, k, v, g, None, None, None)
    name = "qta_decay_attn_backward_workspace_bytes" if back else "qta_decay_attn_workspace_bytes"
    one = B * heads * dk * dv * 4 * (2 if back else 1)
    segs = max(1, getattr(P.lib(), name)(ctypes.byref(a)) // one)
    tokens = -(-q.shape[1] // segs)
    return segs, -(-tokens // 32)


# widths, and batch elements, heads and tokens, that give segments of many chunks, with four, three and two chunks in LDS at a time
MANY = [("bf16", 32, 32, 4, 16, 32, 1171), ("bf16", 64, 64, 4, 16, 16, 1171), ("bf16", 64, 128, 3, 8, 16, 900), ("bf16", 32, 128, 4, 16, 16, 1171),
        ("bf16", 128, 32, 2, 16, 32, 700), ("bf16", 128, 128, 2, 8, 16, 777), ("f32", 32, 32, 4, 16, 32, 1171), ("f32", 32, 64, 3, 16, 16, 900),
        ("f32", 64, 64, 2, 16, 16, 777), ("f32", 128, 128, 2, 8, 16, 777)]


@pytest.mark.parametrize("dtype,dk,dv,depth,B,heads,N", MANY, ids=lambda x: str(x))
def test_segments_of_many_chunks(dev, dtype, dk, dv, depth, B, heads, N):
    """Every place in LDS is used again and again, in several segments, forward and backward, with decays that remember whole segments (e^-1.6 over
    1171 tokens and up), and lengths within and on the borders of segments and chunks."""
    assert depth == (4 if 4 * (2 * dk + dv) * 32 * (2 if dtype == "bf16" else 4) <= 49152 else
                     3 if 3 * (2 * dk + dv) * 32 * (2 if dtype == "bf16" else 4) <= 49152 else 2)
    (q, k, v, _, s), ups = make(dev, B, N, heads, dk, dv, dtype, seed=N + dk)
    g = -torch.logspace(-4.0, -2.9, heads, device=dev)
    args = (q, k, v, g, s)
    for back in (False, True):
        segs, each = chunks(args, back)
        assert segs >= (1 if back else 2) and each >= 2 * depth + 1, (back, segs, each)
    check(args, ups, label="many chunks")
    lens = [N, 0, N - 1, 1, 33, N // 2, N // 2 // 32 * 32, 321, 320][:B]
    check(args, ups, label="many chunks", lens=lens + [N - 5] * (B - len(lens)))


@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 128), (128, 128)])
@pytest.mark.parametrize("B,N", [(2, 60), (1, 300), (2, 5000)])
def test_returned_states_keep_24_bits(dev, B, N, dk, dv):
    """States and their gradients from bf16 tokens, whose weighted values are taken as three bf16 terms, and not as two."""
    (q, k, v, _, s), (dout, dlast) = make(dev, B, N, 4, dk, dv, "bf16", seed=N)
    g = torch.tensor(Bits.DECAYS, device=dev)
    announce(f"decay_attn, bits of the states {B} {N} {dk} {dv}")
    want = R.decay_attention(q, k, v, g, state=s, dout=dout, dstate_out=dlast)
    _, last = P.decay_attn(q, k, v, g, state=s, return_state=True)
    dstate = P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast)[3]
    for n, t in (("state", last), ("dstate", dstate)):
        off = Bits.rms(t.double(), want[n][0])
        print(f"{n}: {[round(x, 2) for x in off]} f", file=sys.stderr)
        assert max(off) <= Bits.STATE, (n, off)


@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("B,N", [(2, 12), (2, 60), (1, 300), (2, 3000)])
def test_fp32_keeps_its_bits(dev, B, N, dk, dv):
    """The root mean square of the errors, where the bounds element by element are worst cases that leave room for products of far fewer bits. f = 2^-24,
    independent roundings of 0.4 f: a score and a row of the state's product sum up to 128 terms, 4.5 f each; a weight, a product of two to
    four powers and a rounded exponent, is off by 2 f; a state is rounded with every chunk that it remembers, and in the scan, 2.2 f each as in
    tests/decay_bits.py. Together 7.5 f, and twice that is the limit. Products of 16 bits are off by 2^-17 = 128 f, and of bf16 terms by
    2^-16."""
    (q, k, v, _, s), (dout, dlast) = make(dev, B, N, 4, dk, dv, "f32", seed=N + 1)
    g = torch.tensor(Bits.DECAYS, device=dev)
    announce(f"decay_attn, fp32 bits {B} {N} {dk} {dv}")
    want = R.decay_attention(q, k, v, g, state=s, dout=dout, dstate_out=dlast)
    got = (*P.decay_attn(q, k, v, g, state=s, return_state=True), *P.decay_attn_backward(q, k, v, g, dout, state=s, dstate_out=dlast))
    for n, t in zip(("out", "state", "dq", "dk", "dv", "dstate"), got):
        off = Bits.rms(t.double(), want[n][0], 2 if n in ("out", "dq", "dk", "dv") else 1)
        print(f"{n}: {[round(x, 1) for x in off]} f", file=sys.stderr)
        assert max(off) <= 15.0, (n, off)
