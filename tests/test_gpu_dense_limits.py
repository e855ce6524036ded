"""Rotary positions and differential attention on the GPU at the border of what they take: the largest sizes, calls that are
refused, and what lies in places that nothing may use. Values against tests/dense_ref.py, as in test_gpu_dense.py."""
import math
import sys

import pytest
import torch
from torch.autograd import forward_ad

import paper_2201_02767_amd as P
from tests import dense_ref as R
from tests.test_gpu_dense import announce, check, dev, gen, make, within  # noqa: F401

pytestmark = pytest.mark.gpu


def test_rotary_of_more_workgroups_than_a_launch_takes(dev):
    """A token a workgroup, and more tokens than the 2^24 - 1 workgroups of 256 threads that one launch can have: around that
    border, and at the end."""
    N, d, rot = (1 << 24) + 300, 514, 4
    announce(f"rotary {N} x {d}")
    x = gen(71, dev)(1, 1, 1, d).bfloat16()
    freqs = P.rotary_freqs(rot, device=dev)
    y = P.rotary(x.expand(1, N, 1, d), freqs)
    for at in (0, (1 << 24) - 50, N - 100):
        p = torch.arange(at, at + 100, device=dev)[None, :, None]
        within(f"tokens from {at} on", y[:, at:at + 100], R.rotary(x.expand(1, 100, 1, d), freqs, p))
        assert torch.equal(y[:, at:at + 100, :, rot:], x[..., rot:].expand(1, 100, 1, d - rot))


def test_rotary_positions_that_are_refused(dev):
    x, f = torch.zeros(1, 3, 4, 2, 32, device=dev), P.rotary_freqs(32, axes=2, device=dev)
    for start in (1, 2 ** 32 + 5):
        with pytest.raises(ValueError, match="start"):
            P.rotary(x, f, start=start)                     # rows and columns have no start
    assert P.rotary(x, f, axes=1, start=5).shape == x.shape
    wide = torch.zeros(1, 1, 1, 32, device=dev).expand(1, 2 ** 32 + 12, 1, 32)
    with pytest.raises(ValueError, match="2\\^31"):
        P.rotary(wide, P.rotary_freqs(32, device=dev))


def test_in_place_tensors_that_overlap(dev):
    """Refused; parts that lie apart are turned."""
    fused = gen(72, dev)(2, 11, 7, 64)
    f = P.rotary_freqs(64, device=dev)
    before = fused.clone()
    for x, k in ((fused, fused), (fused[:, :, :4], fused[:, :, 3:]), (fused[:, :10], fused[:, 1:])):
        with pytest.raises(ValueError, match="share memory"):
            P.rotary(x, f, k=k, inplace=True)
    with pytest.raises(ValueError, match="share memory"):
        P.rotary(fused.as_strided((1, 9, 2, 64), (0, 64, 64, 1)), f, inplace=True)
    assert torch.equal(fused, before)
    want = P.rotary(fused[:, :, 1::2], f), P.rotary(fused[:, :, ::2], f)
    P.rotary(fused[:, :, 1::2], f, k=fused[:, :, ::2], inplace=True)
    assert torch.equal(fused[:, :, 1::2], want[0]) and torch.equal(fused[:, :, ::2], want[1])


def test_frequencies_that_require_gradients(dev):
    x, f = gen(73, dev)(1, 4, 2, 32), P.rotary_freqs(32, device=dev)
    want = P.rotary(x, f)
    for t in (x, x.clone().requires_grad_()):
        with pytest.raises(ValueError, match="freqs"):
            P.rotary(t, f.clone().requires_grad_())
    with torch.no_grad():
        assert torch.equal(P.rotary(x, f.clone().requires_grad_()), want)


def test_forward_mode_derivatives(dev):
    q, k, v, lam, _ = make(dev, 1, 5, 6, 2, 1, 32, "f32")
    f = P.rotary_freqs(32, device=dev)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        for call in (lambda: P.rotary(dual, f), lambda: P.rotary(dual, f, inverse=True), lambda: P.diff_attention(dual, k, v, lam)):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()
        assert torch.equal(P.diff_attention(q, k, v, lam), P.diff_attn(q, k, v, lam))


def test_scales_that_are_refused(dev):
    """None alone stands for 1/sqrt(d): a scale of zero or below, or one that is no number, is no other name of it."""
    q, k, v, lam, do = make(dev, 1, 5, 6, 2, 1, 32, "f32")
    _, kept = P.diff_attn(q, k, v, lam, keep=True)
    for scale in (0.0, -0.5, math.nan, math.inf, 1e-45, 1e-60, 1e39):
        for call in (lambda: P.diff_attn(q, k, v, lam, scale=scale), lambda: P.diff_attention(q.clone().requires_grad_(), k, v, lam, scale=scale),
                     lambda: P.diff_attn_backward(q, k, v, lam, kept, do, scale=scale)):
            with pytest.raises(ValueError, match="scale"):
                call()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_and_large_scales(dev, dtype):
    args = make(dev, 1, 40, 300, 2, 1, 32, dtype, seed=74)
    for scale in (2.0 ** -96, 1e-12, 3.0):
        check(dev, *args, scale=scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64])
def test_rows_that_see_no_key_may_hold_anything(dev, d, dtype):
    """Queries before the first key (left padding) and those of elements without keys: NaN and infinities in their q, dout and
    weight give zeros and reach no gradient, whether keys and rows are taken whole or in parts."""
    for shape, lens, pos in (((4, 70, 90, 4, 2), [90, 50, 0, 90], [-40, -69, 3, -200]), ((3, 40, 2600, 4, 2), [2600, 31, 0], [-33, -9, 0]),
                             ((3, 700, 130, 8, 1), [130, 9, 0], [-590, -699, 0]), ((3, 1, 700, 4, 1), [700, 0, 650], [-1, 0, 699])):
        q, k, v, lam, do = make(dev, *shape, d, dtype, seed=75, token_lam=True)
        rows = [t.clone() for t in (q, lam, do)]
        for b, (n, p) in enumerate(zip(lens, pos)):
            empty = shape[1] if n == 0 else min(max(-p, 0), shape[1])
            for t, x in ((q, math.nan), (lam, math.inf), (do, -math.inf)):
                t[b, :empty] = x
                t[b, :empty // 2] = math.nan
        announce(f"rows without a key {shape} {d} {dtype}")
        how = dict(causal=True, lens=torch.tensor(lens, dtype=torch.int32, device=dev), q_pos=torch.tensor(pos, dtype=torch.int32, device=dev))
        ref = R.diff_attention(rows[0], k, v, rows[1], dout=rows[2], causal=True, lens=lens, q_pos=pos)
        out, kept = P.diff_attn(q, k, v, lam, keep=True, **how)
        got = (P.diff_attn(q, k, v, lam, **how), out, *P.diff_attn_backward(q, k, v, lam, kept, do, **how))
        torch.cuda.synchronize()
        for n, t in zip(("out", "out", "dq", "dk", "dv", "dlam"), got):
            within(n, t, ref[n])
        # one weight a head: no sum over the rows takes them in
        one = rows[1][0, -1].clone()
        ref = R.diff_attention(rows[0], k, v, one, dout=rows[2], causal=True, lens=lens, q_pos=pos)
        _, kept = P.diff_attn(q, k, v, one, keep=True, **how)
        for n, t in zip(("dq", "dk", "dv", "dlam"), P.diff_attn_backward(q, k, v, one, kept, do, **how)):
            within(n, t, ref[n])


def test_in_place_past_32_bits(dev):
    """More than 2^31 elements turned where they lie: tokens at the start, around element 2^31 and at the end."""
    N, heads, d = 270000, 128, 64
    announce(f"in place {N} x {heads} x {d}")
    x = gen(76, dev)(1, 100, heads, d).bfloat16().repeat(1, N // 100, 1, 1)
    assert x.numel() > 2 ** 31
    freqs, places = P.rotary_freqs(d, device=dev), (0, 2 ** 31 // (heads * d) - 50, N - 100)
    before = [x[:, at:at + 100].clone() for at in places]
    y = P.rotary(x, freqs, inplace=True)
    assert y.data_ptr() == x.data_ptr()
    for at, t in zip(places, before):
        within(f"tokens from {at} on", x[:, at:at + 100], R.rotary(t, freqs, torch.arange(at, at + 100, device=dev)[None, :, None]))


def test_gradients_past_32_bits(dev):
    """dQ, dout and the kept maps of more than 2^31 elements. Only the last rows have an upstream gradient, so that every
    gradient is that of a call on these rows alone, and zero elsewhere."""
    N, heads, d, last = 270000, 64, 64, 200
    announce(f"gradients {N} x {heads} x {d}")
    r = gen(77, dev)
    q = r(1, 100, 2 * heads, d).bfloat16().repeat(1, N // 100, 1, 1)
    k, v, lam = r(1, 40, 2 * heads, d).bfloat16(), r(1, 40, heads, 2 * d).bfloat16(), 0.5 + 0.1 * r(heads)
    do = torch.zeros(1, N, heads, 2 * d, dtype=torch.bfloat16, device=dev)
    do[:, -last:] = r(1, last, heads, 2 * d).bfloat16()
    out, kept = P.diff_attn(q, k, v, lam, keep=True)
    dq, dk, dv, dlam = P.diff_attn_backward(q, k, v, lam, kept, do)
    torch.cuda.synchronize()
    assert dq.numel() > 2 ** 31 and out.numel() > 2 ** 31
    ref = R.diff_attention(q[:, -last:], k, v, lam, dout=do[:, -last:])
    for n, t in (("out", out[:, -last:]), ("dq", dq[:, -last:]), ("dk", dk), ("dv", dv), ("dlam", dlam)):
        within(n, t, ref[n])
    assert not bool((dq[:, :-last] != 0).any())


@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("shape", [(2, 300, 300, 4, 2), (2, 3, 3000, 4, 2), (1, 700, 130, 8, 1)], ids=lambda s: "x".join(map(str, s)))
def test_fp32_keeps_its_bits(dev, shape, d):
    """The root mean square of the errors, where the bounds element by element are worst cases that leave room for products
    of far fewer bits. With f = 2^-24 and independent roundings of 0.4 f of the value each: a logit of d products is off by
    0.4 f sqrt(d) of its size 1.3, 4 f at d = 64; its exponent, below 16, by 2^-21 / sqrt(3) ln 2 = 3.2 f; D = dO V^T, of 2d
    products, by 0.4 f sqrt(2d) = 4.5 f; a sum of N terms by 0.28 f sqrt(N), 15 f for the 3000 of a row in one piece. Together
    sqrt(16 + 10 + 20 + 225) f = 17 f of a result at most, and twice that is the limit. Products of 16 bits of mantissa are
    off by 2^-17 = 128 f."""
    q, k, v, lam, do = make(dev, *shape, d, "f32", seed=78, token_lam=True)
    announce(f"fp32 bits {shape} {d}")
    ref = R.diff_attention(q, k, v, lam, dout=do)
    out, kept = P.diff_attn(q, k, v, lam, keep=True)
    for n, t in zip(("out", "dq", "dk", "dv", "dlam"), (out, *P.diff_attn_backward(q, k, v, lam, kept, do))):
        off = float((t.double() - ref[n][0]).square().mean().sqrt() / ref[n][0].square().mean().sqrt()) * 2 ** 24
        print(f"{n}: {off:.1f} f", file=sys.stderr)
        assert off <= 34.0, (n, off)


@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("shape", [(4, 1, 512, 8, 8), (2, 1, 5000, 16, 4), (3, 5, 1025, 8, 2)], ids=lambda s: "x".join(map(str, s)))
def test_bf16_tokens_are_rounded_once(dev, shape, d):
    """A token or a few over a cache, bf16: off by the rounding of the result, and by 2^-17 of the weights, whose two bf16
    terms hold 16 bits: (2^-8)^2 more of its square, and 100 times that where the two maps cancel to a tenth, 0.2%."""
    q, k, v, lam, _ = make(dev, *shape, d, "bf16", seed=79)
    announce(f"bf16 tokens {shape} {d}")
    ref = R.diff_attention(q, k, v, lam)["out"][0]
    off = float((P.diff_attn(q, k, v, lam).double() - ref).square().mean().sqrt() / (ref.bfloat16().double() - ref).square().mean().sqrt())
    print(f"{off:.3f} of the rounding", file=sys.stderr)
    assert off <= 1.02
