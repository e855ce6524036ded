"""Sizes and arguments at the border of what rotary positions and differential attention take, on the host: what is past it
is refused before anything reaches a device."""
import ctypes
import math
import os
import random
import subprocess
import sys

import pytest
import torch
from torch.autograd import forward_ad

import paper_2201_02767_amd as P
from paper_2201_02767_amd import dense
from paper_2201_02767_amd.dense import RotaryTensor
from tests.test_dense_abi import BF16, FAKE, INVALID, UNSUPPORTED, WORKSPACE, backward, diff_args, forward, rotary

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BLOCKS = 1 << 24        # of 256 threads: 2^32 threads, the first count that HIP does not take


def fwd_bytes(**kw):
    return P.lib().qta_diff_attn_workspace_bytes(ctypes.byref(diff_args(**kw)))


def bwd_bytes(**kw):
    return P.lib().qta_diff_attn_backward_workspace_bytes(ctypes.byref(diff_args(**kw)))


@pytest.mark.parametrize("fits,past", [
    (dict(B=BLOCKS - 1, heads=1, kv_heads=1, Nq=1, Nk=1), dict(B=BLOCKS, heads=1, kv_heads=1, Nq=1, Nk=1)),
    (dict(B=(1 << 20) - 1, heads=16, kv_heads=16, Nq=1, Nk=1), dict(B=1 << 20, heads=16, kv_heads=16, Nq=1, Nk=1)),
    # 260 rows of a key head, five tiles of 64
    (dict(B=(BLOCKS - 1) // 20, heads=16, kv_heads=4, Nq=65, Nk=1), dict(B=BLOCKS // 20 + 1, heads=16, kv_heads=4, Nq=65, Nk=1)),
    (dict(B=15, heads=1, kv_heads=1, Nq=1 << 26, Nk=1), dict(B=16, heads=1, kv_heads=1, Nq=1 << 26, Nk=1)),
], ids=["batch", "windows", "rows", "long"])
def test_forward_launches_stay_below_2_32_threads(fits, past):
    assert fwd_bytes(**fits) >= 256
    assert fwd_bytes(**past) == 0
    assert forward(**past) == UNSUPPORTED


@pytest.mark.parametrize("fits,past", [
    # workgroups of the key pass, and one more for every head's weight
    (dict(B=BLOCKS - 2, heads=1, kv_heads=1, Nq=1, Nk=1), dict(B=BLOCKS - 1, heads=1, kv_heads=1, Nq=1, Nk=1)),
    (dict(B=(1 << 17) - 1, heads=1, kv_heads=1, Nq=1, Nk=1 << 14), dict(B=1 << 17, heads=1, kv_heads=1, Nq=1, Nk=1 << 14)),
    (dict(B=31, heads=1, kv_heads=1, Nq=1 << 26, Nk=1), dict(B=32, heads=1, kv_heads=1, Nq=1 << 26, Nk=1)),
], ids=["batch", "keys", "rows"])
def test_backward_launches_stay_below_2_32_threads(fits, past):
    assert bwd_bytes(**fits) > 256
    assert bwd_bytes(**past) == 0
    assert backward(nbytes=1 << 60, kw=past) == UNSUPPORTED


@pytest.mark.parametrize("start", [2 ** 31, 2 ** 31 + 1, 2 ** 32 + 5, -2 ** 31, -2 ** 32])
def test_rotary_start_past_32_bits(start):
    """Not taken modulo 2^32."""
    with pytest.raises(ValueError, match="start"):
        P.rotary(torch.zeros(1, 4, 4, 32), P.rotary_freqs(32), start=start)


def test_rotary_start_on_a_map():
    assert rotary(axes=2, width=4, start=1) == INVALID


class Shaped:
    """A tensor's shape and strides without its memory."""
    dtype, device, is_cuda = torch.float32, torch.device("cuda:0"), True

    def __init__(self, shape, stride):
        self.shape, self._stride = torch.Size(shape), stride

    def stride(self):
        return self._stride

    def numel(self):
        return self.shape.numel()


@pytest.mark.parametrize("shape", [(1, 2 ** 32 + 12, 4, 32), (2 ** 31, 1, 4, 32), (1, 4, 2 ** 32 + 2, 32), (1, 2 ** 16, 2 ** 16, 4, 32)])
def test_sizes_past_32_bits(shape, monkeypatch):
    """Not taken modulo 2^32: of a broadcast tensor they need no memory."""
    monkeypatch.setattr(torch, "Tensor", Shaped)
    with pytest.raises(ValueError, match="2\\^31"):
        dense._tokens(Shaped(shape, (0,) * (len(shape) - 1) + (1,)), "x")
    assert dense._tokens(Shaped((3, 2 ** 30, 4, 32), (0, 0, 0, 1)), "x")[:4] == (3, 2 ** 30, 4, 32)


# ---- in place: a head is read and written by threads of its own ----

def brute_apart(xs):
    """Every element's place, counted."""
    seen = set()
    for t in xs:
        for e in torch.ones(t.shape).nonzero().tolist():
            at = t.data_ptr() + t.element_size() * sum(i * s for i, s in zip(e, t.stride()))
            if at in seen:
                return False
            seen.add(at)
    return True


def apart(xs, monkeypatch):
    with monkeypatch.context() as m:
        m.setattr(torch.Tensor, "is_cuda", True)
        shapes = [dense._tokens(t, "x") for t in xs]
    return dense._apart(xs, shapes)


def test_overlaps_of_what_is_turned_in_place(monkeypatch):
    fused = torch.zeros(2, 11, 7, 8)
    heads_first = torch.zeros(2, 9, 5, 8).transpose(1, 2)
    pairs = torch.zeros(2, 5, 3, 2, 8)
    sound = [(fused,), (fused[:, :, :4], fused[:, :, 4:]), (fused[:, :, 5:], fused[:, :, :5]), (fused[:1], fused[1:]),
             (fused[:, :6], fused[:, 5:][:, 1:]), (heads_first[:, :, :6], heads_first[:, :, 6:]),
             (pairs[..., 0, :], pairs[..., 1, :]), (pairs[:, :, :2, 0], pairs[..., 1, :]), (fused, fused.clone()),
             (torch.zeros(40).as_strided((1, 2, 3, 2), (0, 6, 4, 1)),), (fused[:0], fused[:0]), (fused[:, :, ::2], fused[:, :, 1::2])]
    together = [(fused, fused), (fused[:, :, :4], fused[:, :, 3:]), (fused[:, :, 4:], fused[:, :, :5]), (fused[:, :10], fused[:, 1:]),
                (fused[:, :1].expand(-1, 11, -1, -1),), (pairs[..., 0, :], pairs[:, :, 1:, 0]),
                (torch.zeros(99).as_strided((1, 6, 2, 8), (0, 8, 8, 1)),)]
    for xs in sound:
        assert brute_apart(xs) and apart(xs, monkeypatch), [(t.shape, t.stride(), t.storage_offset()) for t in xs]
    for xs in together:
        assert not brute_apart(xs) and not apart(xs, monkeypatch), [(t.shape, t.stride(), t.storage_offset()) for t in xs]


def test_overlaps_of_any_strides(monkeypatch):
    """Against every element's place, for tensors of one store at random places."""
    rng, store, found = random.Random(3), torch.zeros(4000), [0, 0]
    for _ in range(3000):
        B, N, d = rng.randint(1, 3), rng.randint(1, 4), rng.choice([2, 4])
        alike = (rng.randint(0, 60), rng.choice([0, 1, 4, 8, 12, 16, 24, 48]))
        xs = []
        for _ in range(rng.choice([1, 2, 2])):
            lead = alike if rng.random() < 0.7 else (rng.randint(0, 60), rng.randint(0, 24))
            xs.append(store.as_strided((B, N, rng.randint(1, 3), d), (*lead, rng.choice([2, 4, 4, 8, 12, 50]), 1), rng.randint(0, 99)))
        want = brute_apart(xs)
        found[want] += 1
        assert apart(xs, monkeypatch) == want, [(t.shape, t.stride(), t.storage_offset()) for t in xs]
    assert min(found) > 300


def test_two_tensors_that_write_one_place():
    e = dict(heads=4, x_batch=1536, x_token=128, x_head=32, y_batch=1536, y_token=128, y_head=32)
    at = lambda i: FAKE + i * 65536
    for x0, y0, x1, y1 in ((0, 0, 0, 0), (0, 1, 2, 1), (0, 0, 0, 1), (0, 1, 1, 2), (0, 1, 2, 0)):
        table = (RotaryTensor * 2)(RotaryTensor(x=at(x0), y=at(y0), **e), RotaryTensor(x=at(x1), y=at(y1), **e))
        assert P.lib().qta_rotary(ctypes.addressof(table), 2, 2, 12, 32, 32, 1, 0, 0, 0, 0, FAKE, None, 0, 0, 1.0, None) == INVALID


# ---- derivatives that there are none of ----

@pytest.mark.parametrize("leaf", [False, True])
def test_frequencies_that_require_gradients(leaf):
    x, f = torch.zeros(1, 4, 4, 32, requires_grad=leaf), P.rotary_freqs(32).requires_grad_()
    with pytest.raises(ValueError, match="freqs"):
        P.rotary(x, f)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):       # taken, but for the place of x
        P.rotary(x, f)


@pytest.mark.parametrize("leaf", [False, True])
def test_forward_mode_derivatives(leaf):
    """Refused wherever the dual tensor comes in, with gradients on or off."""
    def refused(call, *tensors, **more):
        for i in range(len(tensors)):
            args = [forward_ad.make_dual(t, torch.ones_like(t)) if j == i else t for j, t in enumerate(tensors)]
            for mode in (torch.enable_grad, torch.no_grad):
                with mode(), pytest.raises(NotImplementedError, match="forward-mode"):
                    call(*args, **more)

    x = torch.zeros(1, 4, 4, 32, requires_grad=leaf)
    with forward_ad.dual_level():
        refused(P.rotary, x, P.rotary_freqs(32))
        refused(lambda a, b: P.rotary(a, P.rotary_freqs(32), k=b), x, x)
        refused(P.rotary, x.detach(), P.rotary_freqs(32), inverse=True)
        refused(P.rotary, x.detach(), P.rotary_freqs(32), inplace=True)
        refused(P.diff_attention, x, x, torch.zeros(1, 4, 2, 64), torch.zeros(2))
        with pytest.raises(ValueError, match="GPU"):                        # no dual tensor: taken, but for their place
            P.rotary(x.detach(), P.rotary_freqs(32))


def test_import_without_a_gpu_build_of_torch():
    """Such a torch does not have the names of its GPU side."""
    code = ("import torch\n"
            "for n in [n for n in vars(torch._C) if n.startswith('_cuda_getCurrent')]: delattr(torch._C, n)\n"
            "import paper_2201_02767_amd as P\n"
            "assert P.level_dims(8, 8, 2) and P.rotary_freqs(8).numel() == 4")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0, r.stderr


def test_alignment_of_the_small_arguments():
    """Every pointer by its type."""
    for n in ("lam", "lens", "q_pos"):
        assert forward(causal=1, **{n: FAKE + 2}) == INVALID, n
    half = dict(dtype=BF16, lam_dtype=BF16)
    assert forward(lam=FAKE + 1, **half) == INVALID
    assert backward(nbytes=16, kw=dict(half, lam=FAKE + 2), dlam=FAKE + 2) == WORKSPACE       # as far as that is checked
    for kw, n, off in (({}, "dlam", 2), (half, "dlam", 1), ({}, "lse", 2)):
        assert backward(nbytes=16, kw=kw, **{n: FAKE + off}) == INVALID, n


def test_scales_of_the_library():
    for scale in (math.nan, math.inf, 2.0 ** 97, 2.0 ** -97, 1e-45):
        assert forward(scale=scale) == INVALID, scale
        assert backward(nbytes=16, kw=dict(scale=scale)) == INVALID, scale
    for scale in (0.0, -1.0, -math.inf, 2.0 ** 96, 2.0 ** -96):
        assert backward(nbytes=16, kw=dict(scale=scale)) == WORKSPACE, scale      # as far as that is checked


def test_sources_that_may_see_a_nan():
    """A weight of the backward overflows where its row does not see the key: compiled for NaNs."""
    from paper_2201_02767_amd import build
    assert "diff_attn_bwd.hip" not in build.NO_NAN_SOURCES


def test_overlaps_under_a_default_device(monkeypatch):
    """Places are counted on the host, whatever device new tensors go to."""
    store = torch.zeros(60)
    for stride, want in (((0, 3, 2, 1), False), ((0, 6, 4, 1), True)):
        x = store.as_strided((1, 2, 3, 2), stride)
        with torch.device("meta"):
            assert apart((x,), monkeypatch) == want
