"""Sizes and arguments at the border of what rotary positions and differential attention take, on the host: what is past it
is refused before anything reaches a device."""
import ctypes

import pytest
import torch

import paper_2201_02767_amd as P
from paper_2201_02767_amd import dense
from tests.test_dense_abi import INVALID, UNSUPPORTED, backward, diff_args, forward, rotary

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
