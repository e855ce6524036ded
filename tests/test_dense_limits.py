"""Sizes and arguments at the border of what rotary positions and differential attention take, on the host: what is past it
is refused before anything reaches a device."""
import ctypes

import pytest

import paper_2201_02767_amd as P
from tests.test_dense_abi import UNSUPPORTED, backward, diff_args, forward

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
