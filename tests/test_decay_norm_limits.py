"""The sizes that include/qta.h names for decay attention and group norm are taken (host only: workspace queries, which are 0 for what
is refused)."""
import ctypes

import pytest

import paper_2201_02767_amd as P
from tests.test_decay_norm_abi import BF16, F32, decay_args, norm_args


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk", [32, 64, 128])
@pytest.mark.parametrize("dv", [32, 64, 128])
def test_decay_takes_2_to_the_22_heads(dk, dv, dtype):
    lib = P.lib()
    for heads in (1, 16, 1 << 16):
        for N in (1, 16, 17, 600, 1 << 29):
            a = decay_args(B=(1 << 22) // heads, heads=heads, N=N, dk=dk, dv=dv, dtype=dtype)
            assert lib.qta_decay_attn_workspace_bytes(ctypes.byref(a)) > 0
            assert lib.qta_decay_attn_backward_workspace_bytes(ctypes.byref(a)) > 0
    a = decay_args(B=1 << 22, heads=4, N=17, dk=dk, dv=dv, dtype=dtype)
    assert lib.qta_decay_attn_backward_workspace_bytes(ctypes.byref(a)) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_takes_2_to_the_21_maps(dtype):
    lib = P.lib()
    for C, groups in ((1, 1), (512, 1), (512, 512), (513, 1), (513, 27), (1, 1), (1023, 33), (1026, 2), (2050, 2), (4100, 4), (8196, 1),
                      (8208, 8), (1 << 20, 1), (1 << 20, 1 << 20), (513 * 2043, 2043)):
        for B in {1, 7, min(1 << 21, (1 << 30) // C)}:
            for N in {1, min(2000, (1 << 30) // B), (1 << 30) // B}:
                a = norm_args(B=B, N=N, C=C, groups=groups, dtype=dtype)
                assert lib.qta_group_norm_workspace_bytes(ctypes.byref(a)) > 0, (B, N, C, groups)
                assert lib.qta_group_norm_backward_workspace_bytes(ctypes.byref(a)) > 0, (B, N, C, groups)
    for B, N, C in ((1 << 30, 1, 1), (1 << 23, 128, 64)):
        for per_token in (0, 1):
            a = norm_args(B=B, N=N, C=C, groups=1, dtype=dtype, per_token=per_token)
            assert (lib.qta_group_norm_workspace_bytes(ctypes.byref(a)) > 0) == bool(per_token)
