"""The workspaces that group norm asks for, on the host: 256 bytes say that a call takes none."""
import ctypes

import pytest

import paper_2201_02767_amd as P
from tests.test_decay_norm_abi import BF16, F32, norm, norm_args, norm_back


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [dict(), dict(B=1, N=1, C=1, groups=1), dict(B=1, N=1, C=64, groups=1), dict(B=3, N=2, C=8, groups=8),
                                   dict(N=20, C=4104, groups=1), dict(B=1, N=100000, C=16, groups=2)], ids=str)
def test_calls_that_take_a_workspace_ask_for_more_than_256_bytes(shape, dtype):
    lib = P.lib()
    args = dict(shape, dtype=dtype)
    for per_token in (0, 1):
        a = norm_args(**args, per_token=per_token)
        forward, back = lib.qta_group_norm_workspace_bytes(ctypes.byref(a)), lib.qta_group_norm_backward_workspace_bytes(ctypes.byref(a))
        assert back > 256 and (forward == 256 if per_token else forward > 256)
        # NULL is refused wherever more than 256 bytes are asked for
        assert norm_back(ws=None, kw=dict(args, per_token=per_token)) != 0
        assert norm_back(ws=None, nbytes=0, kw=dict(args, per_token=per_token)) != 0
        if not per_token:
            assert norm(ws=None, **args) != 0 and norm(ws=None, nbytes=0, **args) != 0
