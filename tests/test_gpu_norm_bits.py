"""Group norm over maps on the GPU where statistics lose bits, against tests/norm_bits.py's bounds."""
import pytest
import torch

import paper_2201_02767_amd as P
from tests import norm_bits as R
from tests.test_gpu_dense import announce, dev, gen, within                # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [0.0, 30.0, 1000.0, -1e5])
@pytest.mark.parametrize("C,groups", [(16, 2), (16, 16), (64, 1)])
def test_a_slab_unlike_the_others(dev, C, groups, apart):
    """256 slabs of 1024 tokens (C = 64: 4096), of which the first, or another one, lies apart."""
    N = 256 * 16 * 1024 // C * (4 if C == 64 else 1)
    r = gen(41, dev)
    announce(f"group_norm, {N} tokens of {C} channels, {groups} groups, a slab {apart} apart")
    for at in (0, 77):
        x = r(1, N, C)
        x[:, at * N // 256:(at + 1) * N // 256] += apart
        within("y", P.group_norm(x, groups), R.group_norm(x, groups, N * C // 256 // 4096, N // 256))
