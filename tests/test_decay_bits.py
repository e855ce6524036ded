"""What tests/decay_bits.py's limit tells apart, with terms of bf16 on the host."""
import math

import pytest
import torch

from tests import decay_bits as B


@pytest.mark.parametrize("g", B.DECAYS)
@pytest.mark.parametrize("n", [60, 300])
def test_two_terms_exceed_the_limit_and_three_do_not(n, g):
    r = torch.Generator().manual_seed(n)
    k, v = (torch.randn(n, 64, generator=r).bfloat16() for _ in range(2))
    apart = torch.arange(n - 1, -1, -1)
    want = (k.double() * torch.exp(g * apart.double())[:, None]).T @ v.double()
    w = torch.exp(g * apart.float())[:, None] * v.float()
    off = [B.rms((k.double().T @ B.split(w, terms))[None], want[None], 0)[0] for terms in (2, 3)]
    assert off[0] > B.STATE > 2 * off[1], off
