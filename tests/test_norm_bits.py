"""What tests/norm_bits.py's bounds tell apart, with sums in 32 bits on the host."""
import pytest
import torch

from tests import norm_bits as R


def share(x, groups, mean, var):
    """How much of the bound the results of these statistics [groups] (fp32) use, the rest in 64 bits; 64 slabs of 4 tokens a thread."""
    value, bound = R.group_norm(x, groups, 4, x.shape[1] // 64)
    y = ((x.double().unflatten(-1, (groups, -1)) - mean.double()[:, None]) / (var.double() + 1e-5).sqrt()[:, None]).flatten(-2)
    return float(((y - value).abs() / bound).max())


def inputs(shift, apart):
    x = torch.randn(1, 65536, 8, generator=torch.Generator().manual_seed(3)) + shift
    x[:, :1024] += apart
    return x


def joined(x, groups):
    """Statistics in 32 bits as the kernel makes them: slabs' means and squared distances, joined by distances from the mean."""
    X = x[0].unflatten(-1, (groups, -1)).transpose(0, 1).reshape(groups, 64, -1)              # [groups, slabs, values]
    m = X.mean(-1, keepdim=True)
    sq = (X - m).square().sum(-1)
    m, n = m[..., 0], X.shape[-1]
    first = m.mean(-1, keepdim=True)
    c = (m - first).mean(-1)
    return first[:, 0] + c, ((sq + n * (m - first) ** 2).sum(-1) / (64 * n) - c * c), (m, sq, n)


@pytest.mark.parametrize("shift,apart", [(0.0, 0.0), (300.0, 0.0), (0.0, 30.0), (0.0, 1000.0), (0.0, -1e5)])
def test_joined_statistics_are_within(shift, apart):
    x = inputs(shift, apart)
    mean, var, _ = joined(x, 2)
    assert share(x, 2, mean, var) <= 1.0


def test_a_sum_of_squares_is_not():
    x = inputs(300.0, 0.0)
    X = x[0].unflatten(-1, (2, -1))
    mean = X.mean((0, 2))
    assert share(x, 2, mean, ((X * X).mean((0, 2)) - mean * mean).clamp(min=0)) > 1.0


@pytest.mark.parametrize("apart", [30.0, 1000.0])
def test_distances_from_an_unlike_slab_are_not(apart):
    """The slabs' squares joined in one pass, with distances from the first slab's mean."""
    x = inputs(0.0, apart)
    mean, _, (m, sq, n) = joined(x, 2)
    d = m - m[:, :1]
    at = d.mean(-1)
    assert share(x, 2, mean, (sq + n * d * d).sum(-1) / (64 * n) - at * at) > 1.0
