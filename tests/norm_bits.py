"""How far group norm over maps may be off, from the lengths of the kernel's own sums. f = 2^-24; L: tokens that a thread takes one
after the other, of which it keeps a running mean and the sum of squared distances from it.

  - a running mean moves by a rounded part of a rounded difference: 4 f of the thread's largest value a step, which is at most L times the
    mean magnitude of its values. So the thread's mean is off by 4 L f times that at most, and the group's, the mean of its threads', by
    4 L^2 f mean|x|. Joining adds sums of the entries' means (corrected by the sum of the distances from the first result, so that its
    rounding does not stay): 3 f |mean| and JOIN f mean|x - mean|. JOIN: the longest chain of additions in the two joins (rows through LDS, then
    slabs), 24 here at most each.
  - distances are rounded once: f |x - mean|, and what the mean is off.
  - squared distances: 6 f of each and L + JOIN f for their sums, all relative; (x - mean)^2 over a thread's tokens further by twice what the
    thread's running mean is off, 4 L f of its slab's largest value, times |x - mean|, whose sum is at most twice that of the distances from the
    slab's mean. What the group's mean is off adds its square alone (its first power drops out of a sum of distances from the mean). r is off by
    half of all that relative to var + eps, and 4 f.
"""
import torch

F = 2.0 ** -24
JOIN = 48


def group_norm(x, groups, L, slab, *, eps=1e-5):
    """(value, bound) of the normalised x [B, N, C] in slabs of `slab` tokens (which divides N), in 64 bits."""
    B, N, C = x.shape
    X = x.double().reshape(B, N, groups, C // groups)
    over = lambda t: t.mean((1, 3), keepdim=True)
    mean = over(X)
    d = X - mean
    var = over(d * d)
    r = 1 / torch.sqrt(var + eps)
    dm = F * (4 * L * L * over(X.abs()) + 3 * mean.abs() + JOIN * over(d.abs()))
    slabs = X.reshape(B, N // slab, slab, groups, C // groups)
    local = (slabs - slabs.mean((2, 4), keepdim=True)).abs().mean((2, 4)) * slabs.abs().amax((2, 4))      # [B, slabs, groups]
    dvar = (L + 6 + JOIN) * F * var + dm * dm + 16 * L * F * local.mean(1)[:, None, :, None]
    dr = 0.5 * dvar / (var + eps) + 4 * F
    n = d * r
    bound = r * (F * d.abs() + dm) + n.abs() * (dr + 3 * F) + torch.finfo(x.dtype).eps / 2 * n.abs()
    return n.reshape(x.shape), bound.reshape(x.shape)
