"""Gradients of decay attention and group norm on the GPU where autograd hands back other tensors than it was given: kept tensors that moved,
upstream gradients of any layout, maps; and what function transforms are told."""
import pytest
import torch

import paper_2201_02767_amd as P
from tests import decay_ref, norm_ref
from tests.test_gpu_decay import make
from tests.test_gpu_dense import DT, announce, dev, gen, i32, within       # noqa: F401

pytestmark = pytest.mark.gpu


def moved(t):
    return t.clone()


def wider(t):
    """The same values, each token's channels apart from the next one's (statistics and vectors: moved)."""
    if t.dim() < 3 or t.shape[-1] == 2:
        return t.clone()
    return torch.cat((t, t), -1)[..., :t.shape[-1]]


def apart(t):
    """A contiguous tensor that starts one element behind a 16-byte border."""
    return torch.cat((t.new_zeros(1), t.reshape(-1)))[1:].view(t.shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [5, 90, 700])
def test_decay_gradients_of_kept_tensors_that_moved(dev, N, dtype):
    (q, k, v, g, s), (dout, dlast) = make(dev, 2, N, 3, 32, 64, dtype, seed=N)
    lens = i32([N - 2, N], dev)
    announce(f"decay_attention, kept tensors moved {N} {dtype}")
    want = decay_ref.decay_attention(q, k, v, g, state=s, dout=dout, dstate_out=dlast, lens=lens)
    grads = []
    keep_state = lambda how: (lambda t: t.clone() if t.shape == s.shape else how(t))
    for how in (lambda t: t, moved, wider):
        leaves = [t.clone().requires_grad_() for t in (q, k, v, s)]
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.clone(), keep_state(how)):
            out, last = P.decay_attention(*leaves[:3], g, state=leaves[3], lens=lens, return_state=True)
        for ups in ((dout, dlast), (apart(dout), apart(dlast)), (dout.transpose(1, 2).contiguous().transpose(1, 2), dlast.mT.contiguous().mT)):
            grads.append(torch.autograd.grad((out, last), leaves, ups, retain_graph=True))
    for n, t in zip(("dq", "dk", "dv", "dstate"), grads[0]):
        within(n, t, want[n])
    for other in grads[1:]:
        assert all(torch.equal(a, b) for a, b in zip(grads[0], other))


def test_decay_refuses_a_kept_state_of_another_layout(dev):
    (q, k, v, g, s), (dout, dlast) = make(dev, 1, 40, 2, 32, 64, "f32", seed=1)
    q.requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.mT.contiguous().mT if t.shape == s.shape else t):
        out = P.decay_attention(q, k, v, g, state=s)
    with pytest.raises(ValueError, match="state"):
        out.backward(dout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 3, 5), (1, 20, 31), (2, 1, 40), (2, 40, 1)], ids=str)
def test_decay_gradients_of_maps(dev, shape, dtype):
    """Maps are read row by row: the gradients of the sequences, whose heads may lie before the tokens."""
    B, H, W = shape
    (q, k, v, g, s), (dout, dlast) = make(dev, B, H * W, 2, 64, 32, dtype, seed=7)
    announce(f"decay_attention of maps {shape} {dtype}")
    grads = []
    for as_map in (False, True):
        leaves = [(t.unflatten(1, (H, W)) if as_map else t).clone().requires_grad_() for t in (q, k, v)]
        given = [leaves[0], leaves[1].movedim(-2, 1).contiguous().movedim(1, -2), leaves[2]]
        out, last = P.decay_attention(*given, g, state=s, return_state=True)
        assert out.shape == (*leaves[0].shape[:-1], 32)
        d = torch.autograd.grad((out, last), leaves, (dout.reshape(out.shape), dlast))
        grads.append([t.reshape(B, H * W, *t.shape[-2:]) for t in d])
    want = decay_ref.decay_attention(q, k, v, g, state=s, dout=dout, dstate_out=dlast)
    for n, a, b in zip(("dq", "dk", "dv"), *grads):
        within(n, a, want[n])
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("per_token", [False, True])
def test_norm_gradients_of_kept_tensors_that_moved(dev, per_token, dtype):
    r = gen(51, dev)
    x, w, b, dy = (t.to(DT[dtype]) for t in (r(2, 6, 7, 64), 1 + 0.3 * r(64), r(64), r(2, 6, 7, 64)))
    announce(f"group_norm, kept tensors moved {per_token} {dtype}")
    want = norm_ref.group_norm(x, 4, w, b, act="silu", per_token=per_token, dy=dy)
    grads = []
    for how in (lambda t: t, moved, wider):
        leaves = [t.clone().requires_grad_() for t in (x, w, b)]
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t.clone(), how):
            y = P.group_norm(leaves[0], 4, *leaves[1:], act="silu", per_token=per_token)
        for up in (dy, apart(dy), dy.transpose(1, 2).contiguous().transpose(1, 2), wider(dy)):
            grads.append(torch.autograd.grad(y, leaves, up, retain_graph=True))
    for g in grads:
        for n, t in zip(("dx", "dweight", "dbias"), g):
            within(n, t, want[n])
        # (an address off 16 bytes takes narrower accesses, whose sums are in another order)
        assert all(a.shape == t.shape for a, t in zip(g, grads[0]))
    assert all(torch.equal(a, c) for a, c in zip(grads[0], grads[4]))


def test_function_transforms_are_refused(dev):
    (q, k, v, g, _), _ = make(dev, 2, 20, 2, 32, 32, "f32", seed=2, state=False)
    announce("decay_attn and group_norm under function transforms")
    stack = torch.stack((q, q))
    for f in (lambda t: P.decay_attn(t, k, v, g), lambda t: P.decay_attention(t, k, v, g), lambda t: P.group_norm(t.flatten(-2), 2)):
        with pytest.raises(RuntimeError):
            torch.vmap(f)(stack)
        with pytest.raises(RuntimeError):
            torch.func.grad(lambda t: f(t).sum())(q)
    with pytest.raises(RuntimeError):
        torch.vmap(lambda t: P.decay_attention(t, k, v, g))(stack.requires_grad_())
