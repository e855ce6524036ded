"""Host-side checks of the rotary and differential-attention entry points that need no GPU: every call below fails
validation (nothing reaches the device), and the helpers that run on the host."""
import ctypes
import math

import pytest
import torch

import paper_2201_02767_amd as P
from paper_2201_02767_amd.dense import DiffAttnArgs, RotaryTensor
from tests import dense_ref as R

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x100000
F32, BF16 = 0, 1


def diff_args(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, lam=FAKE, B=2, heads=4, kv_heads=2, Nq=8, Nk=16, d=32, dtype=F32, lam_dtype=F32,
             q_batch=2048, q_token=256, q_head=32, k_batch=2048, k_token=128, k_head=32, v_batch=2048, v_token=128,
             v_head=64, lam_batch=0, lam_token=0, lam_head=1, lens=None, q_pos=None, causal=0, scale=0.0)
    a.update(kw)
    return DiffAttnArgs(**a)


def forward(out=FAKE, maps=None, lse=None, ws=None, nbytes=0, **kw):
    return P.lib().qta_diff_attn(ctypes.byref(diff_args(**kw)), out, maps, lse, ws, nbytes, None)


def backward(ws=FAKE, nbytes=0, heads_lam=1, kw={}, **p):
    a = dict(maps=FAKE, lse=FAKE, dout=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, dlam=FAKE)
    a.update(p)
    return P.lib().qta_diff_attn_backward(ctypes.byref(diff_args(**kw)), *a.values(), heads_lam, ws, nbytes, None)


def test_diff_attn_validation():
    assert P.lib().qta_diff_attn(None, FAKE, None, None, None, 0, None) == INVALID
    for n in ("q", "k", "v", "lam"):
        assert forward(**{n: None}) == INVALID, n
    for n in ("q", "k", "v"):
        assert forward(**{n: FAKE + 4}) == INVALID, n
    assert forward(out=None) == INVALID
    assert forward(out=FAKE + 8) == INVALID
    assert forward(maps=FAKE) == INVALID and forward(lse=FAKE) == INVALID      # one without the other
    for n in ("B", "heads", "kv_heads", "Nq", "Nk", "d"):
        assert forward(**{n: 0}) == INVALID, n
        assert forward(**{n: -1}) == INVALID, n
    assert forward(heads=3) == INVALID                                          # not a multiple of kv_heads
    assert forward(dtype=2) == INVALID and forward(lam_dtype=5) == INVALID
    assert forward(lam_dtype=BF16) == INVALID                                   # with fp32 inputs
    assert forward(d=16) == UNSUPPORTED and forward(d=128) == UNSUPPORTED
    for n in ("q_batch", "q_token", "q_head", "k_batch", "k_token", "k_head", "v_batch", "v_token", "v_head"):
        assert forward(**{n: 34}) == INVALID, n                                 # 136 bytes
        assert forward(**{n: -32}) == INVALID, n
    for n in ("lam_batch", "lam_token", "lam_head"):
        assert forward(**{n: -1}) == INVALID, n
    assert forward(k_token=1 << 24) == UNSUPPORTED and forward(v_token=1 << 24) == UNSUPPORTED
    assert forward(q_token=1 << 24) == UNSUPPORTED and forward(q_head=1 << 28) == UNSUPPORTED
    assert forward(Nq=1 << 27) == UNSUPPORTED and forward(Nk=1 << 29) == UNSUPPORTED


def test_diff_attn_workspace():
    """Few rows over many keys need room for their parts."""
    size = P.lib().qta_diff_attn_workspace_bytes
    long = dict(Nq=1, Nk=8192, k_batch=128 * 8192, v_batch=128 * 8192)
    need = size(ctypes.byref(diff_args(**long)))
    assert need > 256 and need % 256 == 0
    assert size(ctypes.byref(diff_args())) == 256
    assert forward(ws=FAKE, nbytes=need - 1, **long) == WORKSPACE
    assert forward(**long) == WORKSPACE
    assert forward(ws=None, nbytes=need, **long) == INVALID
    assert forward(ws=FAKE + 16, nbytes=need, **long) == INVALID
    for kw in (dict(B=0), dict(d=48), dict(heads=3), dict(dtype=7)):
        assert size(ctypes.byref(diff_args(**kw))) == 0
    assert size(None) == 0


def test_diff_attn_backward_validation():
    need = P.lib().qta_diff_attn_backward_workspace_bytes(ctypes.byref(diff_args()))
    assert need > 0 and need % 256 == 0
    assert backward(nbytes=need - 1) == WORKSPACE
    for n in ("maps", "lse", "dout", "dq", "dk", "dv", "dlam"):
        assert backward(nbytes=need, **{n: None}) == INVALID, n
    for n in ("maps", "dout", "dq", "dk", "dv"):
        assert backward(nbytes=need, **{n: FAKE + 4}) == INVALID, n
    assert backward(ws=None, nbytes=need) == INVALID
    assert backward(ws=FAKE + 16, nbytes=need) == INVALID
    assert backward(nbytes=need, kw=dict(d=48)) == UNSUPPORTED
    for kw in (dict(B=0), dict(d=48), dict(heads=3), dict(dtype=7)):
        assert P.lib().qta_diff_attn_backward_workspace_bytes(ctypes.byref(diff_args(**kw))) == 0
    assert P.lib().qta_diff_attn_backward_workspace_bytes(None) == 0


def rotary(count=1, tensors=True, B=2, N=12, d=32, rot=32, axes=1, width=0, dtype=F32, freqs=FAKE, pos=None,
           pos_batch=0, start=0, **kw):
    t = dict(x=FAKE, y=FAKE + 4096, heads=4, x_batch=1536, x_token=128, x_head=32, y_batch=1536, y_token=128, y_head=32)
    t.update(kw)
    table = (RotaryTensor * 2)(RotaryTensor(**t), RotaryTensor(**t))
    return P.lib().qta_rotary(ctypes.addressof(table) if tensors else None, count, B, N, d, rot, axes, width, 0, 0, dtype,
                              freqs, pos, pos_batch, start, 1.0, None)


def test_rotary_validation():
    assert rotary(tensors=False) == INVALID
    assert rotary(count=0) == INVALID and rotary(count=3) == INVALID
    assert rotary(freqs=None) == INVALID and rotary(freqs=FAKE + 4) == INVALID
    assert rotary(x=None) == INVALID and rotary(y=None) == INVALID and rotary(x=FAKE + 2) == INVALID
    assert rotary(heads=0) == INVALID
    for n in ("B", "N", "d", "rot"):
        assert rotary(**{n: 0}) == INVALID, n
    assert rotary(rot=34) == INVALID and rotary(rot=31) == INVALID
    assert rotary(axes=3) == INVALID and rotary(axes=0) == INVALID
    assert rotary(axes=2, rot=30, width=4) == INVALID                            # not a multiple of 4
    assert rotary(axes=2) == INVALID and rotary(axes=2, width=5) == INVALID      # 12 tokens are no rows of 5
    assert rotary(dtype=3) == INVALID
    assert rotary(pos=FAKE + 2) == INVALID and rotary(pos=FAKE, pos_batch=-1) == INVALID
    assert rotary(start=2 ** 31 - 5) == INVALID
    for n in ("x_batch", "x_token", "x_head", "y_batch", "y_token", "y_head"):
        assert rotary(**{n: -1}) == INVALID, n
    assert rotary(y=FAKE, y_token=256) == INVALID                                # in place with other strides
    assert rotary(d=8192) == UNSUPPORTED
    assert rotary(B=1 << 16, N=1 << 16) == UNSUPPORTED
    assert rotary(count=2, heads=40000) == UNSUPPORTED


def test_rotary_freqs():
    f = P.rotary_freqs(64)
    assert f.dtype == torch.float64 and f.shape == (32,)
    assert torch.allclose(f, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32), rtol=1e-15)
    two = P.rotary_freqs(32, axes=2, theta=100.0)
    assert torch.equal(two[:8], two[8:]) and float(two[0]) == 1.0
    assert torch.allclose(P.rotary_freqs(64, factor=4.0), f / 4.0, rtol=1e-15)
    parts = P.rotary_freqs(64, factor=4.0, trained=2048)
    turns = f * 2048 / (2 * math.pi)
    assert torch.equal(parts[turns > 32], f[turns > 32])
    assert torch.allclose(parts[turns < 1], f[turns < 1] / 4.0, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert bool(mid.any()) and bool(((parts < f) & (parts > f / 4.0))[mid].all())
    for bad in (dict(rot=0), dict(rot=33), dict(rot=34, axes=2), dict(rot=32, theta=0.0), dict(rot=32, factor=0.5),
                dict(rot=32, low=4.0, high=4.0), dict(rot=32, axes=3)):
        with pytest.raises(ValueError):
            P.rotary_freqs(**bad)


def test_tensors_must_be_on_a_gpu():
    q = torch.zeros(1, 4, 4, 32)
    with pytest.raises(ValueError):
        P.diff_attn(q, q, torch.zeros(1, 4, 2, 64), torch.zeros(2))
    with pytest.raises(ValueError):
        P.rotary(q, P.rotary_freqs(32))


# ---- the 64-bit statement the GPU is compared with ----

def test_reference_against_autograd():
    """dense_ref's gradients against autograd of its own forward formula, with empty rows."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    q, k, v, lam = r(2, 5, 4, 8), r(2, 7, 2, 8), r(2, 7, 1, 16), r(2, 5, 2)
    do, lens = r(2, 5, 2, 16), [0, 4]
    ref = R.diff_attention(q, k, v, lam, lens=lens, causal=True, q_pos=[0, -2], dout=do)
    leaves = [t.clone().requires_grad_() for t in (q, k, v, lam)]
    x, y, w, l = leaves
    outs = []
    for b in range(2):
        see = R.visible(5, 7, q.device, lens[b], True, [0, -2][b])
        rows = []
        for h in range(2):
            p = []
            for m in (0, 1):
                s = (x[b, :, 2 * h + m] @ y[b, :, m].T / math.sqrt(8)).masked_fill(~see, -1e30)
                p.append(torch.softmax(s, -1) * see)
            rows.append(p[0] @ w[b, :, 0] - l[b, :, h, None] * (p[1] @ w[b, :, 0]))
        outs.append(torch.stack(rows, 1))
    out = torch.stack(outs)
    assert torch.allclose(ref["out"][0], out.detach(), atol=1e-12)
    for n, t in zip(("dq", "dk", "dv", "dlam"), torch.autograd.grad(out, leaves, do)):
        assert torch.allclose(ref[n][0], t, atol=1e-12), n


@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_rotary_is_a_rotation(interleaved):
    """Lengths and the products of turned vectors at equal distances are kept; the inverse undoes it."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(1, 6, 1, 16, generator=g, dtype=torch.float64)
    f = P.rotary_freqs(16)
    p = torch.arange(6)[None, :, None]
    y, _ = R.rotary(x, f, p, interleaved=interleaved)
    z, _ = R.rotary(x, f, p + 1000, interleaved=interleaved)
    assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1))
    assert torch.allclose((y[:, 1:] * y[:, :-1]).sum(-1), (z[:, 1:] * z[:, :-1]).sum(-1))
    assert torch.allclose(R.rotary(y, f, p, interleaved=interleaved, inverse=True)[0], x)
