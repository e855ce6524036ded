"""Host-side checks of the decay attention and group norm entry points that need no GPU: every call below fails validation (nothing
reaches the device), and the references against plain sums and differences."""
import ctypes
import math

import pytest
import torch

import paper_2201_02767_amd as P
from paper_2201_02767_amd.decay import DecayAttnArgs
from paper_2201_02767_amd.norm import GroupNormArgs
from tests import decay_ref, norm_ref

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x100000
F32, BF16 = 0, 1


def decay_args(**kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, log_decay=FAKE, state=None, B=2, heads=4, N=8, dk=32, dv=64, dtype=F32, q_batch=1024,
             q_token=128, q_head=32, k_batch=1024, k_token=128, k_head=32, v_batch=2048, v_token=256, v_head=64, lens=None,
             scale=0.0)
    a.update(kw)
    return DecayAttnArgs(**a)


def decay(out=FAKE, last=None, ws=None, nbytes=0, **kw):
    return P.lib().qta_decay_attn(ctypes.byref(decay_args(**kw)), out, last, ws, nbytes, None)


def decay_back(ws=FAKE, nbytes=1 << 40, kw={}, **p):
    a = dict(dout=FAKE, dstate_out=None, dq=FAKE, dk=FAKE, dv=FAKE, dstate=None)
    a.update(p)
    return P.lib().qta_decay_attn_backward(ctypes.byref(decay_args(**kw)), *a.values(), ws, nbytes, None)


BAD = [  # what, status
    *[({n: None}, INVALID) for n in ("q", "k", "v", "log_decay")], *[({n: FAKE + 4}, INVALID) for n in ("q", "k", "v", "state")],
    ({"log_decay": FAKE + 2}, INVALID), ({"lens": FAKE + 2}, INVALID),
    *[({n: x}, INVALID) for n in ("B", "heads", "N", "dk", "dv") for x in (0, -1)],
    ({"dtype": 2}, INVALID), *[({n: x}, UNSUPPORTED) for n in ("dk", "dv") for x in (16, 48, 96, 256)],
    *[({n: x}, INVALID) for n in ("q_batch", "q_token", "q_head", "k_batch", "k_token", "k_head", "v_batch", "v_token", "v_head")
      for x in (34, -32)],
    *[({n: 1 << 24}, UNSUPPORTED) for n in ("q_token", "k_token", "v_token")],
    ({"scale": 2.0 ** 65}, INVALID), ({"scale": 2.0 ** -65}, INVALID), ({"scale": math.nan}, INVALID),
    ({"N": (1 << 30) + 1}, UNSUPPORTED), ({"heads": (1 << 16) + 1}, UNSUPPORTED), ({"B": 1 << 23}, UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD, ids=lambda x: str(x))
def test_decay_validation(change, status):
    assert decay(**change) == status
    assert decay_back(kw=change) == status


def test_decay_pointers():
    assert P.lib().qta_decay_attn(None, FAKE, None, None, 0, None) == INVALID
    assert decay(out=None) == INVALID and decay(out=FAKE + 8) == INVALID and decay(last=FAKE + 4) == INVALID
    for n in ("dout", "dq", "dk", "dv"):
        assert decay_back(**{n: None}) == INVALID and decay_back(**{n: FAKE + 8}) == INVALID, n
    assert decay_back(dstate=FAKE + 8) == INVALID and decay_back(dstate_out=FAKE + 8) == INVALID
    assert decay_back(dstate=FAKE, dstate_out=FAKE) == INVALID


def test_decay_workspace():
    """Long calls need room for the states of their parts."""
    size, back = P.lib().qta_decay_attn_workspace_bytes, P.lib().qta_decay_attn_backward_workspace_bytes
    long = dict(N=4096, q_batch=1 << 19, k_batch=1 << 19, v_batch=1 << 20)
    need, need_back = size(ctypes.byref(decay_args(**long))), back(ctypes.byref(decay_args(**long)))
    assert need > 256 and need % 256 == 0 and need_back > 256 and need_back % 256 == 0
    assert size(ctypes.byref(decay_args())) == 256 and back(ctypes.byref(decay_args(N=20))) == 256
    for call, n in ((decay, need), (lambda kw={}, **p: decay_back(kw=kw, **p), need_back)):
        kw = long if call is decay else {"kw": long}
        assert call(ws=FAKE, nbytes=n - 1, **kw) == WORKSPACE
        assert call(ws=None, nbytes=n, **kw) == INVALID
        assert call(ws=FAKE + 16, nbytes=n, **kw) == INVALID
    for kw in (dict(B=0), dict(dk=48), dict(dtype=7)):
        assert size(ctypes.byref(decay_args(**kw))) == 0 and back(ctypes.byref(decay_args(**kw))) == 0
    assert size(None) == 0 and back(None) == 0


def norm_args(**kw):
    a = dict(x=FAKE, weight=FAKE, bias=FAKE, B=2, N=10, C=64, groups=8, dtype=F32, param_dtype=F32, x_batch=640, x_token=64,
             per_token=0, act=0, eps=1e-5)
    a.update(kw)
    return GroupNormArgs(**a)


def norm(y=FAKE + 65536, stats=None, ws=FAKE, nbytes=1 << 40, **kw):
    return P.lib().qta_group_norm(ctypes.byref(norm_args(**kw)), y, stats, ws, nbytes, None)


def norm_back(ws=FAKE, nbytes=1 << 40, kw={}, **p):
    a = dict(stats=FAKE, dy=FAKE + 65536, dx=FAKE + 131072, dw=FAKE, db=FAKE)
    a.update(p)
    return P.lib().qta_group_norm_backward(ctypes.byref(norm_args(**kw)), *a.values(), ws, nbytes, None)


@pytest.mark.parametrize("change,status", [
    ({"x": None}, INVALID), ({"x": FAKE + 2}, INVALID), ({"weight": FAKE + 2}, INVALID), ({"bias": FAKE + 1}, INVALID),
    *[({n: x}, INVALID) for n in ("B", "N", "C", "groups") for x in (0, -1)], ({"groups": 7}, INVALID), ({"dtype": 2}, INVALID),
    ({"param_dtype": BF16}, INVALID), ({"param_dtype": 3}, INVALID), ({"act": 4}, INVALID), ({"act": -1}, INVALID),
    ({"eps": -1e-5}, INVALID), ({"eps": math.nan}, INVALID), ({"x_batch": -1}, INVALID), ({"x_token": -1}, INVALID),
    ({"C": 1 << 21}, UNSUPPORTED), ({"B": 1 << 15, "N": 1 << 16}, UNSUPPORTED), ({"B": 1 << 25}, UNSUPPORTED),
], ids=lambda x: str(x))
def test_norm_validation(change, status):
    assert norm(**change) == status
    assert norm_back(kw=change) == status


def test_norm_pointers_and_workspace():
    assert P.lib().qta_group_norm(None, FAKE, None, None, 0, None) == INVALID
    assert norm(y=None) == INVALID and norm(y=FAKE) == INVALID and norm(y=FAKE + 2) == INVALID and norm(stats=FAKE + 4) == INVALID
    for n in ("dy", "dx"):
        assert norm_back(**{n: None}) == INVALID and norm_back(**{n: FAKE + 65538}) == INVALID, n
    assert norm_back(dx=FAKE) == INVALID and norm_back(dx=FAKE + 65536) == INVALID
    assert norm_back(dw=FAKE + 2) == INVALID and norm_back(db=FAKE + 2) == INVALID
    assert norm_back(stats=None) == INVALID and norm_back(stats=FAKE + 4) == INVALID
    size, back = P.lib().qta_group_norm_workspace_bytes, P.lib().qta_group_norm_backward_workspace_bytes
    for kw in (dict(), dict(N=10000, x_batch=640000), dict(C=5000, groups=5), dict(dtype=BF16)):
        a, b = size(ctypes.byref(norm_args(**kw))), back(ctypes.byref(norm_args(**kw)))
        assert a >= 256 and b >= 256
        assert norm(ws=None, **kw) == INVALID and norm(ws=FAKE + 8, **kw) == INVALID and norm_back(ws=None, kw=kw) == INVALID
        assert norm(nbytes=0, **kw) == WORKSPACE and norm_back(nbytes=0, kw=kw) == WORKSPACE
    for kw in (dict(B=0), dict(groups=7), dict(dtype=9), dict(C=1 << 21)):
        assert size(ctypes.byref(norm_args(**kw))) == 0 and back(ctypes.byref(norm_args(**kw))) == 0
    assert size(None) == 0 and back(None) == 0


# ---- the references ----

def test_decay_reference_is_the_recurrence():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    q, k, v, S0 = r(1, 9, 2, 3), r(1, 9, 2, 3), r(1, 9, 2, 4), r(1, 2, 3, 4)
    ld = torch.tensor([-0.3, -math.inf])
    want = decay_ref.decay_attention(q, k, v, ld, scale=0.7, lens=[7], state=S0)
    S = S0[0].clone()
    f = ld.double().exp()
    for t in range(7):
        S = S * f[:, None, None] + k[0, t, :, :, None] * v[0, t, :, None, :]
        assert torch.allclose(want["out"][0][0, t], 0.7 * (q[0, t, :, :, None] * S).sum(1))
    assert torch.allclose(want["state"][0][0], S) and not want["out"][0][0, 7:].any()


def differences(f, x, up, at, h=1e-6):
    """The derivative of sum(f(x) * up) with respect to x's entries `at`, by central differences."""
    d = []
    for i in at:
        e = torch.zeros(x.numel(), dtype=torch.float64)
        e[i] = h
        e = e.reshape(x.shape)
        d.append(sum(float(((a - b) * u).sum()) for a, b, u in zip(f(x + e), f(x - e), up)) / (2 * h))
    return torch.tensor(d, dtype=torch.float64)


def test_decay_reference_gradients():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x = {"dq": r(2, 6, 2, 3), "dk": r(2, 6, 2, 3), "dv": r(2, 6, 2, 4), "dstate": r(2, 2, 3, 4)}
    ld, up = torch.tensor([-0.4, 0.0]), (r(2, 6, 2, 4), r(2, 2, 3, 4))

    def run(**given):
        y = {**x, **given}
        w = decay_ref.decay_attention(y["dq"], y["dk"], y["dv"], ld, lens=[6, 4], state=y["dstate"])
        return w["out"][0], w["state"][0]
    want = decay_ref.decay_attention(x["dq"], x["dk"], x["dv"], ld, lens=[6, 4], state=x["dstate"], dout=up[0], dstate_out=up[1])
    for n, t in x.items():
        at = range(0, t.numel(), 5)
        assert torch.allclose(differences(lambda y: run(**{n: y}), t, up, at), want[n][0].flatten()[list(at)], atol=1e-6), n


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("per_token", [False, True])
def test_norm_reference_gradients(act, per_token):
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x = {"dx": r(2, 5, 12), "dweight": 1 + 0.2 * r(12), "dbias": r(12)}
    up = r(2, 5, 12)

    def run(**given):
        y = {**x, **given}
        return (norm_ref.group_norm(y["dx"], 3, y["dweight"], y["dbias"], act=act, per_token=per_token)["y"][0],)
    want = norm_ref.group_norm(x["dx"], 3, x["dweight"], x["dbias"], act=act, per_token=per_token, dy=up)
    plain = torch.nn.functional.group_norm(x["dx"].transpose(1, 2), 3, x["dweight"], x["dbias"]).transpose(1, 2)
    if act == "none" and not per_token:
        assert torch.allclose(want["y"][0], plain)
    for n, t in x.items():
        at = range(0, t.numel(), 3)
        assert torch.allclose(differences(lambda y: run(**{n: y}), t, (up,), at), want[n][0].flatten()[list(at)], atol=1e-6), n
