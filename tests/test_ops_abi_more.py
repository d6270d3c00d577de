"""The host side of rotary, gated_ff and cross_entropy: what they refuse before
any launch, and their workspaces (no GPU needed)."""
import ctypes
import math

import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import argus as A
from paper_2606_20374_amd import ops

F32, BF16, F16 = 0, 1, 2
P = 0x10000  # an aligned address
MORE = 1 << 50


def _call(fn, p, *args):
    return getattr(ops._lib(), fn)(ctypes.byref(p), *args)


def _need(fn, p):
    return getattr(ops._lib(), fn + "_workspace")(ctypes.byref(p))


def _with(p, kw):
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _rotary(**kw):
    return _with(ops.Rotary(10, 4, 64, 32, 0, 0, BF16, 1.0, 1, P, P, 256, 64, 256, 64), kw)


def _ff(**kw):
    return _with(ops.GatedFf(10, 64, 128, BF16, 0, 64, 64, 64, 128), kw)


def _ce(**kw):
    return _with(ops.CrossEntropy(P, 10, 1, 1000, 64, BF16, 1.0, 0.0, 64, 64), kw)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw", [dict(n_tokens=-1), dict(n_tokens=2**28 + 1), dict(n_heads=0), dict(n_heads=65_536), dict(head_dim=1),
                                dict(head_dim=1025), dict(rot_dim=0), dict(rot_dim=31), dict(rot_dim=66), dict(interleaved=2),
                                dict(inverse=-1), dict(pos_64=2), dict(dtype=3), dict(scale=NAN), dict(scale=INF), dict(pos=P + 4),
                                dict(pos=P + 2, pos_64=0), dict(freq=None), dict(freq=P + 4), dict(x_tok=-1), dict(x_head=-1),
                                dict(out_tok=-1), dict(out_head=-64), dict(out_head=63), dict(out_tok=63), dict(out_tok=192),
                                dict(out_head=256, out_tok=32), dict(out_head=639, out_tok=64), dict(out_tok=0), dict(out_head=0)])
def test_rotary_refuses(kw):
    assert _call("argus_rotary", _rotary(**kw), P, 2 * P, None) == A.EINVAL


def test_rotary_refuses_pointers():
    for x, out in ((None, P), (P, None), (P + 1, P), (P, P + 1)):
        assert _call("argus_rotary", _rotary(), x, out, None) == A.EINVAL
    assert _call("argus_rotary", _rotary(x_tok=320), P, P, None) == A.EINVAL  # in place with other strides
    assert ops._lib().argus_rotary(None, P, P, None) == A.EINVAL


@pytest.mark.parametrize("kw", [dict(n_tokens=-1), dict(n_tokens=2**20 + 1), dict(width=0), dict(width=60), dict(width=65_544),
                                dict(ff=0), dict(ff=100), dict(ff=131_080), dict(dtype=F32), dict(dtype=3), dict(act=-1), dict(act=3),
                                dict(x_stride=56), dict(x_stride=68), dict(x_stride=2**21 + 8), dict(wg_stride=0), dict(wg_stride=2**40),
                                dict(wu_stride=65), dict(wu_stride=-64)])
def test_gated_ff_refuses(kw):
    p = _ff(**kw)
    assert _call("argus_gated_ff", p, P, P, P, P, P, P, P, MORE, None) == A.EINVAL
    assert _call("argus_gated_ff_bwd", p, P, P, P, P, P, P, P, P, P, P, MORE, None) == A.EINVAL
    assert _need("argus_gated_ff", p) == 0 and _need("argus_gated_ff_bwd", p) == 0


def test_gated_ff_refuses_pointers_and_workspace():
    p = _ff()
    ok = [P] * 6
    for i in range(6):  # g and u may be left out together
        assert _call("argus_gated_ff", p, *[None if j == i else a for j, a in enumerate(ok)], P, MORE, None) == A.EINVAL, i
        assert _call("argus_gated_ff", p, *[a + 8 if j == i else a for j, a in enumerate(ok)], P, MORE, None) == A.EINVAL, i
    need = _need("argus_gated_ff_bwd", p)
    assert need >= 10 * 2 * 128 * 2
    ok = [P] * 9
    for i in range(9):
        assert _call("argus_gated_ff_bwd", p, *[None if j == i else a for j, a in enumerate(ok)], P, need, None) == A.EINVAL, i
        assert _call("argus_gated_ff_bwd", p, *[a + 8 if j == i else a for j, a in enumerate(ok)], P, need, None) == A.EINVAL, i
    for ws, n in ((None, need), (P + 64, need), (P, need - 1)):
        assert _call("argus_gated_ff_bwd", p, *ok, ws, n, None) == A.EINVAL
    for bad in (120, 132, 2**21 + 8):
        assert _call("argus_gated_ff_bwd", _ff(dh_stride=bad), *ok, P, need, None) == A.EINVAL
    assert ops._lib().argus_gated_ff(None, P, P, P, P, P, P, P, MORE, None) == A.EINVAL
    assert ops._lib().argus_gated_ff_bwd(None, *ok, P, need, None) == A.EINVAL


@pytest.mark.parametrize("kw", [dict(labels=None), dict(labels=P + 4), dict(labels=P + 2, ids_64=0), dict(n_tokens=-1),
                                dict(n_tokens=2**20 + 1), dict(n_tokens=2**19, n_vocab=2**19), dict(ids_64=2), dict(n_vocab=0),
                                dict(n_vocab=2**20 + 1), dict(width=0), dict(width=68), dict(width=16_392), dict(dtype=F32),
                                dict(dtype=F16), dict(scale=NAN), dict(scale=INF), dict(z_loss=-1.0), dict(z_loss=NAN),
                                dict(x_stride=56), dict(x_stride=66), dict(w_stride=0), dict(w_stride=2**21 + 8)])
def test_cross_entropy_refuses(kw):
    p, o = _ce(**kw), ops.CrossEntropyOut(*[P] * 5)
    assert _call("argus_cross_entropy", p, P, P, ctypes.byref(o), P, MORE, None) == A.EINVAL
    assert _call("argus_cross_entropy_bwd", p, P, P, P, P, P, P, P, P, P, P, MORE, None) == A.EINVAL
    assert _need("argus_cross_entropy", p) == 0 and _need("argus_cross_entropy_bwd", p) == 0


def test_cross_entropy_refuses_pointers_and_workspace():
    p = _ce()
    need = _need("argus_cross_entropy", p)
    good = ops.CrossEntropyOut(*[P] * 5)
    for x, w, ws, n in ((None, P, P, need), (P, None, P, need), (P + 8, P, P, need), (P, P + 8, P, need), (P, P, None, need),
                        (P, P, P + 64, need), (P, P, P, need - 1)):
        assert _call("argus_cross_entropy", p, x, w, ctypes.byref(good), ws, n, None) == A.EINVAL
    for f in ops.CROSS_ENTROPY_FIELDS:
        for bad in (None, P + 2):
            if bad is None and f == "dev_status":
                continue
            o = ops.CrossEntropyOut(*[P] * 5)
            setattr(o, f, bad)
            assert _call("argus_cross_entropy", p, P, P, ctypes.byref(o), P, need, None) == A.EINVAL, f
    assert _call("argus_cross_entropy", p, P, P, None, P, need, None) == A.EINVAL
    need = _need("argus_cross_entropy_bwd", p)
    ok = [P] * 8  # x, w, lse, n_valid, dmean, dloss, dx, dw
    for i in (0, 1, 2, 3, 6, 7):
        assert _call("argus_cross_entropy_bwd", p, *[None if j == i else a for j, a in enumerate(ok)], P, P, need, None) == A.EINVAL, i
    for i in range(8):
        assert _call("argus_cross_entropy_bwd", p, *[a + 2 if j == i else a for j, a in enumerate(ok)], P, P, need, None) == A.EINVAL, i
    assert _call("argus_cross_entropy_bwd", p, P, P, P, P, None, None, P, P, None, P, need, None) == A.EINVAL
    assert _call("argus_cross_entropy_bwd", p, *ok, P + 1, P, need, None) == A.EINVAL
    for ws, n in ((None, need), (P + 64, need), (P, need - 1)):
        assert _call("argus_cross_entropy_bwd", p, *ok, P, ws, n, None) == A.EINVAL
    assert ops._lib().argus_cross_entropy(None, P, P, ctypes.byref(good), P, MORE, None) == A.EINVAL
    assert ops._lib().argus_cross_entropy_bwd(None, *ok, P, P, MORE, None) == A.EINVAL


def test_workspaces_at_the_limits():
    # no tokens, one, and the most; a null descriptor has none
    for T in (0, 1, 2**20):
        for W, F in ((8, 8), (65_536, 131_072)):
            p = _ff(n_tokens=T, width=W, ff=F, x_stride=W, wg_stride=W, wu_stride=W, dh_stride=F)
            assert T * 2 * F * 2 <= _need("argus_gated_ff_bwd", p) < 1 << 46
        for W, V in ((8, 1), (16_384, 2**17)):
            p = _ce(n_tokens=T, width=W, n_vocab=V, x_stride=W, w_stride=W)
            assert 0 < _need("argus_cross_entropy", p) < 1 << 46
            assert T * W * 6 <= _need("argus_cross_entropy_bwd", p) < 1 << 46
    for f in ("gated_ff", "gated_ff_bwd", "cross_entropy", "cross_entropy_bwd"):
        assert getattr(ops._lib(), f"argus_{f}_workspace")(None) == 0


def test_binding_refuses_other_types_shapes_and_places():
    x, w, f = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(16, 8, dtype=torch.bfloat16), torch.ones(4, dtype=torch.float64)
    labels = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: pa.gated_ff(x, w, w), lambda: pa.cross_entropy(x, w, labels), lambda: pa.rotary(x[None], f)):
        with pytest.raises(AssertionError):
            call()  # host memory
    for call in (lambda: pa.gated_ff(x, w, w, act="relu"), lambda: pa.cross_entropy(x, w, labels.float()),
                 lambda: pa.rotary(x[None], f.float()), lambda: pa.rotary(x[None], f, pos=torch.zeros(1)),
                 lambda: pa.rotary(x[None], f, pos=labels)):
        with pytest.raises(pa.ArgusError):
            call()


def test_rotary_freq():
    # the definitions, written out
    f, s = pa.rotary_freq(8, base=100.0, device="cpu")
    assert s == 1 and torch.allclose(f, torch.tensor([1, 100**-0.25, 0.1, 100**-0.75], dtype=torch.float64), rtol=1e-15)
    g, s = pa.rotary_freq(8, base=100.0, factor=4.0, device="cpu")
    assert s == 1 and torch.allclose(g, f / 4, rtol=1e-15)
    g, s = pa.rotary_freq(8, base=100.0, factor=4.0, how="base", device="cpu")
    assert s == 1 and g[0] == 1 and math.isclose(g[3], f[3] / 4, rel_tol=1e-14)
    f, _ = pa.rotary_freq(128, device="cpu")
    g, s = pa.rotary_freq(128, factor=8.0, how="parts", context=4096, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert math.isclose(s, 1 + 0.1 * math.log(8)) and torch.equal(g[turns >= 32], f[turns >= 32])
    assert torch.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 8).all()
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, base=0.0), dict(rot_dim=8, factor=0.5),
                dict(rot_dim=8, how="other"), dict(rot_dim=8, how="parts", slow=4.0, fast=4.0)):
        with pytest.raises(pa.ArgusError):
            pa.rotary_freq(device="cpu", **bad)
