"""argus_layer_norm and argus_layer_norm_bwd against the definition in 64 bits.

Tolerances. A sum over a row takes at most 4 x 8 terms in a thread, 6 steps in
a wavefront and 16 wavefronts: with G = 64 2^-24 it is off by at most G of the
sum of magnitudes. So the mean is off by dm = G mean|x|, the deviations'
square root by (G + 2^-22) of itself plus dm, and a normalised value by
e = rstd dm (1 + |xhat|) + (G + 2^-21) |xhat|, twice that covering second
order; sums over r rows add at most r 2^-24 of their terms' magnitudes."""
import ctypes

import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 2.0**-126, torch.bfloat16: 2.0**-126, torch.float16: 2.0**-24}
G = 64 * 2.0**-24
SIZES = [(1, 1), (3, 2), (5, 33), (64, 768), (7, 1000), (33, 1025), (300, 2048), (9, 5000), (4, 8192), (3, 12_289),
         (2, 16_384), (2000, 24)]


def _data(rows, cols, dtype, wdtype, pad=0, level=0.7):
    g = torch.Generator().manual_seed(rows * 31 + cols)
    x = (torch.randn(rows, cols + pad, generator=g) * 2 + level).to(dtype)
    dy = (torch.randn(rows, cols + pad, generator=g) * 0.3).to(dtype)
    w = (1 + 0.2 * torch.randn(cols, generator=g)).to(wdtype)
    b = (0.2 * torch.randn(cols, generator=g)).to(wdtype)
    return x, dy, w, b


def _ref(x, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = 1 / torch.sqrt((x - mean[:, None]).square().mean(1) + eps)
    return mean, rstd, (x - mean[:, None]) * rstd[:, None]


def _near(got, ref, tol, what):
    bad = ~((got.cpu().double() - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), (got.cpu().double() - ref).abs().max())


def _xhat_tol(x, rstd, xhat):
    dm = G * x.double().abs().mean(1, keepdim=True)
    return 2 * (rstd[:, None] * dm * (1 + xhat.abs()) + (G + 2.0**-21) * xhat.abs())


@pytest.mark.parametrize("dtype,wdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                          (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype, wdtype):
    x, _, w, b = _data(rows, cols, dtype, wdtype, pad=3 if rows % 2 else 0)
    for bias in (b, None):
        got = pa.layer_norm(x.to(DEV)[:, :cols], w.to(DEV), None if bias is None else bias.to(DEV), eps=1e-5)
        xs = x[:, :cols]
        mean, rstd, xhat = _ref(xs, 1e-5)
        y = xhat * w.double() + (0 if bias is None else bias.double())
        e = _xhat_tol(xs, rstd, xhat)
        _near(got["mean"], mean, G * xs.double().abs().mean(1) + 2.0**-23 * mean.abs(), "mean")
        _near(got["rstd"], rstd, rstd * (2 * G + 2.0**-21 + 2 * rstd * G * xs.double().abs().mean(1)), "rstd")
        _near(got["y"], y, e * w.double().abs() + (UNIT[dtype] + 2.0**-22) * y.abs() + 2.0**-23 * xhat.abs() + TINY[dtype], "y")


@pytest.mark.parametrize("dtype,wdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                          (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(rows, cols, dtype, wdtype):
    x, dy, w, _ = _data(rows, cols, dtype, wdtype, pad=5 if rows % 2 else 0)
    x, dy = x[:, :cols], dy[:, :cols]
    mean, rstd, _ = _ref(x, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    xhat = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    ex = 2.0**-22 * (xhat.abs() + rstd.double()[:, None] * mean.double().abs()[:, None])  # one subtraction, one product
    g = dy.double() * w.double()
    m0, m1 = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    dx = rstd.double()[:, None] * (g - m0 - xhat * m1)
    ag = g.abs()
    t0 = (G + 2.0**-22) * ag.mean(1, keepdim=True)
    t1 = (G + 2.0**-22) * (ag * xhat.abs()).mean(1, keepdim=True) + (ag * ex).mean(1, keepdim=True)
    tdx = 2 * rstd.double()[:, None] * (t0 + xhat.abs() * t1 + ex * m1.abs() + 2.0**-22 * (ag + m0.abs() + (xhat * m1).abs()))
    xd, dyd = x.to(DEV), dy.to(DEV)
    for bias in (True, False):
        got = pa.layer_norm_bwd(dyd, xd, mean.to(DEV), rstd.to(DEV), w.to(DEV), bias=bias)
        _near(got["dx"], dx, tdx + UNIT[dtype] * dx.abs() + TINY[dtype], "dx")
        dw, n = (dy.double() * xhat).sum(0), (rows + 2) * 2.0**-24
        _near(got["dweight"], dw, n * (dy.double() * xhat).abs().sum(0) + (dy.double().abs() * ex).sum(0) + UNIT[wdtype] * dw.abs()
              + TINY[wdtype], "dweight")
        assert ("dbias" in got) == bias
        if bias:
            db = dy.double().sum(0)
            _near(got["dbias"], db, n * dy.double().abs().sum(0) + UNIT[wdtype] * db.abs() + TINY[wdtype], "dbias")


def test_constant_rows_and_large_levels():
    # deviations of 1 around 10,000: the squares are summed after the mean is taken off
    x = torch.cat([torch.full((2, 640), 5.0), 1e4 + torch.randn(3, 640, generator=torch.Generator().manual_seed(1))])
    w = torch.ones(640)
    got = pa.layer_norm(x.to(DEV), w.to(DEV), eps=1e-5)
    mean, rstd, xhat = _ref(x, 1e-5)
    assert torch.all(got["y"][:2].cpu().abs() <= 5.0 * G * 320)  # |x - mean| <= G |x|, rstd = 1 / sqrt(eps)
    e = _xhat_tol(x, rstd, xhat)[2:]
    _near(got["y"][2:], xhat[2:], e + 2.0**-22 * xhat[2:].abs(), "y")


def test_a_bad_row_stays_alone():
    x = torch.randn(9, 700)
    x[4, 30] = float("inf")
    x[6, 2] = float("nan")
    w = torch.ones(700)
    got = pa.layer_norm(x.to(DEV), w.to(DEV))["y"].cpu()
    assert torch.isnan(got[4]).any() and torch.isnan(got[6]).all()
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(got[keep], pa.layer_norm(x[keep].contiguous().to(DEV), w.to(DEV))["y"].cpu())


def test_no_rows():
    w = torch.ones(40, device=DEV)
    e = torch.empty(0, 40, device=DEV)
    assert pa.layer_norm(e, w)["y"].shape == (0, 40)
    z = torch.empty(0, device=DEV)
    out = pa.layer_norm_bwd(e, e, z, z, w)
    assert torch.all(out["dweight"] == 0) and torch.all(out["dbias"] == 0)


def test_backward_of_a_broadcast_gradient():
    x, _, w, _ = _data(50, 384, torch.float32, torch.float32)
    f = pa.layer_norm(x.to(DEV), w.to(DEV))
    one = torch.full((1, 384), 0.25, device=DEV)
    a = pa.layer_norm_bwd(one.expand(50, 384), x.to(DEV), f["mean"], f["rstd"], w.to(DEV))
    b = pa.layer_norm_bwd(one.repeat(50, 1), x.to(DEV), f["mean"], f["rstd"], w.to(DEV))
    for k in ("dx", "dweight", "dbias"):
        assert torch.equal(a[k], b[k])


def test_backward_against_differences():
    # L = sum dy y along a direction in x, w and b. Central differences of step
    # h: truncation h^2 / 6 of the third derivative (bounded through h = 2^-3
    # against 2^-4: the error falls by 4, so their difference bounds it), and
    # the rounding of y, 2^-21 of its magnitude and G of x's, over h.
    x, dy, w, b = _data(40, 520, torch.float32, torch.float32)
    g = torch.Generator().manual_seed(3)
    vx, vw, vb = torch.randn(40, 520, generator=g), torch.randn(520, generator=g), torch.randn(520, generator=g)

    def loss(h):
        y = pa.layer_norm((x + h * vx).to(DEV), (w + h * vw).to(DEV), (b + h * vb).to(DEV))["y"]
        return (y.cpu().double() * dy.double()).sum()

    f = pa.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV))
    d = pa.layer_norm_bwd(dy.to(DEV), x.to(DEV), f["mean"], f["rstd"], w.to(DEV))
    want = sum((d[k].cpu().double() * v.double()).sum() for k, v in (("dx", vx), ("dweight", vw), ("dbias", vb)))
    wide, near = ((loss(h) - loss(-h)) / (2 * h) for h in (2.0**-3, 2.0**-4))
    rounding = (dy.double().abs() * (f["y"].cpu().double().abs() + 1) * (G + 2.0**-20)).sum() / 2.0**-4
    assert abs(near - want) <= abs(wide - near) + rounding, (near, want, wide)
    assert rounding < 0.05 * abs(want) + 1  # the bound says something


@pytest.mark.parametrize("dtype,wdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                          (torch.float16, torch.float16)])
@pytest.mark.parametrize("rows,cols", [(20_001, 24), (17_000, 200), (2_501, 2_048), (1_700, 5_000), (1_300, 8_192)])
def test_rows_that_follow_one_another_in_a_workgroup(rows, cols, dtype, wdtype):
    # more rows than all workgroups take at once: each takes two or more
    test_forward(rows, cols, dtype, wdtype)
    test_backward(rows, cols, dtype, wdtype)
    p = ops.LayerNorm(rows, cols, ops.DTYPES[dtype], ops.DTYPES[wdtype], 1e-5, cols, cols)
    groups = ops._lib().argus_layer_norm_bwd_workspace(ctypes.byref(p)) // (8 * cols)
    narrow = cols <= (512 if dtype == torch.float32 else 1024)  # four rows to a workgroup
    assert rows > groups * (4 if narrow else 1)
