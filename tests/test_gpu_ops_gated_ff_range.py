"""argus_gated_ff_bwd where float16's range is short of the operands: gradients
of a mean loss, far below 2^-14, and products above 65,504.

Tolerances. dg and du round by UNIT of themselves as long as they lie within
2^28 of the largest of them; below, by half of float16's last step, which is
2^-39 of the largest. Sums, activations and outputs as in the other tests of
these operators; an output below 2^-14 rounds by 2^-25 at most. In norm two
roundings that are independent and spread evenly are off by sqrt(2 / 3) UNIT at
most: UNIT is allowed, and what outputs below 2^-14 round by."""
import math

import pytest
import torch

import paper_2606_20374_amd as pa

from .test_gpu_ops_gated_ff import ACTS, _act

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16 = torch.float16
UNIT, STEP = 2.0**-11, 2.0**-25


def _data(T, W, F, size, seed=0):
    """Inputs whose gradients float16 holds: `size` is that of d_h, and above 1
    of u as well."""
    g = torch.Generator(device=DEV).manual_seed(T + 3 * W + 5 * F + seed)
    r = lambda n, m, std: (torch.randn(n, m, generator=g, device=DEV) * std).to(F16)  # noqa: E731
    w, x = (64.0, 256.0) if size < 1 else (2.0**-14, 2.0**-13)
    return r(T, F, size), r(T, W, x), r(F, W, w), r(F, W, w), r(T, F, 1.0), r(T, F, max(1.0, size))


def _check(got, dh, x, wg, wu, g, u, act, rows=slice(None)):
    dh, x, wg, wu, g, u = (t.double() for t in (dh, x, wg, wu, g, u))
    a, da, size = _act(g, act)
    dg, du = dh * u * da, dh * a
    least = 2.0**-39 * float(torch.maximum(dg.abs(), du.abs()).max())
    eg = UNIT * dg.abs() + 2.0**-19 * size * (1 + g.abs()) * (dh * u).abs() + least
    eu = UNIT * du.abs() + 2.0**-20 * size * du.abs() + least
    T, F = dg.shape
    s = 2.0**-23
    refs = {"dx": (dg @ wg + du @ wu, (eg + 2 * F * s * dg.abs()) @ wg.abs() + (eu + 2 * F * s * du.abs()) @ wu.abs()),
            "dwg": (dg.T @ x, (eg + T * s * dg.abs()).T @ x.abs()), "dwu": (du.T @ x, (eu + T * s * du.abs()).T @ x.abs())}
    for name, (ref, tol) in refs.items():
        out = got[name].double()
        if name == "dx":
            ref, tol, out = ref[rows], tol[rows], out[rows]
        elif rows != slice(None):
            continue
        bad = ~((out - ref).abs() <= 1.02 * tol + UNIT * ref.abs() + STEP)
        assert not bad.any(), (name, int(bad.sum()), float((out - ref).abs().max()))
        assert float((out - ref).norm()) <= UNIT * float(ref.norm()) + STEP * ref.numel()**0.5, name


# few tokens, tiles of both sizes, parts of either product
@pytest.mark.parametrize("size", [1e-6, 1e-5, 300.0])
@pytest.mark.parametrize("T,W,F", [(5, 40, 136), (130, 264, 328), (999, 1000, 2720), (2_000, 264, 1_000), (10_000, 136, 200)])
def test_gradients_of_any_size(T, W, F, size):
    act = ACTS[(T + F // 8) % 3]
    dh, x, wg, wu, g, u = _data(T, W, F, size)
    assert size < 1 or float((dh.float() * u.float()).abs().max()) > 65_504
    _check(pa.gated_ff_bwd(dh, x, wg, wu, g, u, act), dh, x, wg, wu, g, u, act)


@pytest.mark.parametrize("T", [6, 300])
def test_tokens_that_hold_infinities_do_not_set_the_range(T):
    dh, x, wg, wu, g, u = _data(T, 72, 264, 1e-6)
    dh2 = dh.clone()
    dh2[3], dh2[4, 7] = math.inf, math.nan
    got = pa.gated_ff_bwd(dh2, x, wg, wu, g, u)
    rest = torch.tensor([t for t in range(T) if t not in (3, 4)], device=DEV)
    _check(got, dh, x, wg, wu, g, u, "silu", rest)
    assert not got["dx"][[3, 4]].isfinite().all(1).any()


def test_no_gradient_at_all():
    dh, x, wg, wu, g, u = _data(200, 72, 264, 1.0)
    got = pa.gated_ff_bwd(torch.zeros_like(dh), x, wg, wu, g, u)
    assert not any(got[k].any() for k in ("dx", "dwg", "dwu"))


def test_rows_of_a_wider_tensor():
    # what lies beside the rows is not looked at
    dh, x, wg, wu, g, u = _data(140, 72, 264, 1e-6)
    wide = torch.full((140, 264 + 16), 60_000.0, dtype=F16, device=DEV)
    wide[:, :264] = dh
    _check(pa.gated_ff_bwd(wide[:, :264], x, wg, wu, g, u), dh, x, wg, wu, g, u, "silu")


def test_replays_take_the_range_of_their_inputs():
    data = [_data(300, 136, 264, size) for size in (1e-6, 300.0, 1e-5)]
    ins = [t.clone() for t in data[0]]
    out = pa.alloc_gated_ff_bwd(300, 136, 264, F16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        pa.gated_ff_bwd(*ins, out=out)
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            pa.gated_ff_bwd(*ins, out=out)
    torch.cuda.current_stream().wait_stream(s)
    for d in data + data:
        for a, b in zip(ins, d):
            a.copy_(b)
        out["_workspace"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: out[k].clone() for k in ("dx", "dwg", "dwu")}
        _check(got, *d, "silu")
        pa.gated_ff_bwd(*ins, out=out)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], out[k]) for k in got)
