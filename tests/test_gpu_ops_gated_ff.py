"""argus_gated_ff and argus_gated_ff_bwd against the definition in 64 bits.

Tolerances. A product of two 16-bit values is exact in 32 bits; a sum of K of
them in any order is off by at most K 2^-24 of the sum of magnitudes, twice
that where the matrix instructions drop bits instead of rounding. The
activation takes an exponential, a reciprocal and a few products, off by less
than 2^-20 of itself times (1 + |argument|). Operands and outputs round by UNIT.
In norm, two roundings that are independent and spread evenly are off by
sqrt(2 / 3) UNIT at most: UNIT is allowed."""
import math

import pytest
import torch

import paper_2606_20374_amd as pa

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.bfloat16: 2.0**-126, torch.float16: 2.0**-24}
ACTS = ["silu", "gelu", "gelu_tanh"]


def _act(g, act):
    """act(g), its derivative, and 1 + |argument of the exponential|."""
    k = math.sqrt(2 / math.pi)
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s), 1 + g.abs()
    if act == "gelu":
        c = 0.5 * torch.erfc(-g * math.sqrt(0.5))  # special.ndtr loses its tail
        return g * c, c + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), 1 + g * g
    s = torch.sigmoid(2 * k * (g + 0.044715 * g**3))
    return g * s, s + g * s * (1 - s) * 2 * k * (1 + 0.134145 * g * g), 1 + 2 * g.abs() + 0.1 * g.abs()**3


def _data(T, W, F, dtype, pad=0):
    g = torch.Generator(device=DEV).manual_seed(T * 7 + W * 3 + F)
    r = lambda n, m, std: (torch.randn(n, m + pad, generator=g, device=DEV) * std).to(dtype)[:, :m]  # noqa: E731
    return r(T, W, 1.0), r(F, W, 1.5 * W**-0.5), r(F, W, W**-0.5), r(T, F, 0.2)


def _within(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[0].tolist(), float((got.double() - ref).abs().max()))


def _sums(a, b):
    """a b^T in 64 bits and the bound of its error in 32."""
    return a @ b.T, 2 * a.shape[1] * 2.0**-24 * (a.abs() @ b.abs().T)


def _check_forward(got, x, wg, wu, act):
    dt = x.dtype
    x, wg, wu = x.double(), wg.double(), wu.double()
    (g, eg), (u, eu) = _sums(x, wg), _sums(x, wu)
    a, _, size = _act(g, act)
    # the derivative is below 1.2 in size
    tol = u.abs() * (1.2 * eg + 2.0**-20 * size * a.abs()) + (a.abs() + 1.2 * eg) * eu + 2.0**-23 * (a * u).abs()
    _within(got["h"], a * u, tol * 1.01 + UNIT[dt] * (a * u).abs() + TINY[dt], "h")
    if "g" in got:
        _within(got["g"], g, 1.01 * eg + UNIT[dt] * g.abs() + TINY[dt], "g")
        _within(got["u"], u, 1.01 * eu + UNIT[dt] * u.abs() + TINY[dt], "u")


def _check_backward(got, dh, x, wg, wu, g, u, act):
    dt = x.dtype
    dh, x, wg, wu, g, u = (t.double() for t in (dh, x, wg, wu, g, u))
    a, da, size = _act(g, act)
    dg, du = dh * u * da, dh * a
    # the derivative is a sum of terms of at most 1.2 (1 + |g|)
    eg = UNIT[dt] * dg.abs() + 2.0**-19 * size * (1 + g.abs()) * (dh * u).abs() + TINY[dt]
    eu = UNIT[dt] * du.abs() + 2.0**-20 * size * du.abs() + TINY[dt]
    T, F = dg.shape
    s = 2.0**-23
    dx = dg @ wg + du @ wu
    tol = (eg + 2 * F * s * dg.abs()) @ wg.abs() + (eu + 2 * F * s * du.abs()) @ wu.abs()
    _within(got["dx"], dx, 1.02 * tol + UNIT[dt] * dx.abs() + TINY[dt], "dx")
    for name, d, e in (("dwg", dg, eg), ("dwu", du, eu)):
        ref = d.T @ x
        _within(got[name], ref, 1.02 * (e + T * s * d.abs()).T @ x.abs() + UNIT[dt] * ref.abs() + TINY[dt], name)
        if T:
            assert float((got[name].double() - ref).norm()) <= UNIT[dt] * float(ref.norm()) + TINY[dt] * ref.numel()**0.5, name
    if T:
        assert float((got["dx"].double() - dx).norm()) <= UNIT[dt] * float(dx.norm()) + TINY[dt] * dx.numel()**0.5


# one token to several tiles of each size; widths below, at and past a tile's k
SIZES = [(1, 8, 8), (1, 4096, 1000), (2, 64, 72), (4, 1024, 512), (15, 40, 136), (16, 256, 64), (17, 96, 264), (33, 104, 128),
         (64, 512, 320), (65, 32, 8), (127, 24, 248), (128, 72, 64), (130, 1000, 200), (257, 520, 392), (999, 1000, 344)]
LARGE = [(3_130, 72, 2_056), (6_300, 136, 1_000)]  # more workgroups than CUs


@pytest.mark.parametrize("dtype", list(UNIT))
@pytest.mark.parametrize("T,W,F", SIZES + LARGE)
def test_forward(T, W, F, dtype):
    act, pad = ACTS[(T + F // 8) % 3], 8 * (T % 3)
    x, wg, wu, _ = _data(T, W, F, dtype, pad)
    got = pa.gated_ff(x, wg, wu, act, save=True)
    _check_forward(got, x, wg, wu, act)
    lean = pa.gated_ff(x, wg, wu, act)
    assert list(lean) == ["h"] and torch.equal(lean["h"], got["h"])


@pytest.mark.parametrize("dtype", list(UNIT))
@pytest.mark.parametrize("act", ACTS)
def test_activations_over_their_range(act, dtype):
    # one element to a sum: g itself goes from far below to far above 0, where
    # bfloat16 still holds the activation's tail
    W = 8
    x = torch.zeros(2, W, device=DEV, dtype=dtype)
    x[:, 0] = 1
    x[:, 1] = torch.tensor([1.0, -2.0])
    wg, wu = torch.zeros(4000, W, device=DEV, dtype=dtype), torch.zeros(4000, W, device=DEV, dtype=dtype)
    wg[:, 0], wu[:, 1] = torch.linspace(-12, 12, 4000, device=DEV).to(dtype), 1.0
    got = pa.gated_ff(x, wg, wu, act, save=True)
    _check_forward(got, x, wg, wu, act)
    dh = torch.full((2, 4000), 0.5, device=DEV, dtype=dtype)
    _check_backward(pa.gated_ff_bwd(dh, x, wg, wu, got["g"], got["u"], act), dh, x, wg, wu, got["g"], got["u"], act)


@pytest.mark.parametrize("dtype", list(UNIT))
@pytest.mark.parametrize("T,W,F", SIZES + [(100, 2048, 3_080), (3_210, 3_848, 64), (3_130, 264, 520)])
def test_backward(T, W, F, dtype):
    act, pad = ACTS[(T + F // 8) % 3], 8 * (T % 3)
    x, wg, wu, dh = _data(T, W, F, dtype, pad)
    f = pa.gated_ff(x, wg, wu, act, save=True)
    got = pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"], act)
    _check_backward(got, dh, x, wg, wu, f["g"], f["u"], act)


# forward: tiles of 192 x 128, 128 x 256, 128 x 128 and 256 x 256; backward: the
# input's gradient in parts, the weights', both; large tiles and small ones
@pytest.mark.parametrize("T,W,F", [(500, 1000, 5_112), (201, 1000, 12_000), (6_300, 136, 1_000), (1_001, 520, 8_000), (999, 1000, 2_720),
                                   (2_000, 264, 5_000), (20_011, 136, 200), (10_000, 512, 1_000)])
def test_tiles_and_parts(T, W, F):
    x, wg, wu, dh = _data(T, W, F, torch.bfloat16, 8)
    f = pa.gated_ff(x, wg, wu, "gelu", save=True)
    _check_forward(f, x, wg, wu, "gelu")
    got = pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"], "gelu")
    _check_backward(got, dh, x, wg, wu, f["g"], f["u"], "gelu")


@pytest.mark.parametrize("T", [7, 200, 3_130])
def test_every_tensor_has_its_own_stride(T):
    W, F = 72, 2_056
    x, wg, wu, dh = _data(T, W, F, torch.bfloat16)
    own = lambda t, pad: torch.nn.functional.pad(t, (0, pad), value=math.nan)[:, :t.shape[1]]  # noqa: E731
    x, wg, wu, dh = own(x, 8), own(wg, 40), own(wu, 16), own(dh, 24)
    f = pa.gated_ff(x, wg, wu, save=True)
    _check_forward(f, x, wg, wu, "silu")
    _check_backward(pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"]), dh, x, wg, wu, f["g"], f["u"], "silu")


def test_many_tokens_of_a_narrow_block():
    # the weights' gradients sum over a long axis by parts
    x, wg, wu, dh = _data(40_011, 40, 72, torch.bfloat16)
    f = pa.gated_ff(x, wg, wu, save=True)
    _check_forward(f, x, wg, wu, "silu")
    _check_backward(pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"]), dh, x, wg, wu, f["g"], f["u"], "silu")


def test_gradient_against_differences():
    # the loss sum(h dh) along a direction of each input, in steps that 16 bits resolve
    x, wg, wu, dh = _data(48, 64, 96, torch.float16)
    f = pa.gated_ff(x, wg, wu, save=True)
    got = pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"])
    loss = lambda *a: float((pa.gated_ff(*a)["h"].double() * dh.double()).sum())  # noqa: E731
    ins = [x, wg, wu]
    for i, name in enumerate(("dx", "dwg", "dwu")):
        # along the gradient itself: a step that changes the loss by about 2 t |grad|^2
        way = got[name].float()
        t = 0.02 * float(ins[i].float().norm()) / float(way.norm())
        lo, hi = ([(a.float() + s * t * way).half() if j == i else a for j, a in enumerate(ins)] for s in (-1, 1))
        moved = (hi[i].double() - lo[i].double())
        want = float((moved * got[name].double()).sum())
        # third derivatives at a step of 2 % and the roundings of 4,608 values of h: below 1 %
        assert abs(loss(*hi) - loss(*lo) - want) < 0.01 * abs(want), name


def test_rows_do_not_meet():
    # a token with NaN reaches its own rows alone, forward and in dx
    x, wg, wu, dh = _data(150, 80, 136, torch.bfloat16)
    f = pa.gated_ff(x, wg, wu, save=True)
    b = pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"])
    x2, dh2 = x.clone(), dh.clone()
    x2[77], dh2[78] = math.nan, math.inf
    f2 = pa.gated_ff(x2, wg, wu, save=True)
    rest = torch.arange(150, device=DEV) != 77
    for k in ("h", "g", "u"):
        assert torch.equal(f2[k][rest], f[k][rest]) and f2[k][77].isnan().all()
    b2 = pa.gated_ff_bwd(dh2, x, wg, wu, f["g"], f["u"])
    rest = torch.arange(150, device=DEV) != 78
    assert torch.equal(b2["dx"][rest], b["dx"][rest])


@pytest.mark.parametrize("T", [1, 13, 140, 3_150])
def test_no_more_is_written(T):
    W, F = 72, 2_056
    x, wg, wu, dh = _data(T, W, F, torch.bfloat16)
    room = lambda n, m: torch.full((n + 6, m), 7.0, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    rooms = {k: room(T, F) for k in "hgu"}
    f = pa.gated_ff(x, wg, wu, save=True, out={k: r[2:2 + T] for k, r in rooms.items()})
    back = {"dx": room(T, W), "dwg": room(F, W), "dwu": room(F, W)}
    pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"], out={k: r[2:-4] for k, r in back.items()})
    for k, r in {**rooms, **back}.items():
        assert (r[:2] == 7).all() and (r[-4:] == 7).all() and not (r[2:-4] == 7).all(), k
    _check_forward(f, x, wg, wu, "silu")


def test_no_tokens():
    x, wg, wu, dh = _data(0, 64, 72, torch.bfloat16)
    f = pa.gated_ff(x, wg, wu, save=True)
    assert f["h"].shape == (0, 72)
    b = pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"])
    assert b["dx"].shape == (0, 64) and not b["dwg"].any() and not b["dwu"].any()


def test_same_bits_on_any_stream_and_with_a_used_workspace():
    x, wg, wu, dh = _data(1_500, 264, 520, torch.bfloat16)
    f = pa.gated_ff(x, wg, wu, save=True)
    b = pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"])
    want = {k: b[k].clone() for k in ("dx", "dwg", "dwu")}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b["_workspace"].fill_(255)
    with torch.cuda.stream(s):
        f2 = pa.gated_ff(x, wg, wu, save=True)
        pa.gated_ff_bwd(dh, x, wg, wu, f2["g"], f2["u"], out=b)
    s.synchronize()
    assert all(torch.equal(f[k], f2[k]) for k in "hgu") and all(torch.equal(b[k], want[k]) for k in want)
