"""argus_rotary in both directions against complex products in 64 bits.

Tolerances. The angle's fraction of a turn is rounded to 32 bits (2^-25 of half
a turn), sine and cosine are off by at most 2 units of 2^-23, the scale, two
products and a sum round by 2^-24 each: together less than 2^-20 of scale (|u| +
|v|) for a pair (u, v), then the output's own rounding."""
import math

import pytest
import torch

import paper_2606_20374_amd as pa

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 2.0**-126, torch.bfloat16: 2.0**-126, torch.float16: 2.0**-24}
DTYPES = list(UNIT)


def _pairs(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _ref(x, freq, pos, interleaved, scale, inverse):
    """The result and, per element, the bound without the output's rounding."""
    x = x.double()
    re, im = _pairs(2 * len(freq), interleaved)
    turn = torch.polar(torch.full((), scale, dtype=torch.float64), pos.double().outer(freq))
    turn = (turn.conj() if inverse else turn)[:, None]
    z = torch.complex(x[..., re], x[..., im]) * turn
    out, tol = x.clone(), torch.zeros_like(x)
    out[..., re], out[..., im] = z.real, z.imag
    tol[..., re] = tol[..., im] = 2.0**-20 * abs(scale) * (x[..., re].abs() + x[..., im].abs())
    return out, tol


def _check(got, x, freq, pos, interleaved=False, scale=1.0, inverse=False):
    ref, tol = _ref(x, freq, pos, interleaved, scale, inverse)
    tol = tol + torch.where(tol > 0, UNIT[x.dtype] * ref.abs() + TINY[x.dtype], 0.0)  # what is copied is the same
    assert ((got.cpu().double() - ref).abs() <= tol).all()


def _x(shape, dtype, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,rot", [(1, 1, 2, 2), (1, 40, 128, 128), (130, 16, 64, 64), (77, 3, 96, 32),
                                                  (33, 5, 18, 6), (19, 2, 1024, 1022), (65, 7, 40, 40), (1000, 1, 130, 130),
                                                  (257, 9, 33, 32), (2100, 6, 256, 64), (5, 300, 24, 16)])
def test_both_directions(tokens, heads, dim, rot, interleaved, dtype):
    freq, _ = pa.rotary_freq(rot, device="cpu")
    pos = torch.randint(0, 5000, (tokens,), generator=torch.Generator().manual_seed(tokens))
    x = _x((tokens, heads, dim), dtype, tokens + dim)
    for call, name, inverse, p in ((pa.rotary, "out", False, pos.to(torch.int32)), (pa.rotary_bwd, "dx", True, pos)):
        got = call(x.to(DEV), freq.to(DEV), pos=p.to(DEV), interleaved=interleaved, scale=1.25)[name]
        _check(got, x, freq, pos, interleaved, 1.25, inverse)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(40, 40), (20, 12), (28, 20), (36, 24), (22, 22)])
def test_heads_that_16_bytes_do_not_divide(dim, rot, interleaved, dtype):
    freq, _ = pa.rotary_freq(rot, device="cpu")
    x = _x((301, 5, dim + 3), dtype, dim)
    got = pa.rotary(x.to(DEV)[..., 1:1 + dim], freq.to(DEV), interleaved=interleaved)["out"]
    _check(got, x[..., 1:1 + dim], freq, torch.arange(301), interleaved)


@pytest.mark.parametrize("at", [0, 65_535, 1_000_003, 2**31 - 40, -(2**31) + 40, 2**31 + 2**20])
def test_far_positions(at):
    freq, _ = pa.rotary_freq(64, device="cpu")
    pos = at + torch.arange(33)
    x = _x((33, 2, 64), torch.float32)
    _check(pa.rotary(x.to(DEV), freq.to(DEV), pos=pos.to(DEV))["out"], x, freq, pos)


def test_no_positions_are_token_numbers():
    freq, _ = pa.rotary_freq(48, device="cpu")
    x = _x((300, 3, 48), torch.bfloat16)
    _check(pa.rotary(x.to(DEV), freq.to(DEV))["out"], x, freq, torch.arange(300))


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_in_place(dtype):
    # heads of a wider buffer, heads before tokens, an odd offset, one row for all tokens
    freq, _ = pa.rotary_freq(20, device="cpu")
    wide = _x((50, 9, 31), dtype)
    f = freq.to(DEV)
    for cut in (lambda t: t[:, 2:5, 1:27], lambda t: t.transpose(0, 1)[:, 3:4, 5:], lambda t: t[7:8].expand(12, 9, 31),
                lambda t: t[:, 4:5].expand(50, 6, 31)):
        x, on = cut(wide), cut(wide.to(DEV))
        _check(pa.rotary(on, f)["out"], x, freq, torch.arange(len(x)))
    # in place: what lies around the slice stays as it was
    on = wide.to(DEV)
    part = on[3:40, 2:8, 4:27]
    pa.rotary(part, f, interleaved=True, out={"out": part})
    _check(part, wide[3:40, 2:8, 4:27], freq, torch.arange(37), True)
    on[3:40, 2:8, 4:27] = wide[3:40, 2:8, 4:27].to(DEV)
    assert torch.equal(on.cpu(), wide)


def test_rotation_is_undone_and_matches_differences():
    freq, _ = pa.rotary_freq(64)
    x = _x((60, 4, 64), torch.float32).to(DEV)
    back = pa.rotary_bwd(pa.rotary(x, freq)["out"], freq)["dx"]
    assert float((back - x).abs().max()) < 2.0**-18 * float(x.abs().max())
    # the map is linear: <R x, y> = <x, R^T y>
    y = _x((60, 4, 64), torch.float32, 9).to(DEV)
    a = (pa.rotary(x, freq, scale=0.5)["out"].double() * y.double()).sum()
    b = (x.double() * pa.rotary_bwd(y, freq, scale=0.5)["dx"].double()).sum()
    assert abs(float(a - b)) < 2.0**-19 * float((x.abs() * y.abs()).sum())


def test_infinities_and_nan_stay_in_their_pair():
    freq, _ = pa.rotary_freq(16)
    x = _x((9, 2, 20), torch.float32).to(DEV)
    ref = pa.rotary(x, freq)["out"]
    x[4, 1, 3], x[5, 0, 18] = math.nan, math.inf
    got = pa.rotary(x, freq)["out"]
    assert got[4, 1, [3, 11]].isnan().all() and got[5, 0, 18] == math.inf
    same = torch.ones_like(got, dtype=torch.bool)
    same[4, 1, 3] = same[4, 1, 11] = same[5, 0, 18] = False
    assert torch.equal(got[same], ref[same])


def test_nothing_and_no_more_is_written():
    freq, _ = pa.rotary_freq(32)
    assert pa.rotary(torch.empty(0, 3, 32, device=DEV), freq)["out"].shape == (0, 3, 32)
    x = _x((37, 5, 40), torch.bfloat16).to(DEV)
    room = torch.full((50, 5, 40), 7.0, dtype=torch.bfloat16, device=DEV)
    got = pa.rotary(x, freq, out={"out": room[4:41]})["out"]
    assert torch.equal(got, pa.rotary(x, freq)["out"])
    assert (room[:4] == 7).all() and (room[41:] == 7).all()


def test_many_tokens():
    # more workgroups than the chip holds at once, offsets past 2^31 bytes
    freq, _ = pa.rotary_freq(128)
    x = torch.randn(140_001, 64, 128, device=DEV, dtype=torch.bfloat16)
    got = pa.rotary(x, freq)["out"]
    for t in (0, 1, 70_000, 131_072, 139_999, 140_000):
        _check(got[t:t + 1].cpu(), x[t:t + 1].cpu(), freq.cpu(), torch.tensor([t]))
