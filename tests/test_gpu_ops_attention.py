"""argus_attention and argus_attention_bwd against the definition in 64 bits,
from the same bfloat16 inputs.

Tolerances, per element, with u = 2^-8 twice the half unit of bfloat16's
rounding (8 significant bits: 2^-9 of a value, here 2^-8 to cover the second
order) and w = 2^-14 for the 32-bit sums and exponentials (S is off by 2^-22
of sum |q k| scale, below 2^-15 for the values here):
  o   P is rounded as an operand, o once: u (sum P |v| + |o|)
  dv  u (sum P |do| + |dv|)
  dq  dS is rounded as an operand, dq once: scale (u + w) sum P (|dP| + |delta|)
      |k| + u |dq|;  dk likewise over its queries
  lse 2^-20 (1 + |lse|) + w 2^-6"""
import ctypes
import math

import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import argus as A
from paper_2606_20374_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
U, W = 2.0**-8, 2.0**-14


def _off(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return torch.tensor(off, dtype=torch.int64)


def _make(q_lens, k_lens, H, N, D, seed=0, fused=False, amp=1.0):
    g = torch.Generator().manual_seed(seed + D + H)
    Tq, Tk = sum(q_lens), sum(k_lens)
    r = lambda *s: (torch.randn(*s, generator=g) * amp).to(torch.bfloat16)  # noqa: E731
    if fused:
        qkv = r(Tq, H + 2 * N, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + N], qkv[:, H + N:]
    else:
        q, k, v = r(Tq, H, D), r(Tk, N, D), r(Tk, N, D)
    return q, k, v, r(Tq, H, D)


def _see(a, b, causal):
    i, j = torch.arange(a)[:, None], torch.arange(b)[None]
    return (j <= i + b - a) if causal else torch.ones(a, b, dtype=torch.bool)


def _forward(q, k, v, q_lens, k_lens, causal, scale):
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    o, lse, tol = torch.zeros(q.shape).double(), torch.full(q.shape[:2], -math.inf).double(), torch.zeros(q.shape).double()
    qo, ko = _off(q_lens).tolist(), _off(k_lens).tolist()
    for d in range(len(q_lens)):
        a, b, c, e = qo[d], qo[d + 1], ko[d], ko[d + 1]
        if a == b or c == e:
            continue
        see = _see(b - a, e - c, causal)
        for h in range(H):
            s = (q[a:b, h].double() @ k[c:e, h // G].double().T * scale).masked_fill(~see, -math.inf)
            ls = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(torch.isfinite(ls), ls, 0.0)[:, None])
            lse[a:b, h], o[a:b, h] = ls, p @ v[c:e, h // G].double()
            tol[a:b, h] = (U + W) * (p @ v[c:e, h // G].double().abs() + o[a:b, h].abs())
    return o, lse, tol


def _backward(do, q, k, v, o, lse, q_lens, k_lens, causal, scale):
    H, G = q.shape[1], q.shape[1] // k.shape[1]
    ref = {n: torch.zeros(t.shape).double() for n, t in (("dq", q), ("dk", k), ("dv", v))}
    tol = {n: torch.zeros(t.shape).double() for n, t in (("dq", q), ("dk", k), ("dv", v))}
    qo, ko = _off(q_lens).tolist(), _off(k_lens).tolist()
    for d in range(len(q_lens)):
        a, b, c, e = qo[d], qo[d + 1], ko[d], ko[d + 1]
        if a == b or c == e:
            continue
        see = _see(b - a, e - c, causal)
        for h in range(H):
            n = h // G
            qq, kk, vv, g = q[a:b, h].double(), k[c:e, n].double(), v[c:e, n].double(), do[a:b, h].double()
            ls = lse[a:b, h].double()
            p = torch.exp((qq @ kk.T * scale) - torch.where(torch.isfinite(ls), ls, 0.0)[:, None])
            p = torch.where(see & torch.isfinite(ls)[:, None], p, 0.0)
            dp, delta = g @ vv.T, (g * o[a:b, h].double()).sum(1, keepdim=True)
            ds, mag = p * (dp - delta), p * (dp.abs() + delta.abs())
            ref["dv"][c:e, n] += p.T @ g
            tol["dv"][c:e, n] += (U + W) * (p.T @ g.abs())
            ref["dq"][a:b, h] = scale * ds @ kk
            tol["dq"][a:b, h] = scale * (U + W) * (mag @ kk.abs())
            ref["dk"][c:e, n] += scale * ds.T @ qq
            tol["dk"][c:e, n] += scale * (U + W) * (mag.T @ qq.abs())
    return ref, {n: tol[n] + U * ref[n].abs() + 2.0**-126 for n in tol}


def _near(got, ref, tol, what):
    bad = ~((got.cpu().double() - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((got.cpu().double() - ref).abs().max()))


def _run(q_lens, k_lens, H, N, D, causal, scale=None, fused=False, amp=1.0, offsets=True, seed=0):
    q, k, v, do = _make(q_lens, k_lens, H, N, D, seed, fused, amp)
    sc = 1 / math.sqrt(D) if scale is None else scale
    qd, kd, vd, dod = (t.to(DEV) for t in (q, k, v, do))
    if fused:
        qkv = torch.cat([q, k, v], 1).to(DEV)
        qd, kd, vd = qkv[:, :H], qkv[:, H:H + N], qkv[:, H + N:]
    off = dict(q_off=_off(q_lens).to(DEV), k_off=_off(k_lens).to(DEV)) if offsets else {}
    f = pa.attention(qd, kd, vd, causal=causal, scale=scale, **off)
    o, lse, tol = _forward(q, k, v, q_lens, k_lens, causal, sc)
    assert int(f["dev_status"]) == 0
    got = f["lse"].cpu().double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(lse))
    fin = torch.isfinite(lse)
    _near(got[fin], lse[fin], 2.0**-20 * (1 + lse[fin].abs()) + W * 2.0**-6, "lse")
    _near(f["o"], o, tol + 2.0**-126, "o")
    assert torch.all(f["o"].cpu()[~fin] == 0)
    b = pa.attention_bwd(dod, qd, kd, vd, f["o"], f["lse"], causal=causal, scale=scale, **off)
    ref, tb = _backward(do, q, k, v, f["o"].cpu(), f["lse"].cpu(), q_lens, k_lens, causal, sc)
    for n in ("dq", "dk", "dv"):
        _near(b[n], ref[n], tb[n], n)
    assert int(b["dev_status"]) == 0


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 400])
def test_lengths(n, causal):
    _run([n], [n], 2, 1, 64, causal)
    _run([n], [n], 2, 2, 128, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [8, 16, 40, 56, 64, 72, 96, 120, 128])
def test_head_dims(D, causal):
    _run([150], [150], 4, 2, D, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,N", [(1, 1), (8, 1), (6, 2), (12, 4), (16, 16), (5, 5)])
def test_head_layouts(H, N, causal):
    _run([70, 140], [70, 140], H, N, 64, causal, fused=True)
    _run([33, 140], [70, 141], H, N, 128, causal)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q_lens,k_lens", [
    ([5, 0, 130, 1, 64], [5, 0, 130, 1, 64]),        # an empty document, a single token
    ([40, 10, 0, 300], [0, 90, 50, 299]),            # no keys: rows that see nothing; no queries; one row too many
    ([300, 200], [100, 17]),                         # more queries than keys: their first rows see nothing
    ([1, 1, 1], [700, 64, 1]),                       # single queries over long keys
    ([64, 64, 64, 64, 64, 64, 64, 64], [64] * 8),    # documents as long as a tile
    ([1] * 150, [1] * 150),                          # many documents of one token
])
@pytest.mark.parametrize("causal", [False, True])
def test_documents(q_lens, k_lens, causal, D):
    _run(q_lens, k_lens, 4, 2, D, causal)


def test_without_offsets_and_scales():
    _run([190], [190], 4, 2, 64, True, offsets=False)
    _run([190], [50], 2, 2, 128, False, offsets=False)
    _run([100], [100], 2, 1, 64, True, scale=0.0)
    _run([100], [100], 2, 1, 64, True, scale=0.9)


def test_sharp_probabilities():
    # scores of some hundreds: the running maximum has to be taken off
    q, k, v, do = _make([260], [260], 2, 1, 128, 5, amp=8.0)
    f = pa.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=1.0)
    o, lse, _ = _forward(q, k, v, [260], [260], True, 1.0)
    assert torch.isfinite(f["o"]).all()
    # S up to 64 * 128 * a few in 32-bit sums: 2^-22 of sum |q k| < 2^15 is 2^-7 in the exponent
    _near(f["lse"], lse, 2.0**-7 + 2.0**-20 * lse.abs(), "lse")
    p_off = 2.0**-5  # of the probabilities, both ways
    _near(f["o"], o, (U + p_off) * 2 * v.double().abs().amax() + 0 * o, "o")
    b = pa.attention_bwd(do.to(DEV), q.to(DEV), k.to(DEV), v.to(DEV), f["o"], f["lse"], scale=1.0)
    assert all(torch.isfinite(b[n]).all() for n in ("dq", "dk", "dv"))


def test_nothing_passes_between_documents():
    lens = [70, 90, 64, 33]
    q, k, v, do = (t.to(DEV) for t in _make(lens, lens, 4, 2, 128, 3))
    off = _off(lens).to(DEV)

    def both(q, k, v, do):
        f = pa.attention(q, k, v, q_off=off)
        b = pa.attention_bwd(do, q, k, v, f["o"], f["lse"], q_off=off)
        return [f["o"], f["lse"], b["dq"], b["dk"], b["dv"]]

    clean = both(q, k, v, do)
    for bad in (float("nan"), float("inf")):
        q2, k2, v2, do2 = (t.clone() for t in (q, k, v, do))
        for t in (q2, k2, v2, do2):
            t[70:160] = bad  # the second document
        for a, b in zip(clean, both(q2, k2, v2, do2)):
            keep = [i for i in range(len(a)) if not 70 <= i < 160]
            assert torch.equal(a[keep], b[keep])


def test_no_tokens():
    z = lambda n, h: torch.zeros(n, h, 64, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    f = pa.attention(z(5, 2), z(0, 1), z(0, 1), causal=False)
    assert torch.all(f["o"] == 0) and torch.all(f["lse"] == -math.inf)
    b = pa.attention_bwd(z(5, 2) + 1, z(5, 2), z(0, 1), z(0, 1), f["o"], f["lse"], causal=False)
    assert torch.all(b["dq"] == 0) and b["dk"].shape == (0, 1, 64)
    f = pa.attention(z(0, 2), z(7, 1), z(7, 1))
    out = pa.alloc_attention_bwd(0, 7, 2, 1, 64)
    out["dk"].fill_(3)
    b = pa.attention_bwd(z(0, 2), z(0, 2), z(7, 1), z(7, 1), f["o"], f["lse"], out=out)
    assert torch.all(b["dk"] == 0) and torch.all(b["dv"] == 0)


@pytest.mark.parametrize("q_off,k_off", [([0, 40, 100], [0, 50, 90]), ([0, 60, 50, 100], [0, 20, 50, 100]),
                                         ([1, 50, 100], [0, 50, 100]), ([0, 100, 100], [0, -5, 100]),
                                         ([0, 50, 2**40], [0, 50, 100])])
def test_malformed_offsets(q_off, k_off):
    q, k, v, do = (t.to(DEV) for t in _make([100], [100], 4, 2, 64))
    off = dict(q_off=torch.tensor(q_off, device=DEV), k_off=torch.tensor(k_off, device=DEV))
    f = pa.attention(q, k, v, **off)
    assert int(f["dev_status"]) == A.DEV_BAD_SEGMENT
    assert torch.all(f["o"] == 0) and torch.all(f["lse"] == -math.inf)
    b = pa.attention_bwd(do, q, k, v, f["o"], f["lse"], **off)
    assert int(b["dev_status"]) == A.DEV_BAD_SEGMENT
    assert all(torch.all(b[n] == 0) for n in ("dq", "dk", "dv"))


def test_long_keys_of_few_queries():
    _run([3, 40], [5000, 3001], 4, 2, 128, True)
    _run([3, 40], [5000, 3001], 4, 2, 64, False)


def test_offsets_past_32_bits():
    # rows of a wide fused buffer: the last token starts past 2^32 bytes
    n, D, wide = 9000, 64, 262_144
    buf = torch.empty(n, wide, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for lo in (0, n - 300):
        buf[lo:lo + 300, :3 * D] = torch.randn(300, 3 * D, generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = (buf[:, i * D:(i + 1) * D].unflatten(1, (1, D)) for i in range(3))
    off = torch.tensor([0, 300, n - 300, n], device=DEV)
    k_off = off.clone()
    # the middle document is left out: it has neither queries nor keys
    q2, k2, v2 = (torch.cat([t[:300], t[n - 300:]]) for t in (q, k, v))
    a = pa.attention(q[n - 300:], k[n - 300:], v[n - 300:])
    b = pa.attention(q2, k2, v2, q_off=torch.tensor([0, 300, 600], device=DEV))
    assert torch.equal(a["o"], b["o"][300:])
    buf[300:n - 300, :3 * D] = 0
    c = pa.attention(q, k, v, q_off=off, k_off=k_off)
    assert torch.equal(c["o"][n - 300:], a["o"]) and torch.equal(c["o"][:300], b["o"][:300])


def test_value_gradient_against_differences():
    # o is linear in v: a difference has no truncation, only bfloat16's
    # rounding of P and of the two outputs, U of sum P |v| each
    lens = [120, 45]
    q, k, v, do = _make(lens, lens, 4, 2, 64, 11)
    v2 = (v.float() + torch.randn(v.shape, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16)
    off = _off(lens).to(DEV)
    a, b = (pa.attention(q.to(DEV), k.to(DEV), x.to(DEV), q_off=off) for x in (v, v2))
    g = pa.attention_bwd(do.to(DEV), q.to(DEV), k.to(DEV), v.to(DEV), a["o"], a["lse"], q_off=off)
    lhs = ((b["o"].cpu().double() - a["o"].cpu().double()) * do.double()).sum()
    rhs = (g["dv"].cpu().double() * (v2.double() - v.double())).sum()
    ta, tb = (_forward(q, k, x, lens, lens, True, 0.125)[2] for x in (v, v2))
    _, tol = _backward(do, q, k, v, a["o"].cpu(), a["lse"].cpu(), lens, lens, True, 0.125)
    bound = ((ta + tb) * do.double().abs()).sum() + (tol["dv"] * (v2.double() - v.double()).abs()).sum()
    assert abs(lhs - rhs) <= bound
    assert bound < 0.1 * (do.double().abs() * (a["o"].cpu().double().abs() + b["o"].cpu().double().abs())).sum()


def test_the_formula_against_differences():
    # the oracle's own gradient in 64 bits: central differences of step 1e-5,
    # whose truncation and rounding stay below 1e-8 of values around 1
    g = torch.Generator().manual_seed(4)
    q, k, v, do = (torch.randn(n, h, 16, generator=g).double() for n, h in ((9, 4), (13, 2), (13, 2), (9, 4)))

    def loss(q, k, v):
        return (_forward(q, k, v, [4, 5], [7, 6], True, 0.3)[0] * do).sum()

    o, lse, _ = _forward(q, k, v, [4, 5], [7, 6], True, 0.3)
    ref, _ = _backward(do, q, k, v, o, lse, [4, 5], [7, 6], True, 0.3)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        d = torch.randn(t.shape, generator=g).double()
        args = lambda h: [x + h * d if x is t else x for x in (q, k, v)]  # noqa: E731
        num = (loss(*args(1e-5)) - loss(*args(-1e-5))) / 2e-5
        assert abs(num - (ref[name] * d).sum()) < 1e-6


def test_same_bits_each_time_and_on_another_stream():
    lens = [500, 700, 90]
    q, k, v, do = (t.to(DEV) for t in _make(lens, lens, 8, 2, 128))
    off = _off(lens).to(DEV)
    f = pa.attention(q, k, v, q_off=off)
    first = pa.attention_bwd(do, q, k, v, f["o"], f["lse"], q_off=off)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        f2 = pa.attention(q, k, v, q_off=off)
        again = pa.attention_bwd(do, q, k, v, f2["o"], f2["lse"], q_off=off)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(f["o"], f2["o"]) and all(torch.equal(first[n], again[n]) for n in ("dq", "dk", "dv"))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nq,nk", [(100, 30), (300, 100), (1300, 1100)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_queries_that_see_nothing_whatever_their_rows_hold(bad, nq, nk, D):
    # causal, more queries than keys: the first nq - nk see none. Their own
    # rows, and the keys and values hidden from them, hold no number
    q, k, v, do = (t.to(DEV) for t in _make([nq, 40], [nk, 40], 4, 2, D, 7))
    off = dict(q_off=_off([nq, 40]).to(DEV), k_off=_off([nk, 40]).to(DEV))
    blind = nq - nk

    def both(q, k, v, do):
        f = pa.attention(q, k, v, **off)
        return f, pa.attention_bwd(do, q, k, v, f["o"], f["lse"], **off)

    _, clean = both(q, k, v, do)
    q2, do2 = q.clone(), do.clone()
    q2[:blind], do2[:blind] = bad, bad
    f, b = both(q2, k, v, do2)
    assert torch.all(f["o"][:blind] == 0) and torch.all(f["lse"][:blind] == -math.inf)
    assert torch.all(b["dq"][:blind] == 0)
    for n in ("dk", "dv"):
        assert torch.equal(b[n], clean[n]), n
    k2, v2 = k.clone(), v.clone()
    k2[0], k2[nk // 2], v2[1], v2[nk - 1] = bad, bad, bad, bad
    for kk, vv in ((k2, v), (k, v2), (k2, v2)):
        f, b = both(q, kk, vv, do)
        assert torch.all(f["o"][:blind] == 0) and torch.all(f["lse"][:blind] == -math.inf)
        assert torch.all(b["dq"][:blind] == 0)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_a_key_that_is_no_number_reaches_all_it_is_normalised_with(D, causal):
    # P of a query that sees the key is no number for any of its keys, and the
    # last query of the document sees all of them
    lens = [70, 150]
    q, k, v, do = (t.to(DEV) for t in _make(lens, lens, 4, 2, D, 9))
    off = _off(lens).to(DEV)
    k2 = k.clone()
    k2[100] = float("nan")
    f, f2 = (pa.attention(q, x, v, q_off=off, causal=causal) for x in (k, k2))
    b, b2 = (pa.attention_bwd(do, q, x, v, g["o"], g["lse"], q_off=off, causal=causal) for x, g in ((k, f), (k2, f2)))
    sees = 100 if causal else 70
    assert torch.isnan(f2["lse"][sees:]).all()
    assert torch.isnan(b2["dq"][sees:]).all()
    for n in ("dk", "dv"):
        assert torch.isnan(b2[n][70:]).all(), n
        assert torch.equal(b2[n][:70], b[n][:70]), n
    assert torch.equal(b2["dq"][:70], b["dq"][:70])


def test_single_tokens_of_head_major_tensors():
    # a view of one token: the stride to the next one is not used, the heads
    # are far apart
    H, N, D, T = 32, 8, 128, 1024
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k, v = (torch.randn(h, T, D, generator=g, device=DEV).to(torch.bfloat16).transpose(0, 1) for h in (H, N, N))
    for a, b in ((slice(500, 501), slice(0, 501)), (slice(0, 300), slice(7, 8)), (slice(9, 10), slice(9, 10))):
        x = q[a], k[b], v[b]
        y = tuple(t.contiguous() for t in x)
        do = torch.randn(y[0].shape, generator=g, device=DEV).to(torch.bfloat16)
        f, want = (pa.attention(*t, causal=False) for t in (x, y))
        d, d_want = (pa.attention_bwd(do, *t, want["o"], want["lse"], causal=False) for t in (x, y))
        for n in ("o", "lse"):
            assert torch.equal(f[n], want[n]), n
        for n in ("dq", "dk", "dv"):
            assert torch.equal(d[n], d_want[n]), n


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,H,N", [([1300, 700], 8, 1), ([900, 1400], 6, 2), ([2100], 3, 1)])
def test_shared_tiles(lens, H, N, causal, D):
    # few tiles and heads: several workgroups share a tile of keys, their parts
    # begin inside a query head, and (long keys) a tile of queries
    T = sum(lens)
    p = ops.Attention(len(lens), H, N, D, int(causal), 1, 1.0, T, T, 0x1000, 0x1000, H * D, D, N * D, D, N * D, D, None)
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    unshared = 256 + 2 * up(8 * (T // 128 + len(lens))) + up(8 * T * H)
    # at least two workgroups' 32-bit sums of dk and dv
    assert ops._lib().argus_attention_bwd_workspace(ctypes.byref(p)) >= unshared + 2 * 2 * T * N * D * 4
    _run(lens, lens, H, N, D, causal)


@pytest.mark.parametrize("causal", [False, True])
def test_shared_tiles_of_uneven_sides(causal):
    # dk and dv: one document has more queries than keys, one fewer
    _run([2500, 300], [700, 1100], 4, 1, 64, causal)
    _run([600, 900], [2300, 100], 4, 2, 128, causal)
