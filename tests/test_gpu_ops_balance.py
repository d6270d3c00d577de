"""argus_balance and argus_balance_bwd against the definition in 64 bits.

Experts, counts and the number of tokens have to be equal. Tolerances: an
exponential's argument x - m is rounded in base 2, an error of 2^-23 (|x - m|
+ 1) in the result, and the sum of at most 64 terms a lane and 4 steps adds
68 2^-24: a probability is off by e = 2^-22 (|x - m| + 1) + 2^-17 at most (of
itself), lse by 2^-17 + 2^-23 |lse|, a sum over n tokens by n 2^-24 more."""
import math

import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 2.0**-126, torch.bfloat16: 2.0**-126, torch.float16: 2.0**-24}


def _reference(logits, K, mask, alpha):
    x = logits.double()
    T, E = x.shape
    on = torch.ones(T, dtype=torch.bool) if mask is None else mask != 0
    top = torch.where(torch.isnan(x), math.inf, x).amax(1)
    ok = on & ~torch.isnan(x).any(1) & torch.isfinite(top)
    n = int(ok.sum())
    m = torch.where(ok, top, 0.0)[:, None]
    ex = torch.exp(torch.where(ok[:, None], x, 0.0) - m)
    z = ex.sum(1, keepdim=True)
    p = torch.where(ok[:, None], ex / z, 0.0)
    order = torch.argsort(torch.where(ok[:, None], x, 0.0), dim=1, descending=True, stable=True)[:, :K]
    there = ok[:, None] & torch.isfinite(x.gather(1, order))
    expert = torch.where(there, order, -1)
    gate = torch.where(there, p.gather(1, order), 0.0)
    count = torch.bincount(expert[there], minlength=E)
    prob = p.sum(0) / max(n, 1)
    loss = alpha * E * (count.double() / (K * max(n, 1)) * prob).sum()
    lse = torch.where(ok, (m + torch.log(z))[:, 0], -math.inf)
    return dict(expert=expert, gate=gate, count=count, prob=prob, loss=loss, lse=lse, n=n, p=p, ok=ok, bad=bool((on & ~ok).any()))


def _logits(T, E, dtype, kind, seed=0, pad=0):
    g = torch.Generator().manual_seed(seed + T + E)
    x = torch.randn(T, E + pad, generator=g) * 2
    if kind == "ties":
        x = torch.round(x)
    elif kind == "zeros":  # both zeros, nothing else
        x = torch.where(x > 0, 0.0, -0.0)
    elif kind == "wide":
        x = x * 30
    return x.to(dtype)


def _check(got, ref, logits, n_tol):
    assert torch.equal(got["expert"].cpu().long(), ref["expert"])
    assert torch.equal(got["count"].cpu().long(), ref["count"])
    assert int(got["n_valid"]) == ref["n"]
    x = logits.double()
    far = torch.where(ref["ok"][:, None], (x.masked_fill(~torch.isfinite(x), 0) - ref["lse"][:, None].clamp(min=-1e30)).abs(), 0.0)
    e = 2.0**-22 * (far + 1) + 2.0**-17
    eg = torch.where(ref["expert"] >= 0, e.gather(1, ref["expert"].clamp(min=0)), 0.0)
    assert torch.all((got["gate"].cpu().double() - ref["gate"]).abs() <= eg * ref["gate"] + 2.0**-126)
    lse = got["lse"].cpu().double()
    assert torch.equal(torch.isfinite(lse), ref["ok"])
    ok = ref["ok"]
    assert torch.all((lse - ref["lse"])[ok].abs() <= 2.0**-17 + 2.0**-23 * ref["lse"][ok].abs())
    n = max(ref["n"], 1)
    tp = (ref["p"] * e).sum(0) / n + n_tol * 2.0**-24 * ref["prob"] + 2.0**-126
    assert torch.all((got["prob"].cpu().double() - ref["prob"]).abs() <= tp)
    E = logits.shape[1]
    K = got["expert"].shape[1]
    tl = 0.02 * E * (ref["count"].double() / (K * n) * tp).sum() + 2.0**-23 * ref["loss"]
    assert abs(float(got["loss"]) - float(ref["loss"])) <= tl


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ["normal", "ties", "zeros", "wide"])
@pytest.mark.parametrize("T,E,K,pad", [(1, 1, 1, 0), (3, 8, 2, 0), (65, 60, 6, 0), (1000, 128, 8, 0), (257, 160, 16, 3),
                                       (130, 256, 8, 0), (70, 384, 4, 0), (20, 513, 8, 1), (33, 1024, 16, 0), (17, 700, 1, 0)])
def test_forward(T, E, K, pad, dtype, kind):
    x = _logits(T, E, dtype, kind, pad=pad)
    got = pa.balance(x.to(DEV)[:, :E], K, alpha=0.02)
    _check(got, _reference(x[:, :E], K, None, 0.02), x[:, :E], T)
    assert int(got["dev_status"]) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_and_rows_that_hold_nothing(dtype):
    T, E, K = 300, 72, 5
    x = _logits(T, E, dtype, "normal")
    g = torch.Generator().manual_seed(4)
    mask = (torch.rand(T, generator=g) < 0.6).to(torch.uint8)
    mask[:20] = 1
    x[mask == 0] = float("nan")        # masked rows hold anything
    x[2] = float("-inf")               # no finite logit: left out
    x[3, 7] = float("nan")
    x[4, 8] = float("inf")
    x[5, 3:] = float("-inf")           # fewer finite logits than experts to choose
    x[6] = torch.finfo(dtype).min      # the type's lowest value is a logit like others
    x[7, :] = torch.finfo(dtype).min
    x[7, 11] = 0.5
    ref = _reference(x, K, mask, 0.01)
    assert ref["bad"] and not ref["ok"][2:5].any() and ref["ok"][5:8].all()
    for m in (mask, mask.bool()):
        got = pa.balance(x.to(DEV), K, mask=m.to(DEV))
        _check(got | {"loss": got["loss"]}, ref | {"loss": ref["loss"]}, x, T)
        assert int(got["dev_status"]) == ops.DEV_LOGITS
    assert got["expert"][5].tolist()[3:] == [-1, -1] and torch.all(got["gate"][5, 3:] == 0)
    bwd = pa.balance_bwd(x.to(DEV), got["lse"], got["expert"], got["count"], got["n_valid"], torch.ones(1, device=DEV),
                         dgate=torch.ones(T, K, device=DEV))["dlogits"].cpu()
    assert torch.all(bwd[~ref["ok"]] == 0) and torch.isfinite(bwd).all()
    assert torch.all(bwd[5, 3:] == 0)


def test_nothing_takes_part():
    x = torch.randn(40, 16, device=DEV)
    for logits, mask in ((x, torch.zeros(40, dtype=torch.uint8, device=DEV)), (x[:0], None)):
        got = pa.balance(logits, 2, mask=mask)
        assert float(got["loss"]) == 0 and int(got["n_valid"]) == 0 and int(got["dev_status"]) == 0
        assert torch.all(got["count"] == 0) and torch.all(got["prob"] == 0) and torch.all(got["expert"] == -1)
        d = pa.balance_bwd(logits, got["lse"], got["expert"], got["count"], got["n_valid"], torch.ones(1, device=DEV))
        assert torch.all(d["dlogits"] == 0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,K,pad", [(1, 1, 1, 0), (3, 8, 2, 0), (65, 60, 6, 2), (1000, 128, 8, 0), (257, 160, 16, 0),
                                       (130, 256, 8, 0), (70, 384, 4, 0), (33, 1024, 16, 0)])
def test_gradient(T, E, K, pad, dtype):
    x = _logits(T, E, dtype, "normal", pad=pad)[:, :E]
    g = torch.Generator().manual_seed(6)
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8)
    xd = x.to(DEV) if not pad else _logits(T, E, dtype, "normal", pad=pad).to(DEV)[:, :E]
    f = pa.balance(xd, K, mask=mask.to(DEV), alpha=0.5)
    dloss, dgate = torch.tensor([1.25]), torch.randn(T, K, generator=g) * 0.1
    for dg in (dgate, None):
        got = pa.balance_bwd(xd, f["lse"], f["expert"], f["count"], f["n_valid"], dloss.to(DEV),
                             dgate=None if dg is None else dg.to(DEV), alpha=0.5)["dlogits"].cpu().double()
        lse, expert, n = f["lse"].cpu().double(), f["expert"].cpu().long(), max(1, int(f["n_valid"]))
        on = torch.isfinite(lse)[:, None]
        diff = torch.where(on, x.double() - lse.clamp(min=-1e30)[:, None], 0.0)
        p = torch.where(on, torch.exp(diff), 0.0)
        gr = (1.25 * 0.5 * E / (K * n * n) * f["count"].cpu().double()).expand(T, E).clone()
        if dg is not None:
            gr.scatter_add_(1, expert.clamp(min=0), torch.where(expert >= 0, dg.double(), 0.0))
        s = (gr * p).sum(1, keepdim=True)
        ref = p * (gr - s)
        e = 2.0**-22 * (diff.abs() + 1) + 2.0**-17
        tol = p * (e * (gr - s).abs() + 2.0**-21 * gr.abs() + (e * gr.abs() * p).sum(1, keepdim=True) + 2.0**-21 * s.abs())
        assert torch.all((got - ref).abs() <= tol + UNIT[dtype] * ref.abs() + TINY[dtype])


def test_gradient_against_differences():
    # the loss with the counts held (its derivative takes them as constants)
    # plus the gates, through the forward's own prob and gate, along a
    # direction; steps 2^-5 and 2^-6, whose difference bounds the truncation
    T, E, K = 200, 48, 4
    x = _logits(T, E, torch.float32, "normal")
    g = torch.Generator().manual_seed(2)
    v, dgate = torch.randn(T, E, generator=g), torch.randn(T, K, generator=g)
    f = pa.balance(x.to(DEV), K, alpha=10.0)
    at, count = f["expert"].cpu().long(), f["count"].cpu().double()

    def loss(h):
        # all probabilities of a token as gates of E choices
        y = (x + h * v).to(DEV)
        o = pa.balance(y, K)
        p = torch.exp(y.cpu().double() - o["lse"].cpu().double()[:, None])
        return 10.0 * E * (count / (K * T) * o["prob"].cpu().double()).sum() + (p.gather(1, at) * dgate.double()).sum()

    d = pa.balance_bwd(x.to(DEV), f["lse"], f["expert"], f["count"], f["n_valid"], torch.ones(1, device=DEV),
                       dgate=dgate.to(DEV), alpha=10.0)["dlogits"].cpu().double()
    want = (d * v.double()).sum()
    wide, near = ((loss(h) - loss(-h)) / (2 * h) for h in (2.0**-5, 2.0**-6))
    rounding = (2.0**-16 * (dgate.double().abs() * f["gate"].cpu().double()).sum() + 2.0**-16 * 10.0 * E) / 2.0**-6
    assert abs(near - want) <= abs(wide - near) + rounding, (near, want, wide, rounding)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_gradient_of_a_loss_that_is_no_number_spares_masked_tokens(bad):
    x = _logits(50, 24, torch.float32, "normal").to(DEV)
    mask = torch.ones(50, dtype=torch.uint8, device=DEV)
    mask[::3] = 0
    f = pa.balance(x, 2, mask=mask)
    d = pa.balance_bwd(x, f["lse"], f["expert"], f["count"], f["n_valid"], torch.full((1,), bad, device=DEV))["dlogits"]
    assert torch.all(d[mask == 0] == 0) and not torch.isfinite(d[mask == 1]).any()


def test_same_bits_each_time():
    x = _logits(20_000, 128, torch.bfloat16, "normal").to(DEV)
    a, b = pa.balance(x, 8), pa.balance(x, 8)
    for k in ("expert", "gate", "lse", "count", "prob", "loss"):
        assert torch.equal(a[k], b[k])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_repeated_choices_adds_them_in_order(dtype):
    # 2^27 + 1 - 2^27 + 1 from the left is 1 in 32 bits, and 0 or 2 in other
    # orders; tokens of distinct choices beside them, and choices of no expert
    T, E, K = 64, 40, 4
    x = _logits(T, E, dtype, "normal")
    f = pa.balance(x.to(DEV), K, alpha=0.0)
    expert = f["expert"].clone()
    dgate = torch.full((T, K), 0.5)
    expert[::2] = 7
    dgate[::2] = torch.tensor([2.0**27, 1.0, -(2.0**27), 1.0])
    expert[4] = torch.tensor([3, 9, 3, -1])
    dgate[4] = torch.tensor([1.0, 2.0, 4.0, float("nan")])
    got = pa.balance_bwd(x.to(DEV), f["lse"], expert, f["count"], f["n_valid"], torch.ones(1, device=DEV),
                         dgate=dgate.to(DEV), alpha=0.0)["dlogits"].cpu().double()
    p = torch.exp(x.double() - f["lse"].cpu().double()[:, None])
    gr = torch.zeros(T, E).double()
    at = expert.cpu().long()
    for t in range(T):
        if t == 4:
            gr[t, 3], gr[t, 9] = 5.0, 2.0
        elif t % 2 == 0:
            gr[t, 7] = 1.0
        else:
            gr[t, at[t]] = 0.5
    s = (gr * p).sum(1, keepdim=True)
    ref = p * (gr - s)
    # p is off by 2^-16 of itself at most (the file's bound for these logits),
    # the sums by less
    tol = p * 2.0**-15 * (gr + s) + UNIT[dtype] * ref.abs() + TINY[dtype]
    assert torch.all((got - ref).abs() <= tol)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,K", [(1500, 24, 3), (6000, 8, 2), (20_000, 8, 2), (20_011, 40, 9), (34_000, 160, 4),
                                   (20_000, 384, 8)])
def test_tokens_that_share_a_workgroup(T, E, K, dtype):
    # several wavefronts to a workgroup, and past 16,384 tokens (or fewer, of
    # many experts) several tokens to each group of lanes
    x = _logits(T, E, dtype, "ties" if T % 2 else "normal")
    g = torch.Generator().manual_seed(8)
    mask = (torch.rand(T, generator=g) < 0.9).to(torch.uint8)
    x[mask == 0] = float("nan")
    got = pa.balance(x.to(DEV), K, mask=mask.to(DEV), alpha=0.02)
    _check(got, _reference(x, K, mask, 0.02), x, T)
    assert int(got["dev_status"]) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,E,K", [(33_000, 24, 3), (70_003, 12, 5), (100_000, 160, 16)])
def test_gradient_of_tokens_that_share_a_row(T, E, K, dtype):
    # past 32,768 tokens each group of lanes takes several, one after the
    # other, and clears its row of gate gradients between them
    test_gradient(T, E, K, 0, dtype)
