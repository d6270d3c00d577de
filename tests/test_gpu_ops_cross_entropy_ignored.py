"""argus_cross_entropy_bwd where the vocabulary's rows hold infinities: a token
that is not learned has no gradient and gives none, at every size of call.

A logit of -infinity counts as an exponential of 0, so an id whose logits are
that for all learned tokens has a gradient of exactly 0, and dw of the others is
as without it: a probability off by ez + 2^-20 (1 + |z - lse|) of itself, dz and
dw rounded by 2^-8 each; in norm the two are off by sqrt(2 / 3) 2^-8 at most."""
import math

import pytest
import torch

import paper_2606_20374_amd as pa

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
# few tokens in one block and in two, over small and large vocabularies, some, and many
SIZES = [(9, 600, 64), (20, 600, 64), (9, 70_000, 16), (20, 70_000, 16), (100, 600, 64), (300, 1_031, 264), (2_000, 600, 64)]


def _data(T, V, W):
    g = torch.Generator(device=DEV).manual_seed(T + V + W)
    x = torch.randn(T, W, generator=g, device=DEV).to(BF)
    w = (torch.randn(V, W, generator=g, device=DEV) * W**-0.5).to(BF)
    labels = torch.randint(0, V, (T,), generator=g, device=DEV)
    labels[labels == 7] = 8
    labels[torch.rand(T, generator=g, device=DEV) < 0.4] = -100
    labels[:3] = torch.tensor([-1, V, 1])
    return x, w, labels


@pytest.mark.parametrize("T,V,W", SIZES)
def test_logits_of_minus_infinity(T, V, W):
    x, w, labels = _data(T, V, W)
    x[:, 5] = -x[:, 5].abs() - 0.1
    w[7, 5] = math.inf
    on = (labels >= 0) & (labels < V)
    x[~on, 5] = 1.0  # and +infinity for those that are not learned
    f = pa.cross_entropy(x, w, labels)
    b = pa.cross_entropy_bwd(x, w, labels, f["lse"], f["n_valid"], dmean=torch.ones(1, device=DEV))
    z = x[on].double() @ w.double().T
    assert (z[:, 7] == -math.inf).all() and f["mean"].isfinite().all()
    dz = torch.exp(z - f["lse"][on].double()[:, None])
    dz[torch.arange(len(dz), device=DEV), labels[on]] -= 1
    ref = dz.T @ x[on].double() / int(on.sum())
    assert not b["dw"][7].any()
    assert float((b["dw"].double() - ref).norm()) <= 2.0**-8 * float(ref.norm())
    assert not b["dx"][~on].any()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("T,V,W", SIZES)
def test_no_token_is_learned(T, V, W, bad):
    x, w, labels = _data(T, V, W)
    w[7, 5], w[V - 1] = bad, bad
    labels = torch.where(labels % 2 == 0, -1, V)
    f = pa.cross_entropy(x, w, labels)
    b = pa.cross_entropy_bwd(x, w, labels, f["lse"], f["n_valid"], dmean=torch.ones(1, device=DEV))
    assert not b["dw"].any() and not b["dx"].any() and float(f["mean"]) == 0
