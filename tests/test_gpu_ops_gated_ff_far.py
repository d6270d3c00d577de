"""argus_gated_ff far from 0: gates whose square or cube leaves 32 bits, where
the activation is the gate itself or 0 and its derivative 1 or 0, exactly."""
import pytest
import torch

import paper_2606_20374_amd as pa

from .test_gpu_ops_gated_ff import ACTS

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [1, 40])
def test_far_gates(T, act):
    F, W = 16, 8
    far = torch.tensor([1e3, 1e10, 1e13, 1e18, 2e19, 1e25, 1e30, 3e38], device=DEV).to(BF)
    g = torch.cat([far, -far])
    want, slope = torch.where(g > 0, g, 0), (g > 0).to(BF)
    x, w = torch.zeros(T, W, dtype=BF, device=DEV), torch.zeros(F, W, dtype=BF, device=DEV)
    x[:, 0], x[0, 1] = 1, 1  # one token alone reaches the weights' second column
    wg, wu = w.clone(), w.clone()
    wg[:, 0], wu[:, 0] = g, 1
    f = pa.gated_ff(x, wg, wu, act, save=True)
    assert (f["h"] == want).all() and (f["g"] == g).all()
    dh = torch.ones(T, F, dtype=BF, device=DEV)
    b = pa.gated_ff_bwd(dh, x, torch.zeros_like(wg), torch.zeros_like(wu), f["g"], f["u"], act)
    assert (b["dwg"][:, 1] == slope).all() and (b["dwu"][:, 1] == want).all() and not b["dx"].any()
