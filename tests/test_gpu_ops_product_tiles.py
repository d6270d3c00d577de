"""Every tile and every way of taking parts and pieces that the matrix products
of argus_gated_ff and argus_cross_entropy choose from, against 64 bits, with the
tolerances of these operators' own tests. tests/test_product_plan.py checks on
the host that each size below is taken as it says."""
import pytest
import torch

import paper_2606_20374_amd as pa

from .test_gpu_ops_cross_entropy import _check_backward as _check_loss_backward
from .test_gpu_ops_cross_entropy import _check_forward as _check_loss
from .test_gpu_ops_cross_entropy import _data as _loss_data
from .test_gpu_ops_gated_ff import ACTS, _check_backward, _check_forward, _data

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F16 = torch.bfloat16, torch.float16

# (tokens, width, inner width, with g and u): (rows, columns, stages) of the tile
FORWARD = {
    (35, 24, 72, False): (64, 128, 4), (35, 24, 72, True): (64, 128, 4),
    (6_300, 40, 264, False): (64, 128, 2), (10_001, 24, 72, True): (64, 128, 2),
    (10_001, 520, 72, False): (128, 128, 2), (10_001, 1_400, 72, True): (128, 128, 2),
    (10_001, 24, 264, False): (128, 256, 2), (10_001, 24, 264, True): (128, 256, 2),
    (299, 1_104, 8_184, False): (192, 128, 2), (33_011, 264, 72, False): (192, 128, 2), (33_011, 520, 72, True): (192, 128, 2),
    (20_011, 136, 264, False): (256, 256, 2), (20_011, 72, 264, True): (256, 256, 2),
}
# (tokens, ids, width): the tile of the logits
LOSS = {(35, 72, 24): (64, 128, 4), (20_011, 72, 24): (64, 128, 2), (90, 50_021, 24): (128, 128, 2), (199, 50_021, 72): (256, 256, 2)}
# (tokens, width, inner width): (tile, four stages, dx in parts, dwg and dwu in parts)
FF_GRAD = {
    (35, 24, 72): (128, True, False, False), (1_300, 24, 72): (128, True, False, True),
    (35, 24, 520): (128, True, True, False), (1_300, 24, 1_000): (128, True, True, True),
    (999, 2_040, 520): (128, False, False, False), (33_011, 24, 72): (128, False, False, True),
    (35, 136, 8_200): (128, False, True, False), (4_003, 24, 2_056): (128, False, True, True),
    (4_003, 1_000, 2_056): (256, False, False, False), (20_011, 136, 520): (256, False, False, True),
    (701, 136, 12_000): (256, False, True, False), (4_003, 136, 4_104): (256, False, True, True),
}
# (tokens, ids, width): (tokens numbered, pieces, tile, four stages, dx in parts, dw in parts)
LOSS_GRAD = {
    (35, 72, 24): (False, 1, 128, True, False, False), (35, 2_056, 24): (False, 1, 128, True, True, False),
    (999, 2_056, 2_040): (False, 1, 128, False, False, False), (35, 50_021, 24): (False, 1, 128, False, True, False),
    (999, 20_011, 136): (False, 1, 256, False, True, False),
    (1_300, 1_000, 24): (True, 1, 128, True, False, False), (1_300, 72, 24): (True, 1, 128, True, False, True),
    (1_300, 8_200, 24): (True, 1, 128, True, True, False), (1_300, 2_056, 24): (True, 1, 128, True, True, True),
    (1_300, 1_000, 2_040): (True, 1, 128, False, False, False), (33_011, 72, 24): (True, 1, 128, False, False, True),
    (1_300, 20_011, 24): (True, 1, 128, False, True, False), (4_003, 4_104, 24): (True, 1, 128, False, True, True),
    (2_011, 2_056, 2_040): (True, 1, 256, False, False, False), (33_011, 1_000, 136): (True, 1, 256, False, False, True),
    (1_300, 20_011, 136): (True, 1, 256, False, True, False), (4_003, 8_200, 136): (True, 1, 256, False, True, True),
    (20_011, 12_000, 24): (True, 2, 128, True, False, True), (6_200, 50_021, 24): (True, 3, 128, True, True, False),
    (10_001, 20_011, 264): (True, 2, 128, False, False, False), (33_011, 4_104, 24): (True, 2, 128, False, False, True),
    (3_001, 50_021, 24): (True, 2, 128, False, True, False), (40_003, 4_104, 24): (True, 2, 128, False, True, True),
    (10_001, 20_011, 520): (True, 2, 256, False, False, False), (33_011, 4_104, 136): (True, 2, 256, False, False, True),
    (3_001, 50_021, 136): (True, 2, 256, False, True, False), (10_001, 20_011, 136): (True, 2, 256, False, True, True),
}


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("T,W,F,save", FORWARD)
def test_forward(T, W, F, save, dtype):
    x, wg, wu, _ = _data(T, W, F, dtype, 8)
    _check_forward(pa.gated_ff(x, wg, wu, ACTS[W // 8 % 3], save=save), x, wg, wu, ACTS[W // 8 % 3])


@pytest.mark.parametrize("T,V,W", LOSS)
def test_loss(T, V, W):
    x, w, labels = _loss_data(T, V, W, pad=8)
    _check_loss(pa.cross_entropy(x, w, labels, z_loss=1e-3), x, w, labels, 1.0, 1e-3)


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("T,W,F", FF_GRAD)
def test_feed_forward_gradient(T, W, F, dtype):
    act = ACTS[F // 8 % 3]
    x, wg, wu, dh = _data(T, W, F, dtype, 8)
    f = pa.gated_ff(x, wg, wu, act, save=True)
    _check_backward(pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"], act), dh, x, wg, wu, f["g"], f["u"], act)


# nearly all tokens learned, and few of them
@pytest.mark.parametrize("absent", [0.1, 0.9])
@pytest.mark.parametrize("T,V,W", LOSS_GRAD)
def test_loss_gradient(T, V, W, absent):
    x, w, labels = _loss_data(T, V, W, absent=absent, pad=8)
    f = pa.cross_entropy(x, w, labels, z_loss=1e-3)
    got = pa.cross_entropy_bwd(x, w, labels, f["lse"], f["n_valid"], dmean=torch.ones(1, device=DEV), z_loss=1e-3)
    c = torch.full((T,), 1 / int(f["n_valid"]), dtype=torch.float64, device=DEV)
    _check_loss_backward(got, x, w, labels, f["lse"], c, 1.0, 1e-3)
