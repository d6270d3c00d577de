"""The choice of tiles, parts and pieces of the step operators' matrix products
(CPU): a launch that any size inside the operators' limits can have, and that
the sizes which test each choice on the GPU are still taken that way."""
import ctypes
import itertools
import os

import pytest

from .test_gpu_ops_product_tiles import FF_GRAD, FORWARD, LOSS, LOSS_GRAD

PROBE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "probe", "libproductplanprobe.so")


def _probe():
    if not os.path.exists(PROBE):
        import tests.probe.build
        tests.probe.build.build()
    L, I64, I32, V = ctypes.CDLL(PROBE), ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p
    L.probe_forward_tile.argtypes, L.probe_forward_tile.restype = [I64, I64, I64, I32, I32, V], None
    L.probe_gradient_plan.argtypes, L.probe_gradient_plan.restype = [I64] * 5 + [V], None
    L.probe_loss_call.argtypes, L.probe_loss_call.restype = [I64, I32, I32, V], None
    return L


def forward_tile(rows, cols, k, loss=False, three=False):
    """(rows, columns, threads, stages) of a forward product's tile."""
    out = (ctypes.c_int32 * 4)()
    _probe().probe_forward_tile(rows, cols, k, loss, three, out)
    return tuple(out)


def gradient_plan(rows_x, k_x, rows_w, k_w, cols):
    """(tile, four stages, parts of the input's gradient, of the weights', threads, workgroups)."""
    out = (ctypes.c_int64 * 6)()
    _probe().probe_gradient_plan(rows_x, k_x, rows_w, k_w, cols, out)
    return out[0], bool(out[1]), *out[2:]


MOST = 2**32 - 1  # threads of a launch along one axis


@pytest.mark.parametrize("k", [8, 64, 512, 4_096, 16_384])
@pytest.mark.parametrize("tokens", [2**n for n in range(6, 21)] + [2**20 - 1, 2**19 + 1])
def test_forward_launches(tokens, k):
    for cols in (8, 2**13, 2**17, 2**18, 2**19 - 1, 2**20):
        for loss in (False, True):
            # feed-forward has up to 2 x 131,072 columns, the loss below 2^38 logits
            if tokens * cols >= 2**38 if loss else cols > 2**18:
                continue
            for three in (False,) if loss else (False, True):
                tm, tn, threads, _ = forward_tile(tokens, cols, k, loss, three)
                assert -(-tokens // tm) * -(-cols // tn) * threads <= MOST, (cols, loss, three)


@pytest.mark.parametrize("width", [8, 512, 16_384, 65_536])
@pytest.mark.parametrize("tokens", [1, 1_000, 2**16, 2**20])
def test_gradient_launches(tokens, width):
    for inner in (8, 4_096, 2**17):
        wide = -(-inner // 64) * 64
        plans = [gradient_plan(tokens, 2 * wide, 2 * wide, tokens, width)]
        if width <= 16_384:
            plans.append(gradient_plan(tokens, wide, wide, tokens, width))
        for _, _, sx, sw, threads, groups in plans:
            assert 1 <= sx <= 64 and 1 <= sw <= 64 and groups * threads <= MOST, inner
            # joins of parts: eight sums to a thread
            assert sx == 1 or tokens * width // 8 <= MOST
            assert sw == 1 or 2 * wide * width // 8 <= MOST


def _tile(tm, tn, threads, stages):
    return tm, tn, stages


def _feed_forward_plan(T, W, F):
    wide = -(-F // 64) * 64
    tile, deep, sx, sw, _, _ = gradient_plan(T, 2 * wide, 2 * wide, T, W)
    return tile, deep, sx > 1, sw > 1


def _loss_plan(T, V, W):
    out = (ctypes.c_int64 * 3)()
    _probe().probe_loss_call(T, V, W, out)
    few, small, ids = out
    tile, deep, sx, sw, _, _ = gradient_plan(T, ids, ids, T, W)
    assert not few
    return not small, -(-V // ids), tile, deep, sx > 1, sw > 1


def test_the_tested_sizes_take_every_tile():
    assert {c: _tile(*forward_tile(c[0], 2 * c[2], c[1], three=c[3])) for c in FORWARD} == FORWARD
    assert {c: _tile(*forward_tile(*c, loss=True)) for c in LOSS} == LOSS
    tiles = {(64, 128, 4), (64, 128, 2), (128, 128, 2), (128, 256, 2), (192, 128, 2), (256, 256, 2)}
    for three in (False, True):
        assert {t for c, t in FORWARD.items() if c[3] == three} == tiles
    assert set(LOSS.values()) == tiles - {(128, 256, 2), (192, 128, 2)}


def test_the_tested_sizes_take_all_parts_and_pieces():
    assert {c: _feed_forward_plan(*c) for c in FF_GRAD} == FF_GRAD
    assert {c: _loss_plan(*c) for c in LOSS_GRAD} == LOSS_GRAD
    tiles, either = [(128, True), (128, False), (256, False)], [False, True]
    assert set(FF_GRAD.values()) == {(*t, x, w) for t, x, w in itertools.product(tiles, either, either)}
    # numbered tokens: one piece in every way, several but for two that no size was found for
    one = {p[2:] for p in LOSS_GRAD.values() if p[0] and p[1] == 1}
    more = {p[2:] for p in LOSS_GRAD.values() if p[0] and p[1] > 1}
    assert one == set(FF_GRAD.values())
    assert more == one - {(128, True, False, False), (128, True, True, True)}
