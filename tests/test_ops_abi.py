"""The step operators' host side: what they refuse before any launch, and
their workspaces (no GPU needed)."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import argus as A
from paper_2606_20374_amd import ops

BF16, F16 = 1, 2
P = 0x10000  # an aligned address


def _call(fn, p, *args):
    return getattr(ops._lib(), fn)(ctypes.byref(p), *args)


def _embedding(**kw):
    p = ops.Embedding(P, 10, 1, 100, 64, BF16, BF16, 1.0, 64, None)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw", [dict(ids=None), dict(ids=P + 4), dict(n_tokens=-1), dict(n_tokens=2**28 + 1), dict(ids_64=2),
                                dict(n_vocab=0), dict(n_vocab=2**27 + 1), dict(dim=0), dict(dim=65_537), dict(dtype=3), dict(dtype=-1),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(row_stride=-1)])
def test_embedding_refuses(kw):
    p = _embedding(**kw)
    assert _call("argus_embedding", p, P, P, None) == A.EINVAL
    assert _call("argus_embedding_bwd", p, P, P, P, 1 << 40, None) == A.EINVAL


def test_embedding_refuses_pointers_and_workspace():
    p = _embedding()
    for table, out in ((None, P), (P, None), (P + 1, P), (P, P + 1)):
        assert _call("argus_embedding", p, table, out, None) == A.EINVAL
    need = ops._lib().argus_embedding_bwd_workspace(ctypes.byref(p))
    assert need == 512  # sorted keys and token numbers of 10 tokens
    for dout, dt, ws, n in ((None, P, P, need), (P, None, P, need), (P, P, None, need), (P, P, P + 64, need),
                            (P, P, P, need - 1)):
        assert _call("argus_embedding_bwd", p, dout, dt, ws, n, None) == A.EINVAL
    assert _call("argus_embedding_bwd", _embedding(grad_dtype=F16), P, P, P, need, None) == A.EINVAL


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=2**31), dict(cols=0), dict(cols=16_385), dict(dtype=7),
                                dict(weight_dtype=F16), dict(eps=-1.0), dict(eps=float("nan")), dict(x_stride=-1)])
def test_layer_norm_refuses(kw):
    p = ops.LayerNorm(4, 64, BF16, 0, 1e-5, 64, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    assert _call("argus_layer_norm", p, P, P, P, P, P, P, None) == A.EINVAL
    assert _call("argus_layer_norm_bwd", p, P, P, P, P, P, P, P, P, P, 1 << 40, None) == A.EINVAL


def test_layer_norm_refuses_pointers_and_workspace():
    p = ops.LayerNorm(4, 64, BF16, 0, 1e-5, 64, 64)
    ok = [P, P, P, P, P, P]
    for i in (0, 1, 3, 4, 5):  # the bias may be left out
        assert _call("argus_layer_norm", p, *[None if j == i else a for j, a in enumerate(ok)], None) == A.EINVAL
    for i, odd in ((0, 1), (1, 2), (2, 2), (3, 1), (4, 2), (5, 2)):
        assert _call("argus_layer_norm", p, *[a + odd if j == i else a for j, a in enumerate(ok)], None) == A.EINVAL
    need = ops._lib().argus_layer_norm_bwd_workspace(ctypes.byref(p))
    ok = [P] * 9
    for i in (0, 1, 2, 3, 4, 5, 6, 8):  # dbias may be left out
        assert _call("argus_layer_norm_bwd", p, *[None if j == i else a for j, a in enumerate(ok)], need, None) == A.EINVAL
    assert _call("argus_layer_norm_bwd", p, *ok, need - 1, None) == A.EINVAL
    p.dy_stride = -1
    assert _call("argus_layer_norm_bwd", p, *ok, need, None) == A.EINVAL


@pytest.mark.parametrize("kw", [dict(n_tokens=-1), dict(n_experts=0), dict(n_experts=1025), dict(top_k=0), dict(top_k=17),
                                dict(n_experts=4, top_k=5), dict(dtype=3), dict(alpha=float("inf")), dict(row_stride=-1)])
def test_balance_refuses(kw):
    p = ops.Balance(10, 64, 8, 0, 0.01, 64)
    for k, v in kw.items():
        setattr(p, k, v)
    o = ops.BalanceOut(*([P] * 7 + [None]))
    assert _call("argus_balance", p, P, None, ctypes.byref(o), P, 1 << 40, None) == A.EINVAL
    assert _call("argus_balance_bwd", p, P, P, P, P, P, P, None, P, None) == A.EINVAL
    assert ops._lib().argus_balance_workspace(ctypes.byref(p)) == 0


def test_balance_refuses_pointers_and_workspace():
    p = ops.Balance(10, 64, 8, 0, 0.01, 64)
    need = ops._lib().argus_balance_workspace(ctypes.byref(p))
    assert need > 0
    for f in ops.BALANCE_FIELDS[:-1]:
        o = ops.BalanceOut(*([P] * 7 + [None]))
        setattr(o, f, None)
        assert _call("argus_balance", p, P, None, ctypes.byref(o), P, need, None) == A.EINVAL, f
    o = ops.BalanceOut(*([P] * 7 + [None]))
    for logits, ws, n in ((None, P, need), (P + 2, P, need), (P, None, need), (P, P + 8, need), (P, P, need - 1)):
        assert _call("argus_balance", p, logits, None, ctypes.byref(o), ws, n, None) == A.EINVAL
    ok = [P] * 8
    for i in (0, 1, 3, 4, 5, 7):
        assert _call("argus_balance_bwd", p, *[None if j == i else a for j, a in enumerate(ok)], None) == A.EINVAL
    assert _call("argus_balance_bwd", p, P, P, None, P, P, P, P, P, None) == A.EINVAL  # dgate without experts


def _attention(**kw):
    p = ops.Attention(2, 8, 2, 64, 1, BF16, 0.125, 100, 100, P, P, 512, 64, 128, 64, 128, 64, None)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw", [dict(n_docs=0), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=9), dict(n_heads=65_536),
                                dict(head_dim=0), dict(head_dim=60), dict(head_dim=136), dict(causal=2), dict(dtype=0),
                                dict(dtype=F16), dict(scale=float("nan")), dict(scale=-1.0), dict(n_q=-1), dict(n_k=2**31),
                                dict(q_off=None), dict(k_off=None), dict(q_off=P + 4), dict(q_tok=56), dict(q_tok=516),
                                dict(k_head=32), dict(v_tok=2**31), dict(q_off=None, k_off=None)])
def test_attention_refuses(kw):
    p = _attention(**kw)
    assert _call("argus_attention", p, P, P, P, P, P, P, 1 << 40, None) == A.EINVAL
    assert _call("argus_attention_bwd", p, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == A.EINVAL
    assert ops._lib().argus_attention_workspace(ctypes.byref(p)) == 0
    assert ops._lib().argus_attention_bwd_workspace(ctypes.byref(p)) == 0


def test_attention_refuses_pointers_and_workspace():
    p = _attention()
    need = ops._lib().argus_attention_workspace(ctypes.byref(p))
    ok = [P] * 6
    for i in range(6):
        assert _call("argus_attention", p, *[None if j == i else a for j, a in enumerate(ok)], need, None) == A.EINVAL
    for i in range(4):
        assert _call("argus_attention", p, *[a + 8 if j == i else a for j, a in enumerate(ok)], need, None) == A.EINVAL
    assert _call("argus_attention", p, *ok, need - 1, None) == A.EINVAL
    need = ops._lib().argus_attention_bwd_workspace(ctypes.byref(p))
    ok = [P] * 10
    for i in range(10):
        assert _call("argus_attention_bwd", p, *[None if j == i else a for j, a in enumerate(ok)], need, None) == A.EINVAL
    assert _call("argus_attention_bwd", p, *ok, need - 1, None) == A.EINVAL


def test_null_descriptors():
    L = ops._lib()
    o = ops.BalanceOut(*([P] * 7 + [None]))
    assert L.argus_embedding(None, P, P, None) == A.EINVAL
    assert L.argus_embedding_bwd(None, P, P, P, 256, None) == A.EINVAL
    assert L.argus_layer_norm(None, P, P, P, P, P, P, None) == A.EINVAL
    assert L.argus_layer_norm_bwd(None, P, P, P, P, P, P, P, P, P, 256, None) == A.EINVAL
    assert L.argus_balance(None, P, P, ctypes.byref(o), P, 256, None) == A.EINVAL
    assert L.argus_balance(ctypes.byref(ops.Balance(10, 64, 8, 0, 0.01, 64)), P, P, None, P, 1 << 30, None) == A.EINVAL
    assert L.argus_balance_bwd(None, P, P, P, P, P, P, P, P, None) == A.EINVAL
    assert L.argus_attention(None, P, P, P, P, P, P, 256, None) == A.EINVAL
    assert L.argus_attention_bwd(None, P, P, P, P, P, P, P, P, P, P, 256, None) == A.EINVAL
    for f in ("embedding_bwd", "layer_norm_bwd", "balance", "attention", "attention_bwd"):
        assert getattr(L, f"argus_{f}_workspace")(None) == 0


def test_binding_refuses_other_types_and_shapes():
    x = torch.zeros(4, 8)
    with pytest.raises(AssertionError):
        pa.layer_norm(x, torch.ones(8))  # host memory
    with pytest.raises(pa.ArgusError):
        ops._dtype(x.double())
    with pytest.raises(pa.ArgusError):
        ops._need(x, (4, 9), torch.float32, "x")
    with pytest.raises(pa.ArgusError):
        ops._need(x, (4, 8), torch.bfloat16, "x")


def test_refuses_misaligned_outputs_statistics_and_status():
    need = lambda fn, p: getattr(ops._lib(), fn)(ctypes.byref(p))  # noqa: E731
    p = ops.Balance(10, 64, 8, 0, 0.01, 64)
    ws = need("argus_balance_workspace", p)
    for f in ops.BALANCE_FIELDS:
        o = ops.BalanceOut(*([P] * 8))
        setattr(o, f, P + 2)
        assert _call("argus_balance", p, P, None, ctypes.byref(o), P, ws, None) == A.EINVAL, f
    for i in range(8):  # logits, lse, expert, count, n_valid, dloss, dgate, dlogits
        assert _call("argus_balance_bwd", p, *[P + 2 if j == i else P for j in range(8)], None) == A.EINVAL, i
    p = _embedding(dev_status=P + 2)
    assert _call("argus_embedding", p, P, P, None) == A.EINVAL
    assert _call("argus_embedding_bwd", p, P, P, P, need("argus_embedding_bwd_workspace", p), None) == A.EINVAL
    p = _attention(dev_status=P + 1)
    assert _call("argus_attention", p, *[P] * 7, 1 << 40, None) == A.EINVAL
    assert _call("argus_attention_bwd", p, *[P] * 11, 1 << 40, None) == A.EINVAL


def test_host_tensors_are_refused_also_without_assertions():
    # python -O leaves assert statements out; a host address must not get to a kernel
    code = """if True:
        import torch
        from paper_2606_20374_amd import argus, ops
        x = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
        for call in (lambda: argus._ptr(x), lambda: ops._row(x[0]), lambda: ops._heads(x, "q")):
            try:
                call()
            except AssertionError:
                continue
            raise SystemExit(3)
    """
    root = os.path.dirname(os.path.dirname(os.path.abspath(pa.__file__)))
    assert subprocess.run([sys.executable, "-O", "-c", code], cwd=root).returncode == 0


def test_launches_go_to_the_tensors_device(monkeypatch):
    # device 0 is current and the tensors lie on device 1: its null stream is
    # only its own while it is current
    now, seen = [0], []

    class Guard:
        def __init__(self, device):
            self.to = device.index

        def __enter__(self):
            self.back, now[0] = now[0], self.to

        def __exit__(self, *exc):
            now[0] = self.back

    class Tensor:
        """Enough of a [4, 8] float tensor on device 1."""
        device, is_cuda, dtype, shape = torch.device("cuda", 1), True, torch.float32, (4, 8)

        def __init__(self, *shape, dtype=torch.float32):
            self.shape, self.dtype = shape, dtype

        dim = lambda self: len(self.shape)  # noqa: E731
        data_ptr = lambda self: P  # noqa: E731
        stride = lambda self, i: self.shape[1] if i == 0 else 1  # noqa: E731
        is_contiguous = lambda self: True  # noqa: E731

    class Lib:
        @staticmethod
        def argus_layer_norm(*args):
            seen.append((now[0], args[-1]))
            return A.OK

    monkeypatch.setattr(ops, "_lib", lambda: Lib)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 70 + i, raising=False)
    out = {"y": Tensor(4, 8), "mean": Tensor(4), "rstd": Tensor(4)}
    for now[0] in (0, 1):
        before = now[0]
        pa.layer_norm(Tensor(4, 8), Tensor(8), out=out)
        assert seen.pop() == (1, 71) and now[0] == before
