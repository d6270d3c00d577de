"""Thin Python binding of the step operators of libargus (include/argus_ops.h).

Argument marshalling only, as in argus.py: torch supplies device memory and
the current stream, the kernels of libargus.so do the rest. Every call
returns a dict of its outputs; `out` takes one that an alloc_* function or an
earlier call of the same sizes made. Inputs may be slices of wider tensors
(any row stride) as long as their last dimension is contiguous.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from .argus import ArgusError, _check, _ptr, lib

DEV_TOKEN_RANGE, DEV_LOGITS = 512, 1024
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

V, I32, I64, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class Embedding(ctypes.Structure):
    _fields_ = [("ids", V), ("n_tokens", I64), ("ids_64", I32), ("n_vocab", I32), ("dim", I32), ("dtype", I32),
                ("grad_dtype", I32), ("scale", F32), ("row_stride", I64), ("dev_status", V)]


class LayerNorm(ctypes.Structure):
    _fields_ = [("rows", I64), ("cols", I32), ("dtype", I32), ("weight_dtype", I32), ("eps", F32),
                ("x_stride", I64), ("dy_stride", I64)]


class Balance(ctypes.Structure):
    _fields_ = [("n_tokens", I64), ("n_experts", I32), ("top_k", I32), ("dtype", I32), ("alpha", F32),
                ("row_stride", I64)]


BALANCE_FIELDS = ["expert", "gate", "lse", "count", "prob", "n_valid", "loss", "dev_status"]


class BalanceOut(ctypes.Structure):
    _fields_ = [(f, V) for f in BALANCE_FIELDS]


class Attention(ctypes.Structure):
    _fields_ = [("n_docs", I32), ("n_heads", I32), ("n_kv_heads", I32), ("head_dim", I32), ("causal", I32),
                ("dtype", I32), ("scale", F32), ("n_q", I64), ("n_k", I64), ("q_off", V), ("k_off", V),
                ("q_tok", I64), ("q_head", I64), ("k_tok", I64), ("k_head", I64), ("v_tok", I64), ("v_head", I64),
                ("dev_status", V)]


_bound = None


def _lib():
    """libargus with the step operators' signatures."""
    global _bound
    if _bound is None:
        L = lib()
        P, S = ctypes.POINTER, ctypes.c_size_t
        for name, args in {
            "argus_embedding": [P(Embedding), V, V, V],
            "argus_embedding_bwd": [P(Embedding), V, V, V, S, V],
            "argus_layer_norm": [P(LayerNorm), V, V, V, V, V, V, V],
            "argus_layer_norm_bwd": [P(LayerNorm), V, V, V, V, V, V, V, V, V, S, V],
            "argus_balance": [P(Balance), V, V, P(BalanceOut), V, S, V],
            "argus_balance_bwd": [P(Balance), V, V, V, V, V, V, V, V, V],
            "argus_attention": [P(Attention), V, V, V, V, V, V, S, V],
            "argus_attention_bwd": [P(Attention), V, V, V, V, V, V, V, V, V, V, S, V],
        }.items():
            getattr(L, name).argtypes, getattr(L, name).restype = args, ctypes.c_int
        for name, arg in {"argus_embedding_bwd_workspace": Embedding, "argus_layer_norm_bwd_workspace": LayerNorm,
                          "argus_balance_workspace": Balance, "argus_attention_workspace": Attention,
                          "argus_attention_bwd_workspace": Attention}.items():
            getattr(L, name).argtypes, getattr(L, name).restype = [P(arg)], S
        _bound = L
    return _bound


def _dtype(t: torch.Tensor) -> int:
    if t.dtype not in DTYPES:
        raise ArgusError(f"element type {t.dtype}: float32, bfloat16 or float16 expected")
    return DTYPES[t.dtype]


def _row(t: torch.Tensor):
    """(address, row stride) of a 2-D device tensor with contiguous rows."""
    if not (t.is_cuda and t.dim() == 2):
        raise AssertionError("libargus takes 2-D device tensors of rows")
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise AssertionError("the last dimension has to be contiguous")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _need(t: torch.Tensor, shape: tuple, dtype, what: str):
    if t.shape != shape or t.dtype != dtype:
        raise ArgusError(f"{what}: {t.dtype} {tuple(t.shape)}, expected {dtype} {shape}")


def _empty(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


def _call(name: str, device, *args):
    """Calls an entry point on the device's current stream, with the device
    current: its null stream is another device's otherwise."""
    fn = getattr(_lib(), name)
    if device.index != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return _call(name, device, *args)
    # the stream's handle alone: a torch Stream object costs more than a small
    # operator's launches
    _check(fn(*args, torch._C._cuda_getCurrentRawStream(device.index)), name)


def _space(out: dict, need: int, device):
    """The dict's workspace, made or replaced where it is too small."""
    ws = out.get("_workspace")
    if ws is None or ws.numel() < need:
        ws = out["_workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    return ws


# ------------------------------------------------------------------ embedding
def _embedding(ids, n_vocab, dim, dtype, grad_dtype, scale, stride, status) -> Embedding:
    if ids.dtype not in (torch.int32, torch.int64):
        raise ArgusError(f"token ids of {ids.dtype}: int32 or int64 expected")
    return Embedding(_ptr(ids), ids.numel(), int(ids.dtype == torch.int64), n_vocab, dim, dtype, grad_dtype, scale,
                     stride, _ptr(status))


def alloc_embedding(n_tokens: int, dim: int, dtype, device="cuda") -> dict:
    return {"out": _empty((n_tokens, dim), dtype, device), "dev_status": _empty(1, torch.int32, device)}


def embedding(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0, out: Optional[dict] = None) -> dict:
    """argus_embedding: out[t] = scale * table[ids[t]]; an id below 0 is
    padding, one past the table raises DEV_TOKEN_RANGE in dev_status; both
    give zeros."""
    n, dim = ids.numel(), table.shape[1]
    if out is None:
        out = alloc_embedding(n, dim, table.dtype, table.device)
    at, stride = _row(table)
    dt = _dtype(table)
    _need(out["out"], (n, dim), table.dtype, "embedding: out")
    p = _embedding(ids, table.shape[0], dim, dt, dt, scale, stride, out.get("dev_status"))
    _call("argus_embedding", table.device, ctypes.byref(p), at, _ptr(out["out"]))
    return out


def alloc_embedding_bwd(n_vocab: int, dim: int, dtype, device="cuda") -> dict:
    return {"dtable": _empty((n_vocab, dim), dtype, device), "dev_status": _empty(1, torch.int32, device)}


def embedding_bwd(ids: torch.Tensor, dout: torch.Tensor, n_vocab: int, scale: float = 1.0, dtype=None,
                  out: Optional[dict] = None) -> dict:
    """argus_embedding_bwd: dtable[v] = scale * sum of dout[t] over ids[t] = v,
    in dtype (dout's, or float32)."""
    _need(dout, (ids.numel(), dout.shape[-1]), dout.dtype, "embedding_bwd: dout")
    dim = dout.shape[1]
    if out is None:
        out = alloc_embedding_bwd(n_vocab, dim, dtype or dout.dtype, dout.device)
    at, stride = _row(dout)
    _need(out["dtable"], (n_vocab, dim), out["dtable"].dtype, "embedding_bwd: dtable")
    p = _embedding(ids, n_vocab, dim, _dtype(dout), _dtype(out["dtable"]), scale, stride, out.get("dev_status"))
    ws = _space(out, _lib().argus_embedding_bwd_workspace(ctypes.byref(p)), dout.device)
    _call("argus_embedding_bwd", dout.device, ctypes.byref(p), at, _ptr(out["dtable"]), _ptr(ws), ws.numel())
    return out


# ----------------------------------------------------------------- layer norm
def alloc_layer_norm(rows: int, cols: int, dtype, device="cuda") -> dict:
    return {"y": _empty((rows, cols), dtype, device), "mean": _empty(rows, torch.float32, device),
            "rstd": _empty(rows, torch.float32, device)}


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               out: Optional[dict] = None) -> dict:
    """argus_layer_norm over the rows of x [rows, cols]; weight and bias in
    x's type or float32."""
    at, stride = _row(x)
    rows, cols = x.shape
    if out is None:
        out = alloc_layer_norm(rows, cols, x.dtype, x.device)
    _need(weight, (cols,), weight.dtype, "layer_norm: weight")
    if bias is not None:
        _need(bias, (cols,), weight.dtype, "layer_norm: bias")
    _need(out["y"], (rows, cols), x.dtype, "layer_norm: y")
    _need(out["mean"], (rows,), torch.float32, "layer_norm: mean")
    _need(out["rstd"], (rows,), torch.float32, "layer_norm: rstd")
    p = LayerNorm(rows, cols, _dtype(x), _dtype(weight), eps, stride, 0)
    _call("argus_layer_norm", x.device, ctypes.byref(p), at, _ptr(weight), _ptr(bias), _ptr(out["y"]),
          _ptr(out["mean"]), _ptr(out["rstd"]))
    return out


def alloc_layer_norm_bwd(rows: int, cols: int, dtype, weight_dtype, bias: bool = True, device="cuda") -> dict:
    out = {"dx": _empty((rows, cols), dtype, device), "dweight": _empty(cols, weight_dtype, device)}
    if bias:
        out["dbias"] = _empty(cols, weight_dtype, device)
    return out


def layer_norm_bwd(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor,
                   bias: bool = True, out: Optional[dict] = None) -> dict:
    """argus_layer_norm_bwd: dx, dweight and, with bias, dbias from dy and the
    forward's x, mean and rstd."""
    at, stride = _row(x)
    dat, dstride = _row(dy)
    rows, cols = x.shape
    if out is None:
        out = alloc_layer_norm_bwd(rows, cols, x.dtype, weight.dtype, bias, x.device)
    _need(dy, (rows, cols), x.dtype, "layer_norm_bwd: dy")
    _need(mean, (rows,), torch.float32, "layer_norm_bwd: mean")
    _need(rstd, (rows,), torch.float32, "layer_norm_bwd: rstd")
    _need(weight, (cols,), weight.dtype, "layer_norm_bwd: weight")
    _need(out["dx"], (rows, cols), x.dtype, "layer_norm_bwd: dx")
    _need(out["dweight"], (cols,), weight.dtype, "layer_norm_bwd: dweight")
    if bias:
        _need(out["dbias"], (cols,), weight.dtype, "layer_norm_bwd: dbias")
    p = LayerNorm(rows, cols, _dtype(x), _dtype(weight), 0.0, stride, dstride)
    ws = _space(out, _lib().argus_layer_norm_bwd_workspace(ctypes.byref(p)), x.device)
    _call("argus_layer_norm_bwd", x.device, ctypes.byref(p), dat, at, _ptr(mean), _ptr(rstd), _ptr(weight),
          _ptr(out["dx"]), _ptr(out["dweight"]), _ptr(out["dbias"]) if bias else None, _ptr(ws), ws.numel())
    return out


# -------------------------------------------------------------------- balance
def alloc_balance(n_tokens: int, n_experts: int, top_k: int, device="cuda") -> dict:
    # two allocations in place of eight: a small router's time is its host time
    nk = n_tokens * top_k
    gate, lse, prob, loss = _empty(nk + n_tokens + n_experts + 1, torch.float32, device).split([nk, n_tokens, n_experts, 1])
    expert, count, n_valid, status = _empty(nk + n_experts + 2, torch.int32, device).split([nk, n_experts, 1, 1])
    return {"expert": expert.view(n_tokens, top_k), "gate": gate.view(n_tokens, top_k), "lse": lse, "count": count,
            "prob": prob, "n_valid": n_valid, "loss": loss, "dev_status": status}


def balance(logits: torch.Tensor, top_k: int, mask: Optional[torch.Tensor] = None, alpha: float = 0.01,
            out: Optional[dict] = None) -> dict:
    """argus_balance: the top_k experts and gates of each token, tokens per
    expert (count), mean probabilities (prob) and the balance loss. mask:
    bool or uint8, 0 leaves a token out."""
    at, stride = _row(logits)
    n, E = logits.shape
    if out is None:
        out = alloc_balance(n, E, top_k, logits.device)
    for f, shape, dt in (("expert", (n, top_k), torch.int32), ("gate", (n, top_k), torch.float32),
                         ("lse", (n,), torch.float32), ("count", (E,), torch.int32), ("prob", (E,), torch.float32)):
        _need(out[f], shape, dt, "balance: " + f)
    if mask is not None:
        _need(mask, (n,), torch.bool if mask.dtype == torch.bool else torch.uint8, "balance: mask")
    p = Balance(n, E, top_k, _dtype(logits), alpha, stride)
    o = BalanceOut(*[_ptr(out.get(f)) for f in BALANCE_FIELDS])
    ws = _space(out, _lib().argus_balance_workspace(ctypes.byref(p)), logits.device)
    _call("argus_balance", logits.device, ctypes.byref(p), at, _ptr(mask), ctypes.byref(o), _ptr(ws), ws.numel())
    return out


def balance_bwd(logits: torch.Tensor, lse: torch.Tensor, expert: torch.Tensor, count: torch.Tensor,
                n_valid: torch.Tensor, dloss: torch.Tensor, dgate: Optional[torch.Tensor] = None, alpha: float = 0.01,
                out: Optional[dict] = None) -> dict:
    """argus_balance_bwd: dlogits from the forward's lse, expert, count and
    n_valid, the gradient dloss [1] of the loss and, where given, dgate of the
    gates."""
    at, stride = _row(logits)
    n, E = logits.shape
    if out is None:
        out = {"dlogits": _empty((n, E), logits.dtype, logits.device)}
    top_k = expert.shape[1]
    _need(lse, (n,), torch.float32, "balance_bwd: lse")
    _need(expert, (n, top_k), torch.int32, "balance_bwd: expert")
    _need(count, (E,), torch.int32, "balance_bwd: count")
    _need(n_valid, (1,), torch.int32, "balance_bwd: n_valid")
    _need(dloss, (1,), torch.float32, "balance_bwd: dloss")
    if dgate is not None:
        _need(dgate, (n, top_k), torch.float32, "balance_bwd: dgate")
    _need(out["dlogits"], (n, E), logits.dtype, "balance_bwd: dlogits")
    p = Balance(n, E, top_k, _dtype(logits), alpha, stride)
    _call("argus_balance_bwd", logits.device, ctypes.byref(p), at, _ptr(lse), _ptr(expert), _ptr(count),
          _ptr(n_valid), _ptr(dloss), _ptr(dgate), _ptr(out["dlogits"]))
    return out


# ------------------------------------------------------------------ attention
def _heads(t: torch.Tensor, what: str):
    """(address, token stride, head stride) of a [tokens, heads, dim] tensor."""
    if not (t.is_cuda and t.dim() == 3):
        raise AssertionError("libargus takes [tokens, heads, dim] device tensors")
    if t.dtype != torch.bfloat16:
        raise ArgusError(f"{what} of {t.dtype}: attention takes bfloat16")
    if t.stride(2) != 1:
        raise AssertionError("the last dimension has to be contiguous")
    n, h, d = t.shape
    # a dimension of one has no use for its stride, which may lie outside the limits
    return t.data_ptr(), t.stride(0) if n > 1 else d, t.stride(1) if h > 1 else d


def _attention(q, k, v, q_off, k_off, causal, scale, status):
    if k_off is None:
        k_off = q_off
    if (q_off is None) != (k_off is None):
        raise ArgusError("attention: k_off without q_off")
    if q_off is not None and (q_off.dtype != torch.int64 or k_off.dtype != torch.int64):
        raise ArgusError("attention: document offsets are int64")
    if q_off is not None and (q_off.numel() < 2 or q_off.shape != k_off.shape):
        raise ArgusError("attention: q_off and k_off hold n_docs + 1 offsets each")
    (qa, qt, qh), (ka, kt, kh), (va, vt, vh) = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
    _need(v, k.shape, torch.bfloat16, "attention: v")
    if q.shape[2] != k.shape[2]:
        raise ArgusError("attention: q and k have different head dimensions")
    p = Attention(1 if q_off is None else q_off.numel() - 1, q.shape[1], k.shape[1], q.shape[2], int(bool(causal)),
                  DTYPES[torch.bfloat16], 1.0 / math.sqrt(q.shape[2]) if scale is None else scale, q.shape[0],
                  k.shape[0], _ptr(q_off), _ptr(k_off), qt, qh, kt, kh, vt, vh, _ptr(status))
    return p, qa, ka, va


def alloc_attention(n_q: int, n_heads: int, head_dim: int, device="cuda") -> dict:
    return {"o": _empty((n_q, n_heads, head_dim), torch.bfloat16, device),
            "lse": _empty((n_q, n_heads), torch.float32, device), "dev_status": _empty(1, torch.int32, device)}


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_off: Optional[torch.Tensor] = None,
              k_off: Optional[torch.Tensor] = None, causal: bool = True, scale: Optional[float] = None,
              out: Optional[dict] = None) -> dict:
    """argus_attention: o and lse of q [n_q, heads, dim] over k and v [n_k,
    kv_heads, dim], inside the documents of q_off and k_off (int64; k_off
    defaults to q_off, no offsets: one document)."""
    if out is None:
        out = alloc_attention(q.shape[0], q.shape[1], q.shape[2], q.device)
    _need(out["o"], q.shape, torch.bfloat16, "attention: o")
    _need(out["lse"], q.shape[:2], torch.float32, "attention: lse")
    p, qa, ka, va = _attention(q, k, v, q_off, k_off, causal, scale, out.get("dev_status"))
    ws = _space(out, _lib().argus_attention_workspace(ctypes.byref(p)), q.device)
    _call("argus_attention", q.device, ctypes.byref(p), qa, ka, va, _ptr(out["o"]), _ptr(out["lse"]), _ptr(ws),
          ws.numel())
    return out


def alloc_attention_bwd(n_q: int, n_k: int, n_heads: int, n_kv_heads: int, head_dim: int, device="cuda") -> dict:
    return {"dq": _empty((n_q, n_heads, head_dim), torch.bfloat16, device),
            "dk": _empty((n_k, n_kv_heads, head_dim), torch.bfloat16, device),
            "dv": _empty((n_k, n_kv_heads, head_dim), torch.bfloat16, device),
            "dev_status": _empty(1, torch.int32, device)}


def attention_bwd(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor,
                  lse: torch.Tensor, q_off: Optional[torch.Tensor] = None, k_off: Optional[torch.Tensor] = None,
                  causal: bool = True, scale: Optional[float] = None, out: Optional[dict] = None) -> dict:
    """argus_attention_bwd: dq, dk and dv from do and the forward's q, k, v, o
    and lse."""
    if out is None:
        out = alloc_attention_bwd(q.shape[0], k.shape[0], q.shape[1], k.shape[1], q.shape[2], q.device)
    for t, what in ((do, "do"), (o, "o"), (out["dq"], "dq")):
        _need(t, q.shape, torch.bfloat16, "attention_bwd: " + what)
    for t, what in ((out["dk"], "dk"), (out["dv"], "dv")):
        _need(t, k.shape, torch.bfloat16, "attention_bwd: " + what)
    _need(lse, q.shape[:2], torch.float32, "attention_bwd: lse")
    p, qa, ka, va = _attention(q, k, v, q_off, k_off, causal, scale, out.get("dev_status"))
    ws = _space(out, _lib().argus_attention_bwd_workspace(ctypes.byref(p)), q.device)
    _call("argus_attention_bwd", q.device, ctypes.byref(p), _ptr(do), qa, ka, va, _ptr(o), _ptr(lse), _ptr(out["dq"]),
          _ptr(out["dk"]), _ptr(out["dv"]), _ptr(ws), ws.numel())
    return out
