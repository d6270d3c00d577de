"""The measured calls of the training-step operators: embedding, layer norm, attention and the router's balance loss,
each forward and backward.

A rank check runs one training step's operators on a rank that the cross-rank analysis flagged, with known outputs, and
puts their durations through the same summaries; the router's per-expert counts tell a rank that had more tokens from a
machine that is slow. Shapes are those of the training jobs that are traced: sequences of 4,096 tokens and a router of
128 experts of which a token takes 8 (the paper's measured workload), with generic widths, vocabularies and heads;
packed documents of uneven length, odd widths and strided views beside them. Inputs are made on the GPU from the seed
alone.

The plain forms are elementary torch operations in 32 bits, rounded once at the end.
"""
import itertools
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # token lookup of a micro-batch of sixteen sequences, widths of a large model
        {"name": "embedding_large", "path": "embedding", "tokens": 65_536, "vocab": 128_000, "dim": 4096, "dtype": "bf16",
         "ids64": True, "absent": 0.0},
        # the gradient of a few short documents over a small vocabulary: launches and latency
        {"name": "embedding_bwd_small", "path": "embedding_bwd", "tokens": 130, "vocab": 8_000, "dim": 512, "dtype": "f32",
         "ids64": False, "absent": 0.1},
        # the gradient of a micro-batch, Zipf-distributed tokens, some of them padding
        {"name": "embedding_bwd_large", "path": "embedding_bwd", "tokens": 32_768, "vocab": 128_000, "dim": 4096,
         "dtype": "bf16", "ids64": True, "absent": 0.05},
        # the norm of a micro-batch of eight sequences
        {"name": "layer_norm_large", "path": "layer_norm", "rows": 32_768, "cols": 4096, "dtype": "bf16", "wdtype": "f32",
         "bias": True, "pad": 0},
        # the norm's gradient over a short batch of a narrow model
        {"name": "layer_norm_bwd_small", "path": "layer_norm_bwd", "rows": 64, "cols": 768, "dtype": "f32", "wdtype": "f32",
         "bias": True, "pad": 0},
        # the norm's gradient at an odd number of packed rows and a width that is no power of two
        {"name": "layer_norm_bwd_odd", "path": "layer_norm_bwd", "rows": 20_011, "cols": 5_000, "dtype": "bf16",
         "wdtype": "bf16", "bias": True, "pad": 0},
        # the router over one sequence: 128 experts, top 8
        {"name": "balance_sequence", "path": "balance", "tokens": 4_096, "experts": 128, "top_k": 8, "dtype": "bf16",
         "masked": 0.0},
        # the router over a global batch of a wider expert layer, padding tokens masked
        {"name": "balance_large", "path": "balance", "tokens": 131_072, "experts": 256, "top_k": 8, "dtype": "f32",
         "masked": 0.1},
        # the router's gradient over a global batch of the 128-expert layer
        {"name": "balance_bwd_large", "path": "balance_bwd", "tokens": 262_144, "experts": 128, "top_k": 8, "dtype": "bf16",
         "masked": 0.05},
        # attention of a micro-batch: four sequences of 4,096, causal, four query heads to a key head, one fused projection
        {"name": "attention_batch", "path": "attention", "docs": 4, "tokens": 16_384, "lens_seed": 0, "q_part": 1.0,
         "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "fused": True},
        # the gradient over packed documents of uneven length, narrow heads, none shared
        {"name": "attention_bwd_packed", "path": "attention_bwd", "docs": 13, "tokens": 10_007, "lens_seed": 3, "q_part": 1.0,
         "heads": 16, "kv_heads": 16, "dim": 64, "causal": True, "fused": False},
        # the gradient over two long sequences
        {"name": "attention_bwd_long", "path": "attention_bwd", "docs": 2, "tokens": 16_384, "lens_seed": 0, "q_part": 1.0,
         "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "fused": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    path = rng.choice(["embedding", "embedding_bwd", "embedding_bwd", "layer_norm", "layer_norm_bwd", "layer_norm_bwd",
                       "balance", "balance_bwd", "attention", "attention_bwd", "attention_bwd"])
    if path.startswith("embedding"):
        dim = rng.choice([rng.randint(33, 300), 40 * rng.randint(4, 100), rng.choice([256, 768, 1024, 2048, 4096, 5120])])
        vocab = _log_int(rng, 200, min(128_000, 500_000_000 // dim))
        return {"path": path, "tokens": _log_int(rng, 1, min(65_536, 260_000_000 // dim)), "vocab": vocab, "dim": dim,
                "dtype": rng.choice(["bf16", "bf16", "f32", "f16"]), "ids64": rng.random() < 0.5,
                "absent": rng.choice([0.0, 0.05])}
    if path.startswith("layer_norm"):
        cols = rng.choice([rng.randint(33, 2_000), 40 * rng.randint(7, 200), rng.choice([512, 1024, 2048, 4096, 7168, 12_288])])
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        return {"path": path, "rows": _log_int(rng, 1, min(65_536, 130_000_000 // cols)), "cols": cols, "dtype": dtype,
                "wdtype": rng.choice(["f32", dtype]), "bias": rng.random() < 0.7, "pad": rng.choice([0, 0, 64, 3])}
    if path.startswith("balance"):
        experts = rng.choice([8, 16, 60, 64, 128, 128, 160, 256, 384])
        return {"path": path, "tokens": _log_int(rng, 1, 33_000_000 // max(experts, 64)), "experts": experts,
                "top_k": rng.choice([1, 2, 4, 6, 8]), "dtype": rng.choice(["bf16", "f32", "f16"]),
                "masked": rng.choice([0.0, 0.1])}
    dim = rng.choice([64, 64, 128, 128, 96, 40])
    heads, kv_heads = rng.choice([(32, 8), (16, 16), (16, 2), (12, 4), (8, 1)])
    docs = _log_int(rng, 1, 24)
    tokens = _log_int(rng, docs, min(16_384, 8_192 * docs))
    part = rng.choice([1.0, 1.0, 0.25])
    uneven = 64 * docs <= tokens <= 2_048 * docs and rng.random() < 0.6  # the longest document stays within the longest listed ones
    return {"path": path, "docs": docs, "tokens": tokens, "lens_seed": rng.randint(1, 1000) if uneven else 0, "q_part": part,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "causal": rng.random() < 0.7,
            "fused": part == 1.0 and rng.random() < 0.5}


def _lens(case):
    """Lengths of the packed documents: even ones, or uneven ones from the case's own number."""
    n, total = case["docs"], case["tokens"]
    if not case["lens_seed"]:
        k_lens = [total // n + (i < total % n) for i in range(n)]
    else:
        rng = random.Random(case["lens_seed"])
        cuts = [rng.expovariate(1.0) + 0.05 for _ in range(n)]
        k_lens = [max(1, int(total * c / sum(cuts))) for c in cuts]
        k_lens[k_lens.index(max(k_lens))] += total - sum(k_lens)
    q_lens = [max(1, math.ceil(k * case["q_part"])) for k in k_lens]
    return q_lens, k_lens


def _pairs(case):
    """Visible (query, key) pairs of one head."""
    return sum(q * k - q * (q - 1) // 2 if case["causal"] else q * k for q, k in zip(*_lens(case)))


def work(case):
    p, s = case["path"], BYTES.get(case.get("dtype"), 2)
    if p.startswith("embedding"):
        T, V, D = case["tokens"], case["vocab"], case["dim"]
        ids = T * (8 if case["ids64"] else 4)
        if p == "embedding":  # each row of the table that occurs is read once
            prob = np.arange(1, V + 1) ** -1.1
            rows = (1 - (1 - prob / prob.sum()) ** (T * (1 - case["absent"]))).sum()
            return {"bytes": ids + (T + rows) * D * s, "flops": T * D}
        return {"bytes": ids + T * D * s + V * D * s, "flops": 2 * T * D}
    if p.startswith("layer_norm"):
        R, D, w = case["rows"], case["cols"], BYTES[case["wdtype"]]
        if p == "layer_norm":
            return {"bytes": 2 * R * D * s + 8 * R + (2 if case["bias"] else 1) * D * w, "flops": 8 * R * D}
        return {"bytes": 3 * R * D * s + 8 * R + (3 if case["bias"] else 2) * D * w, "flops": 14 * R * D}
    if p.startswith("balance"):
        T, E, K = case["tokens"], case["experts"], case["top_k"]
        if p == "balance":
            return {"bytes": T * E * s + T + 8 * T * K + 4 * T + 8 * E, "flops": 5 * T * E}
        return {"bytes": 2 * T * E * s + 8 * T * K + 4 * T + 4 * E, "flops": 6 * T * E}
    q_lens, k_lens = _lens(case)
    D, qd, kd = case["dim"], sum(q_lens) * case["heads"], sum(k_lens) * case["kv_heads"]
    if p == "attention":
        return {"bytes": 2 * D * (2 * qd + 2 * kd) + 4 * qd, "flops": 4 * D * case["heads"] * _pairs(case)}
    return {"bytes": 2 * D * (4 * qd + 4 * kd) + 4 * qd, "flops": 10 * D * case["heads"] * _pairs(case)}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 16 + 5)


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _token_ids(case, g):
    """Zipf-distributed tokens (exponent 1.1) over a shuffled vocabulary; padding positions hold -1."""
    T, V = case["tokens"], case["vocab"]
    cdf = torch.cumsum(torch.arange(1, V + 1, device=DEV, dtype=torch.float64) ** -1.1, 0)
    u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64) * cdf[-1]
    ids = torch.randperm(V, generator=g, device=DEV)[torch.searchsorted(cdf, u).clamp(max=V - 1)]
    ids = torch.where(torch.rand(T, generator=g, device=DEV) < case["absent"], -1, ids)
    return ids if case["ids64"] else ids.to(torch.int32)


def _padded(g, rows, cols, pad, dtype, std=1.0):
    """Rows of a wider tensor where pad > 0, as a slice of a fused buffer has them."""
    return _normal(g, (rows, cols + pad), std, dtype)[:, :cols]


def _offsets(lens):
    return torch.tensor([0, *itertools.accumulate(lens)], dtype=torch.int64, device=DEV)


def prepare(case, seed):
    g, p = _gen(seed), case["path"]
    st = dict(case)
    dt = DTYPES.get(case.get("dtype"), torch.bfloat16)
    if p.startswith("embedding"):
        st["ids"] = _token_ids(case, g)
        if p == "embedding":
            st["table"] = _normal(g, (case["vocab"], case["dim"]), 0.02, dt)
            st["scale"] = math.sqrt(case["dim"])
        else:
            st["dout"] = _normal(g, (case["tokens"], case["dim"]), 0.01, dt)
            st["scale"] = math.sqrt(case["dim"])
    elif p.startswith("layer_norm"):
        R, D, wd = case["rows"], case["cols"], DTYPES[case["wdtype"]]
        x = _padded(g, R, D, case["pad"], dt, 2.0)
        x += (0.5 * torch.randn((1, D), generator=g, device=DEV)).to(dt)  # channels of their own level
        st["x"] = x
        st["weight"] = (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(wd)
        st["bias_t"] = _normal(g, (D,), 0.1, wd) if case["bias"] else None
        if p == "layer_norm_bwd":
            st["dy"] = _padded(g, R, D, case["pad"], dt, 0.05)
            xf = x.float()
            st["mean"] = xf.mean(1)
            st["rstd"] = (xf - st["mean"][:, None]).square().mean(1).add(1e-5).rsqrt()
    elif p.startswith("balance"):
        T, E, K = case["tokens"], case["experts"], case["top_k"]
        lean = torch.randn((1, E), generator=g, device=DEV)  # some experts are chosen more than others
        st["logits"] = (_normal(g, (T, E), 1.5) + lean).to(dt)
        st["mask"] = (torch.rand(T, generator=g, device=DEV) >= case["masked"]).to(torch.uint8) if case["masked"] else None
        if p == "balance_bwd":
            st.update(_balance(st))
            st["dloss"] = _normal(g, (1,), 0.2) + 1.0
            st["dgate"] = _normal(g, (T, K), 1e-3)
    else:
        q_lens, k_lens = _lens(case)
        H, N, D = case["heads"], case["kv_heads"], case["dim"]
        Tq, Tk = sum(q_lens), sum(k_lens)
        bf = torch.bfloat16
        if case["fused"]:  # q, k and v are slices of the projection's one output
            qkv = _normal(g, (Tq, H + 2 * N, D), 1.0, bf)
            st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + N], qkv[:, H + N:]
        else:
            st["q"], st["k"], st["v"] = (_normal(g, (t, h, D), 1.0, bf) for t, h in ((Tq, H), (Tk, N), (Tk, N)))
        st["q_off"], st["k_off"] = _offsets(q_lens), _offsets(k_lens)
        st["max_q"], st["max_k"], st["scale"] = max(q_lens), max(k_lens), 1.25 / math.sqrt(D)
        if p == "attention_bwd":
            st["do"] = _normal(g, (Tq, H, D), 0.1, bf)
            f = _attention(st)
            st["o"], st["lse"] = f["o"], f["lse"]
            del f
    return st


# ------------------------------------------------------------------ plain forms
def _embedding(st):
    ids = st["ids"].long()
    ok = (ids >= 0) & (ids < st["vocab"])
    rows = st["table"][torch.where(ok, ids, 0)].float() * st["scale"]
    return {"out": torch.where(ok[:, None], rows, 0.0).to(st["table"].dtype)}


def _embedding_bwd(st):
    ids, V = st["ids"].long(), st["vocab"]
    ids = torch.where((ids >= 0) & (ids < V), ids, V)
    acc = torch.zeros((V + 1, st["dim"]), device=DEV)
    acc.index_add_(0, ids, st["dout"].float())
    return {"dtable": (acc[:V] * st["scale"]).to(st["dout"].dtype)}


def _layer_norm(st):
    x = st["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = d.square().mean(1).add(1e-5).rsqrt()
    y = d * rstd[:, None] * st["weight"].float()
    if st["bias_t"] is not None:
        y = y + st["bias_t"].float()
    return {"y": y.to(st["x"].dtype), "mean": mean, "rstd": rstd}


def _layer_norm_bwd(st):
    xh = (st["x"].float() - st["mean"][:, None]) * st["rstd"][:, None]
    dy = st["dy"].float()
    gr = dy * st["weight"].float()
    dx = st["rstd"][:, None] * (gr - gr.mean(1, keepdim=True) - xh * (gr * xh).mean(1, keepdim=True))
    out = {"dx": dx.to(st["x"].dtype), "dweight": (dy * xh).sum(0).to(st["weight"].dtype)}
    if st["bias_t"] is not None:
        out["dbias"] = dy.sum(0).to(st["weight"].dtype)
    return out


def _balance(st):
    T, E, K = st["tokens"], st["experts"], st["top_k"]
    x = st["logits"].float()
    on = torch.ones(T, dtype=torch.bool, device=DEV) if st["mask"] is None else st["mask"] != 0
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(1, keepdim=True)
    prob = e / z
    at = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :K]  # stable: ties go to the lowest index
    count = torch.zeros(E + 1, dtype=torch.int64, device=DEV).index_add_(
        0, torch.where(on[:, None], at, E).reshape(-1), torch.ones(T * K, dtype=torch.int64, device=DEV))[:E]
    n = on.sum()
    psum = torch.where(on[:, None], prob, 0.0).sum(0)
    nf = n.clamp(min=1).float()
    loss = 0.01 * E * (count.float() / (K * nf) * (psum / nf)).sum()
    return {"expert": torch.where(on[:, None], at, -1).to(torch.int32), "gate": torch.where(on[:, None], prob.gather(1, at), 0.0),
            "lse": torch.where(on, (m + torch.log(z))[:, 0], -math.inf), "count": count.to(torch.int32),
            "prob": psum / nf, "n_valid": n.to(torch.int32).reshape(1), "loss": loss.reshape(1)}


def _balance_bwd(st):
    E, K = st["experts"], st["top_k"]
    on = (st["lse"] > -math.inf)[:, None]
    prob = torch.where(on, torch.exp(st["logits"].float() - st["lse"][:, None]), 0.0)
    n = st["n_valid"].clamp(min=1).float()
    gr = (st["dloss"] * 0.01 * E * st["count"].float() / (K * n * n)).expand_as(prob)
    gr = gr.scatter_add(1, st["expert"].clamp(min=0).long(), torch.where(st["expert"] >= 0, st["dgate"], 0.0))
    return {"dlogits": (prob * (gr - (gr * prob).sum(1, keepdim=True))).to(st["logits"].dtype)}


def _rows(off, longest):
    """Positions of each document's tokens in the packed tensors, [docs, longest], and which of them exist."""
    lens, at = off[1:] - off[:-1], torch.arange(longest, device=DEV)
    there = at[None] < lens[:, None]
    return torch.where(there, off[:-1, None] + at[None], 0), there


def _split(x, at, groups):
    """[docs, kv heads, query heads of each, longest, dim] in 32 bits."""
    d = x[at].float().permute(0, 2, 1, 3)
    return d.reshape(d.shape[0], groups, d.shape[1] // groups, d.shape[2], d.shape[3])


def _packed(x, off, total):
    """The padded [docs, heads.., longest, dim] tensor's tokens, in their packed order."""
    t = torch.arange(total, device=DEV)
    doc = torch.searchsorted(off[1:].contiguous(), t, right=True)
    x = x.reshape(x.shape[0], -1, x.shape[-2], x.shape[-1])
    return x[doc, :, t - off[doc]]


def _scores(st):
    N, G = st["kv_heads"], st["heads"] // st["kv_heads"]
    qa, qt = _rows(st["q_off"], st["max_q"])
    ka, kt = _rows(st["k_off"], st["max_k"])
    q, k, v = _split(st["q"], qa, N), _split(st["k"], ka, N), _split(st["v"], ka, N)
    see = qt[:, :, None] & kt[:, None, :]
    if st["causal"]:  # the last query sees the last key
        shift = (st["k_off"].diff() - st["q_off"].diff())[:, None, None]
        see = see & (torch.arange(st["max_k"], device=DEV)[None, None] <= torch.arange(st["max_q"], device=DEV)[None, :, None] + shift)
    see = see[:, None, None]
    s = torch.matmul(q, k.transpose(-1, -2).expand(-1, -1, G, -1, -1)).mul_(st["scale"]).masked_fill_(~see, -math.inf)
    return q, k.expand(-1, -1, G, -1, -1), v.expand(-1, -1, G, -1, -1), s, qa


def _attention(st):
    q, k, v, s, _ = _scores(st)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    e = s.sub_(m).exp_()
    z = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(z > 0, z, 1.0)
    lse = m + torch.log(z)
    return {"o": _packed(o, st["q_off"], len(st["q"])).to(st["q"].dtype), "lse": _packed(lse, st["q_off"], len(st["q"]))[..., 0]}


def _attention_bwd(st):
    q, k, v, s, qa = _scores(st)
    N, T = st["kv_heads"], len(st["k"])
    lse = _split(st["lse"][..., None], qa, N)
    do, o = _split(st["do"], qa, N), _split(st["o"], qa, N)
    p = s.sub_(torch.where(lse > -math.inf, lse, 0.0)).exp_()
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    del p
    dq = torch.matmul(ds, k).mul_(st["scale"])
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2).mul_(st["scale"])
    dt = st["q"].dtype
    return {"dq": _packed(dq, st["q_off"], len(st["q"])).to(dt), "dk": _packed(dk, st["k_off"], T).to(dt),
            "dv": _packed(dv, st["k_off"], T).to(dt)}


PLAIN = {"embedding": _embedding, "embedding_bwd": _embedding_bwd, "layer_norm": _layer_norm, "layer_norm_bwd": _layer_norm_bwd,
         "balance": _balance, "balance_bwd": _balance_bwd, "attention": _attention, "attention_bwd": _attention_bwd}


# ------------------------------------------------------------------ the framework's calls
def _own(st):
    import paper_2606_20374_amd as pa

    p = st["path"]
    if p == "embedding":
        return _keep(pa.embedding(st["ids"], st["table"], scale=st["scale"]), "out")
    if p == "embedding_bwd":
        return _keep(pa.embedding_bwd(st["ids"], st["dout"], st["vocab"], scale=st["scale"]), "dtable")
    if p == "layer_norm":
        return _keep(pa.layer_norm(st["x"], st["weight"], st["bias_t"], eps=1e-5), "y", "mean", "rstd")
    if p == "layer_norm_bwd":
        got = pa.layer_norm_bwd(st["dy"], st["x"], st["mean"], st["rstd"], st["weight"], bias=st["bias_t"] is not None)
        return _keep(got, "dx", "dweight", *(["dbias"] if st["bias_t"] is not None else []))
    if p == "balance":
        return _keep(pa.balance(st["logits"], st["top_k"], mask=st["mask"], alpha=0.01),
                     "expert", "gate", "lse", "count", "prob", "n_valid", "loss")
    if p == "balance_bwd":
        return _keep(pa.balance_bwd(st["logits"], st["lse"], st["expert"], st["count"], st["n_valid"], st["dloss"],
                                    dgate=st["dgate"], alpha=0.01), "dlogits")
    off = dict(q_off=st["q_off"], k_off=st["k_off"], causal=st["causal"], scale=st["scale"])
    if p == "attention":
        return _keep(pa.attention(st["q"], st["k"], st["v"], **off), "o", "lse")
    return _keep(pa.attention_bwd(st["do"], st["q"], st["k"], st["v"], st["o"], st["lse"], **off), "dq", "dk", "dv")


def _keep(got, *names):
    return {n: got[n] for n in names}


def run(state):
    return _own(state) if own else PLAIN[state["path"]](state)


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    f64, p = torch.float64, case["path"]
    if p == "embedding":
        out = torch.zeros((case["tokens"], case["dim"]), dtype=f64, device=DEV)
        here = torch.nonzero((st["ids"] >= 0) & (st["ids"] < case["vocab"]))[:, 0]
        out[here] = st["table"][st["ids"][here].long()].to(f64).mul_(st["scale"])
        return {"out": out}
    if p == "embedding_bwd":
        out = torch.zeros((case["vocab"], case["dim"]), dtype=f64, device=DEV)
        here = torch.nonzero((st["ids"] >= 0) & (st["ids"] < case["vocab"]))[:, 0]
        out.index_put_((st["ids"][here].long(),), st["dout"][here].to(f64).mul_(st["scale"]), accumulate=True)
        return {"dtable": out}
    if p.startswith("layer_norm"):
        x, w, D = st["x"].to(f64), st["weight"].to(f64), case["cols"]
        if p == "layer_norm":
            mu = x.sum(1) / D
            x -= mu[:, None]
            r = 1 / torch.sqrt((x * x).sum(1) / D + 1e-5)
            y = x.mul_(r[:, None]).mul_(w)
            return {"y": y if st["bias_t"] is None else y.add_(st["bias_t"].to(f64)), "mean": mu, "rstd": r}
        dy, r = st["dy"].to(f64), st["rstd"].to(f64)[:, None]
        xh = x.sub_(st["mean"].to(f64)[:, None]).mul_(r)
        out = {"dweight": (dy * xh).sum(0)}
        if st["bias_t"] is not None:
            out["dbias"] = dy.sum(0)
        h = dy.mul_(w)
        c1, c2 = h.sum(1, keepdim=True) / D, (h * xh).sum(1, keepdim=True) / D
        out["dx"] = h.sub_(c1).sub_(xh.mul_(c2)).mul_(r)
        return out
    if p.startswith("balance"):
        x, E, K = st["logits"].to(f64), case["experts"], case["top_k"]
        if p == "balance":
            take = torch.arange(case["tokens"], device=DEV) if st["mask"] is None else torch.nonzero(st["mask"])[:, 0]
            n = max(1, len(take))
            lse = torch.full((case["tokens"],), -math.inf, dtype=f64, device=DEV)
            lse[take] = torch.logsumexp(x[take], 1)
            prob = torch.softmax(x[take], 1)
            # the value, then the index: of equal logits the lower index is chosen
            best = torch.argsort(x[take], dim=1, descending=True, stable=True)[:, :K]
            gate = torch.zeros((case["tokens"], K), dtype=f64, device=DEV)
            gate[take] = torch.gather(prob, 1, best)
            count = torch.bincount(best.reshape(-1), minlength=E)
            mean = prob.sum(0) / n
            loss = 0.01 * E * ((count.to(f64) / (K * n)) * mean).sum()
            return {"expert": None, "gate": gate, "lse": lse, "count": count.to(torch.int32), "prob": mean, "n_valid": None,
                    "loss": loss.reshape(1)}
        n = max(1, int(st["n_valid"].item()))
        out = torch.zeros(x.shape, dtype=f64, device=DEV)
        for lo in range(0, len(x), 65_536):  # in pieces: the widest case has 33 million logits
            xs, ls, ex = x[lo:lo + 65_536], st["lse"][lo:lo + 65_536], st["expert"][lo:lo + 65_536].long()
            pr = torch.exp(xs - ls.to(f64)[:, None])
            up = (st["dloss"].to(f64) * 0.01 * E / (K * n * n) * st["count"].to(f64))[None].repeat(len(xs), 1)
            up += (torch.nn.functional.one_hot(ex.clamp(min=0), E) * torch.where(ex >= 0, st["dgate"][lo:lo + 65_536], 0).to(f64)[..., None]).sum(1)
            gr = pr * (up - (up * pr).sum(1, keepdim=True))
            out[lo:lo + 65_536] = torch.where((ls > -math.inf)[:, None], gr, 0.0)
        return {"dlogits": out}
    q_off, k_off, G = st["q_off"].tolist(), st["k_off"].tolist(), case["heads"] // case["kv_heads"]
    outs = {n: torch.zeros(st[a].shape, dtype=f64, device=DEV) for n, a in (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "k"))}
    lse = torch.full(st["q"].shape[:2], -math.inf, dtype=f64, device=DEV)
    for a, b, c, d in zip(q_off, q_off[1:], k_off, k_off[1:]):
        hidden = torch.ones((b - a, d - c), dtype=torch.bool, device=DEV).triu(1 + (d - c) - (b - a)) if case["causal"] else None
        for h in range(case["heads"]):
            q, k, v = st["q"][a:b, h].to(f64), st["k"][c:d, h // G].to(f64), st["v"][c:d, h // G].to(f64)
            s = (q @ k.T) * st["scale"]
            if hidden is not None:
                s.masked_fill_(hidden, -math.inf)
            if p == "attention":
                lse[a:b, h] = torch.logsumexp(s, 1)
                outs["o"][a:b, h] = torch.softmax(s, 1) @ v
                continue
            do = st["do"][a:b, h].to(f64)
            pr = torch.exp(s - st["lse"][a:b, h].to(f64)[:, None])
            outs["dv"][c:d, h // G] += pr.T @ do
            ds = pr * (do @ v.T - (do * st["o"][a:b, h].to(f64)).sum(1, keepdim=True))
            outs["dq"][a:b, h] = (ds @ k) * st["scale"]
            outs["dk"][c:d, h // G] += (ds.T @ q) * st["scale"]
    if p == "attention":
        return {"o": outs["o"], "lse": lse}
    return {n: outs[n] for n in ("dq", "dk", "dv")}
