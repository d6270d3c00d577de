"""The measured calls of the rest of a training step: rotary positions, the gated feed-forward block and the cross entropy
over a large vocabulary, each forward and backward.

Together with the embedding, the norms, attention and the router they make the whole step that a rank check runs on a
rank which the cross-rank analysis flagged. Shapes are generic widths and vocabularies around the traced workload's
sequences of 4,096 tokens; a few tokens, odd counts, widths that fill no tile, and slices of wider buffers beside them.
Inputs are made on the GPU from the seed alone.

The plain forms are elementary torch operations in 32 bits (angles in 64), rounded once at the end.
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # positions of a few short sequences: one launch's latency
        {"name": "rotary_small", "path": "rotary", "tokens": 130, "heads": 16, "dim": 64, "rot": 64, "interleaved": False,
         "dtype": "f32", "ids64": False, "start": 0, "factor": 1.0, "wider": 0, "inverse": False},
        # a third of each head, neighbouring pairs, far positions of a context that was made longer
        {"name": "rotary_part_far", "path": "rotary", "tokens": 20_011, "heads": 24, "dim": 96, "rot": 32, "interleaved": True,
         "dtype": "f16", "ids64": True, "start": 900_000, "factor": 32.0, "wider": 0, "inverse": False},
        # queries and keys inside the projection's one output, a micro-batch of sixteen sequences, the gradient's direction
        {"name": "rotary_large", "path": "rotary", "tokens": 65_536, "heads": 40, "dim": 128, "rot": 128, "interleaved": False,
         "dtype": "bf16", "ids64": True, "start": 0, "factor": 1.0, "wider": 8, "inverse": True},
        # four tokens of a generating model: the weights' bytes
        {"name": "ff_tokens", "path": "ff", "tokens": 4, "width": 4096, "ff": 12_288, "dtype": "bf16", "act": "silu",
         "save": False, "pad": 0},
        # a short prompt in float16
        {"name": "ff_prompt", "path": "ff", "tokens": 300, "width": 2048, "ff": 8192, "dtype": "f16", "act": "gelu",
         "save": False, "pad": 64},
        # a micro-batch of four sequences
        {"name": "ff_large", "path": "ff", "tokens": 16_384, "width": 4096, "ff": 12_288, "dtype": "bf16", "act": "silu",
         "save": True, "pad": 0},
        # the gradient of an odd count of tokens through widths that fill no tile
        {"name": "ff_bwd_odd", "path": "ff_bwd", "tokens": 999, "width": 1000, "ff": 2720, "dtype": "f16", "act": "gelu",
         "save": True, "pad": 8},
        # the gradient of a micro-batch of four sequences
        {"name": "ff_bwd_large", "path": "ff_bwd", "tokens": 16_384, "width": 4096, "ff": 12_288, "dtype": "bf16", "act": "silu",
         "save": True, "pad": 0},
        # the loss of a few short documents over a small vocabulary: launches and latency
        {"name": "ce_small", "path": "ce", "tokens": 130, "vocab": 8_000, "width": 512, "ids64": False, "absent": 0.1,
         "z_loss": 0.0, "pad": 0},
        # the loss of a micro-batch of four sequences
        {"name": "ce_large", "path": "ce", "tokens": 16_384, "vocab": 128_000, "width": 4096, "ids64": True, "absent": 0.0,
         "z_loss": 1e-4, "pad": 0},
        # the gradient of an odd count of tokens, half of them a prompt that is not learned, over an odd vocabulary
        {"name": "ce_bwd_odd", "path": "ce_bwd", "tokens": 1_501, "vocab": 50_257, "width": 1000, "ids64": True, "absent": 0.5,
         "z_loss": 1e-4, "pad": 8},
        # the gradient of a micro-batch of two sequences
        {"name": "ce_bwd_large", "path": "ce_bwd", "tokens": 8_192, "vocab": 128_000, "width": 4096, "ids64": True,
         "absent": 0.05, "z_loss": 0.0, "pad": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    path = rng.choice(["rotary", "ff", "ff", "ff_bwd", "ff_bwd", "ce", "ce", "ce_bwd", "ce_bwd"])
    if path == "rotary":
        dim = rng.choice([64, 128, 128, 96, 40, 256, 2 * rng.randint(9, 60)])
        heads = rng.choice([1, 6, 16, 20, 40, 40])
        rot = rng.choice([dim, dim, 2 * rng.randint(1, dim // 2)])
        return {"path": path, "tokens": _log_int(rng, 1, min(131_072, 330_000_000 // (dim * heads))), "heads": heads,
                "dim": dim, "rot": rot, "interleaved": rng.random() < 0.5, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "ids64": rng.random() < 0.5, "start": rng.choice([0, 0, 100_000, 1_000_000]),
                "factor": rng.choice([1.0, 1.0, 4.0, 32.0]), "wider": rng.choice([0, 0, 2, 8]), "inverse": rng.random() < 0.5}
    width = rng.choice([8 * rng.randint(4, 250), rng.choice([512, 1024, 2048, 4096, 5120])])
    if path.startswith("ff"):
        ff = rng.choice([8 * rng.randint(8, 700), rng.choice([2048, 5120, 8192, 12_288])])
        most = 800_000_000_000 // (width * ff)
        return {"path": path, "tokens": _log_int(rng, 1, min(32_768, most)), "width": width, "ff": ff,
                "dtype": rng.choice(["bf16", "bf16", "f16"]), "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh"]),
                "save": path == "ff_bwd" or rng.random() < 0.5, "pad": rng.choice([0, 0, 8, 64])}
    vocab = _log_int(rng, 300, 128_000)
    most = (8_000_000_000_000 if path == "ce" else 4_000_000_000_000) // (width * vocab)
    return {"path": path, "tokens": _log_int(rng, 1, min(16_384, most)), "vocab": vocab, "width": width,
            "ids64": rng.random() < 0.5, "absent": rng.choice([0.0, 0.1, 0.6]), "z_loss": rng.choice([0.0, 1e-4]),
            "pad": rng.choice([0, 0, 8, 64])}


def work(case):
    p, T = case["path"], case["tokens"]
    if p == "rotary":
        s, n = BYTES[case["dtype"]], T * case["heads"]
        return {"bytes": 2 * n * case["dim"] * s + T * (8 if case["ids64"] else 4) + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    W = case["width"]
    if p.startswith("ff"):
        F = case["ff"]
        if p == "ff":
            return {"bytes": 2 * (T * W + 2 * F * W + T * F * (3 if case["save"] else 1)), "flops": 4 * T * F * W}
        return {"bytes": 2 * (2 * T * W + 4 * F * W + 3 * T * F), "flops": 8 * T * F * W}
    # tokens that are not learned need not be read nor multiplied
    V, ids, n = case["vocab"], T * (8 if case["ids64"] else 4), max(1, round(T * (1 - case["absent"])))
    if p == "ce":
        return {"bytes": 2 * (n * W + V * W) + ids + 8 * T, "flops": 2 * n * V * W}
    return {"bytes": 2 * (n * W + T * W + 2 * V * W) + ids + 4 * T, "flops": 6 * n * V * W}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 16 + 7)


def _normal(g, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _padded(g, rows, cols, pad, dtype, std=1.0):
    """Rows of a wider tensor where pad > 0, as a slice of a fused buffer has them."""
    return _normal(g, (rows, cols + pad), std, dtype)[:, :cols]


def _frequencies(rot, factor, base=10_000.0, context=4096):
    """Radians a position for each pair, in 64 bits. With factor > 1 the pairs that turn less than once over the
    original context are slowed by it, those that turn more than 32 times are not, the others in proportion."""
    f = base ** -(torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    keep = ((context * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return f * (keep + (1 - keep) / factor)


def prepare(case, seed):
    g, p, T = _gen(seed), case["path"], case["tokens"]
    st = dict(case)
    dt = DTYPES[case.get("dtype", "bf16")]
    if p == "rotary":
        wide = _normal(g, (T, case["heads"] + case["wider"], case["dim"]), 1.0, dt)
        st["x"] = wide[:, :case["heads"]]
        starts = torch.rand(T, generator=g, device=DEV) < 1 / 1500  # packed documents begin here
        at = torch.arange(T, device=DEV)
        pos = at - torch.where(starts, at, 0).cummax(0)[0] + case["start"]
        st["pos"] = pos if case["ids64"] else pos.to(torch.int32)
        st["freq"] = _frequencies(case["rot"], case["factor"])
        st["scale"] = 1.0 + 0.1 * math.log(case["factor"])
        return st
    W = case["width"]
    if p.startswith("ff"):
        F = case["ff"]
        st["x"] = _padded(g, T, W, case["pad"], dt)
        st["wg"], st["wu"] = (_padded(g, F, W, case["pad"], dt, W**-0.5) for _ in range(2))
        if p == "ff_bwd":
            st["dh"] = _padded(g, T, F, case["pad"], dt, 0.1)
            f = _ff(st)
            st["g"], st["u"] = f["g"], f["u"]
        return st
    V = case["vocab"]
    st["w"] = _padded(g, V, W, case["pad"], dt, W**-0.5)
    labels = torch.randint(0, V, (T,), generator=g, device=DEV)
    # a model that has learned: the label's logit is raised, by another amount for each token
    sure = 14.0 * torch.rand((T, 1), generator=g, device=DEV)
    x = torch.randn((T, W + case["pad"]), generator=g, device=DEV)
    x[:, :W] += sure * st["w"][labels].float()
    st["x"] = x.to(dt)[:, :W]
    absent = torch.rand(T, generator=g, device=DEV) < case["absent"]
    labels = torch.where(absent, -100, labels)
    st["labels"] = labels if case["ids64"] else labels.to(torch.int32)
    if p == "ce_bwd":
        f = _ce(st)
        st["lse"], st["n_valid"] = f["lse"], f["n_valid"]
        st["dmean"] = 1.0 + _normal(g, (1,), 0.2)
    return st


# ------------------------------------------------------------------ plain forms
def _rotary(st):
    x, R = st["x"].float(), st["rot"]
    angle = st["pos"].double()[:, None] * st["freq"]
    c, s = ((t * st["scale"]).float()[:, None] for t in (torch.cos(angle), torch.sin(angle)))
    if st["inverse"]:
        s = -s
    if st["interleaved"]:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat((a * c - b * s, a * s + b * c), -1)
    return {"out": torch.cat((turned, x[..., R:]), -1).to(st["x"].dtype)}


def _activation(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _ff(st):
    x, dt = st["x"].float(), st["x"].dtype
    g, u = x @ st["wg"].float().t(), x @ st["wu"].float().t()
    out = {"h": (_activation(g, st["act"])[0] * u).to(dt)}
    return {**out, "g": g.to(dt), "u": u.to(dt)} if st["save"] else out


def _ff_bwd(st):
    x, wg, wu, dh, g, u = (st[n].float() for n in ("x", "wg", "wu", "dh", "g", "u"))
    a, da = _activation(g, st["act"])
    dg, du = dh * u * da, dh * a
    dt = st["x"].dtype
    return {"dx": (dg @ wg + du @ wu).to(dt), "dwg": (dg.t() @ x).to(dt), "dwu": (du.t() @ x).to(dt)}


def _valid(st):
    return (st["labels"] >= 0) & (st["labels"] < st["vocab"])


def _ce(st):
    on = _valid(st)
    z = st["x"].float() @ st["w"].float().t()
    m = z.amax(1)
    own_z = z.gather(1, torch.where(on, st["labels"], 0).long()[:, None])[:, 0]
    lse = m + torch.log(z.sub_(m[:, None]).exp_().sum(1))
    loss = torch.where(on, lse - own_z + st["z_loss"] * lse * lse, 0.0)
    n = on.sum()
    return {"loss": loss, "lse": torch.where(on, lse, -math.inf), "mean": (loss.double().sum() / n.clamp(min=1)).float().reshape(1),
            "n_valid": n.to(torch.int32).reshape(1)}


def _ce_bwd(st):
    on = _valid(st)
    x, w = st["x"].float(), st["w"].float()
    lse = torch.where(on, st["lse"], 0.0)[:, None]
    dz = (x @ w.t()).sub_(lse).exp_().mul_(1 + 2 * st["z_loss"] * lse)
    at = torch.arange(len(x), device=DEV)
    dz[at, torch.where(on, st["labels"], 0).long()] -= 1.0
    dz.mul_(torch.where(on, st["dmean"] / st["n_valid"].clamp(min=1), 0.0)[:, None])
    dt = st["x"].dtype
    return {"dx": (dz @ w).to(dt), "dw": (dz.t() @ x).to(dt)}


PLAIN = {"rotary": _rotary, "ff": _ff, "ff_bwd": _ff_bwd, "ce": _ce, "ce_bwd": _ce_bwd}


# ------------------------------------------------------------------ the framework's calls
def _own(st):
    import paper_2606_20374_amd as pa

    p = st["path"]
    if p == "rotary":
        turn = pa.rotary_bwd if st["inverse"] else pa.rotary
        got = turn(st["x"], st["freq"], pos=st["pos"], interleaved=st["interleaved"], scale=st["scale"])
        return {"out": got["dx" if st["inverse"] else "out"]}
    if p == "ff":
        return _keep(pa.gated_ff(st["x"], st["wg"], st["wu"], act=st["act"], save=st["save"]),
                     "h", *(["g", "u"] if st["save"] else []))
    if p == "ff_bwd":
        return _keep(pa.gated_ff_bwd(st["dh"], st["x"], st["wg"], st["wu"], st["g"], st["u"], act=st["act"]), "dx", "dwg", "dwu")
    if p == "ce":
        return _keep(pa.cross_entropy(st["x"], st["w"], st["labels"], z_loss=st["z_loss"]), "loss", "lse", "mean", "n_valid")
    return _keep(pa.cross_entropy_bwd(st["x"], st["w"], st["labels"], st["lse"], st["n_valid"], dmean=st["dmean"],
                                      z_loss=st["z_loss"]), "dx", "dw")


def _keep(got, *names):
    return {n: got[n] for n in names}


def run(state):
    return _own(state) if own else PLAIN[state["path"]](state)


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    f64, p = torch.float64, case["path"]
    if p == "rotary":
        R = case["rot"]
        turn = torch.polar(torch.full((), st["scale"], dtype=f64, device=DEV), st["pos"].to(f64).outer(st["freq"]))
        if case["inverse"]:
            turn = turn.conj()
        out = st["x"].to(f64)
        # pair i of a head: a complex number that is multiplied by scale e^(i angle)
        i = torch.arange(R // 2, device=DEV)
        re, im = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + R // 2)
        z = torch.complex(out[..., re], out[..., im]) * turn[:, None]
        out[..., re], out[..., im] = z.real, z.imag
        return {"out": out}
    if p.startswith("ff"):
        x, wg, wu = (st[n].to(f64) for n in ("x", "wg", "wu"))
        g, u = (x @ wg.T, x @ wu.T) if p == "ff" else (st["g"].to(f64), st["u"].to(f64))
        k = math.sqrt(2 / math.pi)
        if case["act"] == "silu":
            gate = torch.sigmoid(g)
            slope = gate * (1 + g * torch.sigmoid(-g))
        elif case["act"] == "gelu":
            gate = torch.special.ndtr(g)
            slope = gate + g * (-g * g / 2).exp() / math.sqrt(2 * math.pi)
        else:
            gate = torch.sigmoid(2 * k * (g + 0.044715 * g**3))  # (1 + tanh y) / 2 = sigmoid(2 y)
            slope = gate + 2 * k * g * gate * (1 - gate) * (1 + 0.134145 * g * g)
        if p == "ff":
            out = {"h": g * gate * u}
            return {**out, "g": g, "u": u} if case["save"] else out
        dh = st["dh"].to(f64)
        dg, du = slope * u * dh, g * gate * dh
        return {"dx": torch.addmm(dg @ wg, du, wu), "dwg": dg.T @ x, "dwu": du.T @ x}
    T, V = case["tokens"], case["vocab"]
    labels = st["labels"].long()
    take = torch.nonzero((labels >= 0) & (labels < V))[:, 0]
    w, n = st["w"].to(f64), max(1, len(take))
    loss = torch.zeros(T, dtype=f64, device=DEV)
    lse = torch.full((T,), -math.inf, dtype=f64, device=DEV)
    dx, dw = torch.zeros((T, case["width"]), dtype=f64, device=DEV), torch.zeros_like(w)
    for lo in range(0, len(take), 2_048):  # in pieces of the tokens
        t = take[lo:lo + 2_048]
        xs, ys = st["x"][t].to(f64), labels[t]
        z = xs @ w.T
        if p == "ce":
            lse[t] = torch.logsumexp(z, 1)
            loss[t] = torch.nn.functional.cross_entropy(z, ys, reduction="none") + case["z_loss"] * lse[t] ** 2
            continue
        given = st["lse"][t].to(f64)[:, None]
        d = torch.exp(z - given) * (1 + 2 * case["z_loss"] * given)
        d.scatter_add_(1, ys[:, None], torch.full((len(t), 1), -1.0, dtype=f64, device=DEV))
        d *= st["dmean"].to(f64) / n
        dx[t] = d @ w
        dw += d.T @ xs
    if p == "ce":
        return {"loss": loss, "lse": lse, "mean": (loss.sum() / n).reshape(1), "n_valid": None}
    return {"dx": dx, "dw": dw}
