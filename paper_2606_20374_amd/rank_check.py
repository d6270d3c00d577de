"""Check of one rank: a training step with known inputs, timed like a traced job.

argus_cross_rank and argus_l2 name ranks and (rank, kernel) pairs that are
slow. To tell a slow machine from one that had more work, every rank of
interest runs the same seeded step here: token embedding, layer norm,
attention over packed documents, the top-k router with its balance loss, and
their gradients, with the library's matrix products between them. The
operators' durations become one rank's kernel events, and the bits of the
step's outputs, the same on every sound machine, a digest beside them.
`compare` puts the events of several ranks through argus_summarize,
argus_cross_rank and argus_iter_windows, and names the ranks whose outputs
differ from the others'. `expert_load` says how uneven a router's tokens are
over expert-parallel ranks, from the counts that argus_balance gives: the
job's own, where its expert kernels are in question.

    python -m paper_2606_20374_amd.rank_check --save rank0.npz
    python -m paper_2606_20374_amd.rank_check --compare rank0.npz rank1.npz rank2.npz
"""
from __future__ import annotations

import argparse
import dataclasses
import hashlib
from typing import Optional, Sequence

import numpy as np
import torch

from . import argus, ops

# kernel ids of the events, in launch order
NAMES = ("embedding", "norm1", "qkv_product", "attention", "out_product", "norm2", "router_product", "balance",
         "balance_bwd", "router_product_bwd", "norm2_bwd", "out_product_bwd", "attention_bwd", "qkv_product_bwd",
         "norm1_bwd", "embedding_bwd")


# what a step returns
OUTPUTS = ("h", "expert", "gate", "count", "loss", "d_table", "d_norm1", "d_norm2", "d_qkv", "d_out", "d_router")


@dataclasses.dataclass(frozen=True)
class Config:
    """One layer of a mixture-of-experts model; the defaults are the traced
    workload's sequence length, experts and choices, with a generic width."""
    doc_lens: Sequence[int] = (4096, 2048, 1536, 512)
    vocab: int = 32_000
    width: int = 2048
    heads: int = 16
    kv_heads: int = 4
    head_dim: int = 128
    experts: int = 128
    top_k: int = 8
    alpha: float = 0.01
    seed: int = 0


class RankCheck:
    """The step's weights and inputs, from the seed alone."""

    def __init__(self, cfg: Config = Config(), device="cuda"):
        self.cfg, self.device = cfg, torch.device(device)
        g = torch.Generator().manual_seed(cfg.seed)  # on the host: the same on every machine
        H, N, D, W = cfg.heads, cfg.kv_heads, cfg.head_dim, cfg.width
        T = sum(cfg.doc_lens)

        def normal(*shape, std=1.0, dtype=torch.bfloat16):
            return (torch.randn(*shape, generator=g) * std).to(dtype).to(self.device)

        self.ids = torch.randint(0, cfg.vocab, (T,), generator=g).to(self.device)
        self.off = torch.tensor(np.cumsum([0, *cfg.doc_lens]), dtype=torch.int64, device=self.device)
        self.table = normal(cfg.vocab, W, std=W**-0.5)
        self.norm1, self.norm2 = ((1 + normal(W, std=0.1, dtype=torch.float32), normal(W, std=0.1, dtype=torch.float32))
                                  for _ in range(2))
        self.w_qkv, self.w_out = normal(W, (H + 2 * N) * D, std=W**-0.5), normal(H * D, W, std=(H * D)**-0.5)
        self.w_router = normal(W, cfg.experts, std=W**-0.5)
        self.d_gate = normal(T, cfg.top_k, std=1e-2, dtype=torch.float32)  # what the experts would send back
        self.d_out = normal(T, W, std=1e-2)
        self.d_loss = torch.ones(1, device=self.device)

    def step(self, mark=lambda name: None) -> dict:
        """Forward and backward once; `mark(name)` is called as each operator's
        work has been issued. Returns the outputs and all gradients."""
        c, T = self.cfg, len(self.ids)
        H, N, D = c.heads, c.kv_heads, c.head_dim
        scale = c.width**0.5
        x = ops.embedding(self.ids, self.table, scale=scale)["out"]
        mark("embedding")
        n1 = ops.layer_norm(x, *self.norm1)
        mark("norm1")
        qkv = (n1["y"] @ self.w_qkv).view(T, H + 2 * N, D)
        q, k, v = qkv[:, :H], qkv[:, H:H + N], qkv[:, H + N:]
        mark("qkv_product")
        at = ops.attention(q, k, v, q_off=self.off)
        mark("attention")
        o = at["o"].view(T, H * D)
        h = torch.addmm(x, o, self.w_out)
        mark("out_product")
        n2 = ops.layer_norm(h, *self.norm2)
        mark("norm2")
        logits = n2["y"] @ self.w_router
        mark("router_product")
        bal = ops.balance(logits, c.top_k, alpha=c.alpha)
        mark("balance")

        dlogits = ops.balance_bwd(logits, bal["lse"], bal["expert"], bal["count"], bal["n_valid"], self.d_loss,
                                  dgate=self.d_gate, alpha=c.alpha)["dlogits"]
        mark("balance_bwd")
        d_router = n2["y"].t() @ dlogits
        dy2 = torch.addmm(self.d_out, dlogits, self.w_router.t())
        mark("router_product_bwd")
        b2 = ops.layer_norm_bwd(dy2, h, n2["mean"], n2["rstd"], self.norm2[0])
        mark("norm2_bwd")
        d_out_w = o.t() @ b2["dx"]
        do = (b2["dx"] @ self.w_out.t()).view(T, H, D)
        mark("out_product_bwd")
        ab = ops.attention_bwd(do, q, k, v, at["o"], at["lse"], q_off=self.off)
        mark("attention_bwd")
        dqkv = torch.cat([ab["dq"], ab["dk"], ab["dv"]], 1).view(T, -1)
        d_qkv_w = n1["y"].t() @ dqkv
        dy1 = dqkv @ self.w_qkv.t()
        mark("qkv_product_bwd")
        b1 = ops.layer_norm_bwd(dy1, x, n1["mean"], n1["rstd"], self.norm1[0])
        dx = b1["dx"] + b2["dx"]
        mark("norm1_bwd")
        d_table = ops.embedding_bwd(self.ids, dx, c.vocab, scale=scale)["dtable"]
        mark("embedding_bwd")
        return {"h": h, "expert": bal["expert"], "gate": bal["gate"], "count": bal["count"], "loss": bal["loss"],
                "d_table": d_table, "d_norm1": (b1["dweight"], b1["dbias"]), "d_norm2": (b2["dweight"], b2["dbias"]),
                "d_qkv": d_qkv_w, "d_out": d_out_w, "d_router": d_router}

    def trace(self, steps: int = 6, window: int = 10, warmup: int = 3) -> dict:
        """One rank's kernel events over `steps` segments of `window` runs
        each: the arrays of argus_summarize with seg_off, on the host, and the
        digest of the last run's outputs."""
        for _ in range(warmup):
            self.step()
        last = {}
        stream = torch.cuda.current_stream(self.device)
        begin, marks = torch.cuda.Event(enable_timing=True), []

        def mark(name):
            e = torch.cuda.Event(enable_timing=True)
            e.record(stream)
            marks.append((name, e))

        torch.cuda.synchronize(self.device)
        begin.record(stream)
        for _ in range(steps * window):
            mark(None)  # the step's begin
            last = {}  # the run before's memory serves this one
            last = self.step(mark)
        torch.cuda.synchronize(self.device)
        # a difference of events is a 32-bit number of milliseconds: each is taken
        # from its neighbour, which keeps the nanoseconds however long the trace
        events = [begin, *(e for _, e in marks)]
        at = np.cumsum([round(a.elapsed_time(b) * 1e6) for a, b in zip(events, events[1:])], dtype=np.int64)
        kid = np.array([NAMES.index(name) for name, _ in marks if name], dtype=np.int32)
        start = np.array([at[i - 1] for i, (name, _) in enumerate(marks) if name], dtype=np.int64)
        end = np.array([at[i] for i, (name, _) in enumerate(marks) if name], dtype=np.int64)
        seg = np.arange(steps + 1, dtype=np.int64) * window * len(NAMES)
        return {"kernel_id": kid, "stream": np.zeros_like(kid), "start_ns": start, "end_ns": end, "seg_off": seg,
                "digest": digest(last)}


def digest(outputs: dict) -> np.ndarray:
    """64 bits of the SHA-256 of each output's bits, in the dict's order."""
    d = []
    for v in outputs.values():
        h = hashlib.sha256()
        for t in v if isinstance(v, tuple) else (v,):
            h.update(t.detach().contiguous().view(torch.uint8).cpu().numpy())
        d.append(int.from_bytes(h.digest()[:8], "little"))
    return np.array(d, dtype=np.uint64)


def outputs_differ(digests: Sequence[np.ndarray]) -> np.ndarray:
    """[ranks][outputs]: whether a rank's output is another than most ranks
    have; where no value has a majority, every rank's is taken to differ."""
    if any(len(d) != len(digests[0]) for d in digests):
        raise argus.ArgusError("rank_check: the traces have different numbers of outputs")
    a = np.stack(digests)
    same = (a[:, None] == a[None]).sum(1)  # ranks that agree with each, itself among them
    return 2 * same <= len(a)


def compare(traces: Sequence[dict], device="cuda", **params) -> dict:
    """The events of several ranks (as RankCheck.trace gives them, equally many
    segments each) through summarize, cross-rank and iteration windows. Keys:
    `summary`, `cross_rank`, `windows`, and per rank `score_pm` and `straggler`
    [ranks][steps], per (rank, operator) `degraded` (any step), and where all
    traces have their digests `outputs_differ` [ranks][OUTPUTS]."""
    R, S, K = len(traces), len(traces[0]["seg_off"]) - 1, len(NAMES)
    if any(len(t["seg_off"]) - 1 != S for t in traces):
        raise argus.ArgusError("rank_check: the traces have different numbers of segments")
    base = np.cumsum([0] + [len(t["kernel_id"]) for t in traces])
    seg = np.concatenate([t["seg_off"][:-1] + b for t, b in zip(traces, base)] + [base[-1:]])
    ev = {k: torch.from_numpy(np.concatenate([t[k] for t in traces])).to(device)
          for k in ("kernel_id", "stream", "start_ns", "end_ns")}
    ev["seg_off"] = torch.from_numpy(seg).to(device)
    s = argus.summarize(ev, R, S, K, 1)
    x = argus.cross_rank(s["count"], s["sum_ns"], R, S, K, **params)
    w = argus.iter_windows(s["step_ns"], R, S)
    flags = x["flags"].view(R, S, K)
    r = {"summary": s, "cross_rank": x, "windows": w, "score_pm": x["score_pm"].view(R, S).cpu(),
         "straggler": x["straggler"].view(R, S).cpu(), "degraded": (flags & 8).ne(0).any(1).cpu()}
    if all("digest" in t for t in traces):
        r["outputs_differ"] = outputs_differ([t["digest"] for t in traces])
    return r


def expert_load(count: torch.Tensor, expert_ranks: int) -> torch.Tensor:
    """Tokens of each expert-parallel rank, in permille of the even share: a
    rank's slow expert kernels at 1300 are no sign of a slow machine. Experts
    are spread over the ranks in equal, consecutive parts."""
    if expert_ranks < 1 or len(count) % expert_ranks:
        raise argus.ArgusError(f"rank_check: {len(count)} experts do not spread evenly over {expert_ranks} ranks")
    c = count.to(torch.int64).view(expert_ranks, -1).sum(1)
    return c * (1000 * expert_ranks) // c.sum().clamp(min=1)


def main(argv: Optional[Sequence[str]] = None) -> int:
    ap = argparse.ArgumentParser(prog="rank_check", description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=6, help="segments of the trace")
    ap.add_argument("--window", type=int, default=10, help="runs of the step in a segment")
    ap.add_argument("--save", metavar="FILE", help="write this rank's events")
    ap.add_argument("--compare", nargs="+", metavar="FILE", help="compare saved ranks instead of running the step")
    ap.add_argument("--expert-ranks", type=int, default=8)
    a = ap.parse_args(argv)
    if a.compare:
        traces = [dict(np.load(f)) for f in a.compare]
        r = compare(traces)
        for i, f in enumerate(a.compare):
            slow = [NAMES[k] for k in range(len(NAMES)) if r["degraded"][i, k]]
            other = ""
            if "outputs_differ" in r:
                names = [n for n, x in zip(OUTPUTS, r["outputs_differ"][i]) if x]
                other = f"; OUTPUTS DIFFER: {', '.join(names)}" if names else "; outputs as the others'"
            print(f"{f}: score {r['score_pm'][i].tolist()} permille, straggler in {int(r['straggler'][i].sum())} of "
                  f"{len(r['straggler'][i])} segments, degraded operators: {', '.join(slow) or 'none'}{other}")
        return 0
    if a.expert_ranks < 1 or Config.experts % a.expert_ranks:
        ap.error(f"--expert-ranks has to divide the step's {Config.experts} experts")
    check = RankCheck()
    t = check.trace(a.steps, a.window)
    if a.save:
        np.savez(a.save, **t)
    took = (t["end_ns"] - t["start_ns"]) / 1e3
    for k, name in enumerate(NAMES):
        d = took[t["kernel_id"] == k]
        print(f"{name:20s} median {np.median(d):9.1f} us   p99 {np.quantile(d, 0.99):9.1f} us")
    load = expert_load(check.step()["count"], a.expert_ranks)
    print(f"tokens of the step's router on {a.expert_ranks} expert-parallel ranks, permille of the even share: "
          f"{load.tolist()}")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
