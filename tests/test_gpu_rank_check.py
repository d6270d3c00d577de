"""The rank check: its step against the same step in 64 bits under torch's own
differentiation, its trace through the detectors, and repeated graph replays."""
import numpy as np
import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import rank_check as rc

pytestmark = pytest.mark.gpu
SMALL = rc.Config(doc_lens=(70, 33, 1, 96), vocab=120, width=256, heads=4, kv_heads=2, head_dim=64, experts=16, top_k=3)


def _reference(check, expert):
    """The step's gradients on the host in 64 bits; the choice of experts is
    given, since rounding may swap near ties."""
    c = check.cfg
    p = {n: getattr(check, n).cpu().double().requires_grad_() for n in ("table", "w_qkv", "w_out", "w_router")}
    n1, n2 = ([t.cpu().double().requires_grad_() for t in w] for w in (check.norm1, check.norm2))
    T, H, N, D = len(check.ids), c.heads, c.kv_heads, c.head_dim
    x = p["table"][check.ids.cpu()] * c.width**0.5
    y = torch.nn.functional.layer_norm(x, (c.width,), *n1, 1e-5)
    qkv = (y @ p["w_qkv"]).view(T, H + 2 * N, D)
    o, lo = [], 0
    for n in c.doc_lens:
        q, k, v = qkv[lo:lo + n, :H], qkv[lo:lo + n, H:H + N], qkv[lo:lo + n, H + N:]
        k, v = (t.repeat_interleave(H // N, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) / D**0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
        o.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), v))
        lo += n
    h = x + torch.cat(o).reshape(T, H * D) @ p["w_out"]
    z = torch.nn.functional.layer_norm(h, (c.width,), *n2, 1e-5)
    prob = (z @ p["w_router"]).softmax(1)
    at = expert.cpu().long()
    count = torch.bincount(at.reshape(-1), minlength=c.experts).double()
    loss = c.alpha * c.experts * (count / (c.top_k * T) * prob.mean(0)).sum()
    total = loss + (prob.gather(1, at) * check.d_gate.cpu().double()).sum() + (z * check.d_out.cpu().double()).sum()
    total.backward()
    return {"d_table": p["table"].grad, "d_qkv": p["w_qkv"].grad, "d_out": p["w_out"].grad, "d_router": p["w_router"].grad,
            "d_norm1": [t.grad for t in n1], "d_norm2": [t.grad for t in n2], "h": h.detach(), "loss": loss.detach(),
            "prob": prob.detach()}


def test_step_against_64_bits():
    check = rc.RankCheck(SMALL)
    got = check.step()
    ref = _reference(check, got["expert"])
    # every stage rounds to bfloat16 (2^-9 of a value, independent errors); the
    # longest chain has about twenty roundings: sqrt(20) 2^-9 = 0.9 %, and
    # the norms' 1 / std and the softmax at most triple it
    for name in ("h", "d_table", "d_qkv", "d_out", "d_router"):
        a, b = got[name].cpu().double(), ref[name]
        assert float((a - b).norm() / b.norm()) < 0.03, name
    for name in ("d_norm1", "d_norm2"):
        for a, b in zip(got[name], ref[name]):
            assert float((a.cpu().double() - b).norm() / b.norm()) < 0.03, name
    assert abs(float(got["loss"]) - float(ref["loss"])) < 0.03 * float(ref["loss"])
    assert int(got["count"].sum()) == len(check.ids) * SMALL.top_k


def test_same_bits_each_time():
    check = rc.RankCheck(SMALL)
    a, b = check.step(), rc.RankCheck(SMALL).step()
    for k in ("expert", "gate", "count", "loss", "d_table"):
        assert torch.equal(a[k], b[k]), k


def test_trace_and_compare():
    check = rc.RankCheck(SMALL)
    t = check.trace(steps=3, window=9, warmup=2)
    assert len(t["kernel_id"]) == 3 * 9 * len(rc.NAMES) and t["seg_off"].tolist() == [0, 144, 288, 432]
    assert (t["end_ns"] >= t["start_ns"]).all() and (np.diff(t["start_ns"]) >= 0).all()
    # peers made from this rank's own events: the same, one all slower, one
    # with a single slower operator
    def scaled(f, only=None):
        d = (t["end_ns"] - t["start_ns"]).astype(np.float64)
        d = np.where((only is None) | (t["kernel_id"] == (only or 0)), d * f, d).astype(np.int64) + 1000
        return dict(t, end_ns=t["start_ns"] + d)
    slow = rc.NAMES.index("attention_bwd")
    peers = [scaled(1.0) for _ in range(6)] + [scaled(1.6), scaled(3.0, slow)]
    r = rc.compare(peers)
    assert r["straggler"][6].all() and not r["straggler"][:6].any() and not r["straggler"][7].any()
    assert r["degraded"][7].nonzero().flatten().tolist() == [slow]
    assert not r["degraded"][:6].any()
    with pytest.raises(pa.ArgusError):
        rc.compare([t, dict(t, seg_off=t["seg_off"][:-1])])


def test_expert_load():
    count = torch.tensor([10, 10, 30, 30], dtype=torch.int32)
    assert rc.expert_load(count, 2).tolist() == [500, 1500]
    assert rc.expert_load(torch.zeros(4, dtype=torch.int32), 2).tolist() == [0, 0]


def test_command(tmp_path, capsys):
    # the saved events of a rank, compared with copies of themselves
    t = rc.RankCheck(SMALL).trace(steps=2, window=8)
    files = [str(tmp_path / f"r{i}.npz") for i in range(4)]
    for f in files:
        np.savez(f, **t)
    assert rc.main(["--compare", *files]) == 0
    assert capsys.readouterr().out.count("straggler in 0 of 2 segments") == 4


def test_graph_replays():
    # the operators are captured (no allocation, no clearing by the runtime)
    # and replayed with eager work between the replays
    T, H, D = 300, 4, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s, dt=torch.bfloat16: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    ids = torch.randint(0, 90, (2000,), generator=g, device="cuda")
    dout, x, w = r(2000, 72), r(T, 520), r(520, dt=torch.float32)
    q, k, v, do = r(T, H, D), r(T, 2, D), r(T, 2, D), r(T, H, D)
    logits, off = r(T, 40), torch.tensor([0, 110, T], device="cuda")
    outs = {"e": pa.alloc_embedding(2000, 72, torch.bfloat16), "eb": pa.alloc_embedding_bwd(90, 72, torch.bfloat16),
            "l": pa.alloc_layer_norm(T, 520, torch.bfloat16),
            "lb": pa.alloc_layer_norm_bwd(T, 520, torch.bfloat16, torch.float32), "b": pa.alloc_balance(T, 40, 4),
            "bb": {"dlogits": torch.empty_like(logits)}, "a": pa.alloc_attention(T, H, D),
            "ab": pa.alloc_attention_bwd(T, T, H, 2, D)}
    table, one = r(90, 72), torch.ones(1, device="cuda")

    def run():
        pa.embedding(ids, table, 2.0, out=outs["e"])
        pa.embedding_bwd(ids, dout, 90, out=outs["eb"])
        pa.layer_norm(x, w, out=outs["l"])
        pa.layer_norm_bwd(x, x, outs["l"]["mean"], outs["l"]["rstd"], w, out=outs["lb"])
        b = pa.balance(logits, 4, out=outs["b"])
        pa.balance_bwd(logits, b["lse"], b["expert"], b["count"], b["n_valid"], one, out=outs["bb"])
        a = pa.attention(q, k, v, q_off=off, out=outs["a"])
        pa.attention_bwd(do, q, k, v, a["o"], a["lse"], q_off=off, out=outs["ab"])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run()
    torch.cuda.current_stream().wait_stream(s)
    for i in range(3):
        for t in (dout, x, q, logits):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda").to(t.dtype))
        for o in outs.values():
            for n, t in o.items():
                if n != "_workspace":
                    t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = {m: {n: t.clone() for n, t in o.items() if n != "_workspace"} for m, o in outs.items()}
        run()
        torch.cuda.synchronize()
        for m, o in outs.items():
            for n, t in o.items():
                if n != "_workspace":
                    assert torch.equal(got[m][n], t), (i, m, n)


def test_outputs_of_a_machine_that_computes_wrongly_are_named(tmp_path, capsys, monkeypatch):
    good = [rc.RankCheck(SMALL).trace(steps=2, window=8) for _ in range(3)]
    assert tuple(rc.RankCheck(SMALL).step()) == rc.OUTPUTS
    right = pa.ops.balance_bwd

    def wrong(*args, **kw):  # one bit of one logit's gradient
        out = right(*args, **kw)
        out["dlogits"].view(torch.int16)[5, 2] ^= 1 << 12
        return out

    monkeypatch.setattr(pa.ops, "balance_bwd", wrong)
    bad = rc.RankCheck(SMALL).trace(steps=2, window=8)
    d = rc.compare([*good, bad])["outputs_differ"]
    assert not d[:3].any()
    named = {n for n, x in zip(rc.OUTPUTS, d[3]) if x}
    assert "d_router" in named and not named & {"h", "expert", "gate", "count", "loss"}
    files = [str(tmp_path / f"r{i}.npz") for i in range(4)]
    for f, t in zip(files, [*good, bad]):
        np.savez(f, **t)
    assert rc.main(["--compare", *files]) == 0
    lines = capsys.readouterr().out.splitlines()
    assert all("outputs as the others'" in x for x in lines[:3]) and "OUTPUTS DIFFER" in lines[3] and "d_router" in lines[3]
    # events saved without their outputs are still compared by their times
    for f, t in zip(files, [*good, bad]):
        np.savez(f, **{k: v for k, v in t.items() if k != "digest"})
    assert rc.main(["--compare", *files]) == 0
    assert all(x.rpartition("operators: ")[2].count(";") == 0 for x in capsys.readouterr().out.splitlines())
