"""The rank check's dense step (rotary positions, gated feed-forward and cross
entropy among the others): against the same step in 64 bits under torch's own
differentiation, its bits, its trace, and repeated graph replays."""
import math

import numpy as np
import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import rank_check as rc

pytestmark = pytest.mark.gpu
SMALL = rc.Config(doc_lens=(70, 33, 1, 96), vocab=120, width=256, heads=4, kv_heads=2, head_dim=64, ff=328)


def _turn(t, pos, freq):
    """Rotary positions of [tokens, heads, dim], halves' layout, in 64 bits."""
    a = (pos[:, None].double() * freq)[:, None]
    u, v = t.chunk(2, -1)
    return torch.cat([u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()], -1)


def _reference(check):
    c = check.cfg
    names = ("table", "w_qkv", "w_out", "w_gate", "w_up", "w_down", "w_head")
    p = {n: getattr(check, n).cpu().double().requires_grad_() for n in names}
    norms = [[t.cpu().double().requires_grad_() for t in w] for w in (check.norm1, check.norm2, check.norm3)]
    T, H, N, D, W = len(check.ids), c.heads, c.kv_heads, c.head_dim, c.width
    norm = lambda t, w: torch.nn.functional.layer_norm(t, (W,), *w, 1e-5)  # noqa: E731
    x = p["table"][check.ids.cpu()] * W**0.5
    qkv = (norm(x, norms[0]) @ p["w_qkv"]).view(T, H + 2 * N, D)
    pos = torch.cat([torch.arange(n) for n in c.doc_lens])
    freq = c.rope_base ** -(torch.arange(0, D, 2).double() / D)
    q, k, v = _turn(qkv[:, :H], pos, freq), _turn(qkv[:, H:H + N], pos, freq), qkv[:, H + N:]
    o, lo = [], 0
    for n in c.doc_lens:
        qd, kd, vd = q[lo:lo + n], k[lo:lo + n].repeat_interleave(H // N, 1), v[lo:lo + n].repeat_interleave(H // N, 1)
        s = (torch.einsum("ihd,jhd->hij", qd, kd) / D**0.5).masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
        o.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), vd))
        lo += n
    h = x + torch.cat(o).reshape(T, H * D) @ p["w_out"]
    z = norm(h, norms[1])
    h = h + (torch.nn.functional.silu(z @ p["w_gate"].T) * (z @ p["w_up"].T)) @ p["w_down"]
    labels = torch.full((T,), -100)
    lo = 0
    for n in c.doc_lens:
        labels[lo:lo + n - 1] = check.ids[lo + 1:lo + n].cpu()
        lo += n
    loss = torch.nn.functional.cross_entropy(norm(h, norms[2]) @ p["w_head"].T, labels, ignore_index=-100)
    loss.backward()
    return {"h": h.detach(), "loss": loss.detach().view(1), "d_table": p["table"].grad, "d_qkv": p["w_qkv"].grad,
            "d_out": p["w_out"].grad, "d_gate": p["w_gate"].grad, "d_up": p["w_up"].grad, "d_down": p["w_down"].grad,
            "d_head": p["w_head"].grad, **{f"d_norm{i + 1}": [t.grad for t in w] for i, w in enumerate(norms)}}


def test_step_against_64_bits():
    check = rc.DenseCheck(SMALL)
    got, ref = check.step(), _reference(check)
    assert tuple(got) == rc.DENSE_OUTPUTS
    # every stage rounds to bfloat16 (2^-9 of a value, independent errors); the
    # longest chain, forward and back, has about thirty: sqrt(30) 2^-9 = 1.1 %,
    # and the norms' 1 / std and the softmax at most triple it
    for name, want in ref.items():
        pairs = zip(got[name], want) if isinstance(want, list) else [(got[name], want)]
        for a, b in pairs:
            assert float((a.cpu().double().view(b.shape) - b).norm()) < 0.035 * float(b.norm()), name


def test_same_bits_each_time():
    a, b = rc.DenseCheck(SMALL), rc.DenseCheck(SMALL)
    assert (rc.digest(a.step()) == rc.digest(b.step())).all() and (rc.digest(a.step()) == rc.digest(b.step())).all()


def test_trace_and_compare(tmp_path, capsys):
    t = rc.DenseCheck(SMALL).trace(steps=2, window=8, warmup=2)
    assert len(t["kernel_id"]) == 2 * 8 * len(rc.DENSE_NAMES) and tuple(t["names"]) == rc.DENSE_NAMES
    slow = rc.DENSE_NAMES.index("cross_entropy_bwd")

    def rank(f, only=None):
        d = (t["end_ns"] - t["start_ns"]).astype(np.float64) + 1000
        return dict(t, end_ns=t["start_ns"] + np.where((only is None) | (t["kernel_id"] == (only or 0)), d * f, d).astype(np.int64))

    ranks = [rank(1.0) for _ in range(6)] + [rank(1.7), rank(3.0, slow)]
    r = rc.compare(ranks)
    assert r["straggler"][6].all() and not r["straggler"][:6].any()
    assert r["degraded"][7].nonzero().flatten().tolist() == [slow] and not r["outputs_differ"].any()
    files = [str(tmp_path / f"r{i}.npz") for i in range(8)]
    for f, x in zip(files, ranks):
        np.savez(f, **x)
    assert rc.main(["--compare", *files]) == 0
    out = capsys.readouterr().out.splitlines()
    assert "degraded operators: cross_entropy_bwd" in out[7] and "outputs as the others'" in out[0]
    with pytest.raises(pa.ArgusError):  # a rank that ran the other step
        rc.compare([t, rc.RankCheck(SMALL).trace(steps=2, window=8)])


def test_graph_replays():
    # captured (no allocation, no clearing by the runtime) and replayed with
    # eager work between; a second graph shares the buffers and the workspaces
    T, W, F, V = 300, 136, 264, 1_003
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, wg, wu, dh, w, heads = r(T, W), r(F, W), r(F, W), r(T, F), r(V, W), r(T, 6, 40)
    labels = torch.randint(-20, V, (T,), generator=g, device="cuda")
    one, (freq, _) = torch.ones(1, device="cuda"), pa.rotary_freq(32)
    outs = {"r": {"out": torch.empty_like(heads)}, "f": pa.alloc_gated_ff(T, F, torch.bfloat16, True),
            "fb": pa.alloc_gated_ff_bwd(T, W, F, torch.bfloat16), "c": pa.alloc_cross_entropy(T),
            "cb": pa.alloc_cross_entropy_bwd(T, V, W), "few": pa.alloc_cross_entropy(9), "ff1": pa.alloc_gated_ff(3, F, torch.bfloat16)}

    def run():
        pa.rotary(heads, freq, out=outs["r"])
        f = pa.gated_ff(x, wg, wu, save=True, out=outs["f"])
        pa.gated_ff_bwd(dh, x, wg, wu, f["g"], f["u"], out=outs["fb"])
        c = pa.cross_entropy(x, w, labels, out=outs["c"])
        pa.cross_entropy_bwd(x, w, labels, c["lse"], c["n_valid"], dmean=one, out=outs["cb"])
        pa.cross_entropy(x[:9], w, labels[:9], out=outs["few"])
        pa.gated_ff(x[:3], wg, wu, out=outs["ff1"])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(s):
        run()
        s.synchronize()
        for graph in graphs:
            with torch.cuda.graph(graph, stream=s):
                run()
    torch.cuda.current_stream().wait_stream(s)
    for i in range(4):
        for t in (x, dh, w, heads):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda").to(t.dtype))
        labels.copy_(torch.randint(-300 if i % 2 else -20, V, (T,), generator=g, device="cuda"))
        for o in outs.values():
            for n, t in o.items():
                t.fill_(1) if n != "_workspace" else t.fill_(255)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = {m: {n: t.clone() for n, t in o.items() if n != "_workspace"} for m, o in outs.items()}
        run()
        torch.cuda.synchronize()
        for m, o in outs.items():
            for n, t in o.items():
                if n != "_workspace":
                    assert torch.equal(got[m][n], t), (i, m, n)
