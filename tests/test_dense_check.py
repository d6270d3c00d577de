"""The rank check's dense step, host side (no GPU needed)."""
import numpy as np
import pytest
import torch

from paper_2606_20374_amd import argus
from paper_2606_20374_amd import rank_check as rc


def test_names_and_outputs():
    assert len(set(rc.DENSE_NAMES)) == len(rc.DENSE_NAMES) and len(set(rc.DENSE_OUTPUTS)) == len(rc.DENSE_OUTPUTS)
    assert rc.RankCheck.NAMES == rc.NAMES and rc.DenseCheck.NAMES == rc.DENSE_NAMES
    assert rc.step_names({}) == rc.NAMES  # saved before traces held their names
    assert rc.step_names({"names": np.array(rc.DENSE_NAMES)}) == rc.DENSE_NAMES


def test_inputs_on_the_host():
    # the same tokens and weights as the other step's, labels inside documents
    cfg = rc.Config(doc_lens=(5, 1, 3), vocab=50, width=32, heads=2, kv_heads=1, head_dim=16, ff=40, experts=4)
    a, b = rc.RankCheck(cfg, "cpu"), rc.DenseCheck(cfg, "cpu")
    assert torch.equal(a.ids, b.ids) and torch.equal(a.w_qkv, b.w_qkv)
    assert b.pos.tolist() == [0, 1, 2, 3, 4, 0, 0, 1, 2]
    ids = a.ids.tolist()
    assert b.labels.tolist() == [*ids[1:5], -1, -1, *ids[7:9], -1]


def test_traces_of_different_steps_are_refused():
    t = {"seg_off": np.arange(3)}
    with pytest.raises(argus.ArgusError, match="different steps"):
        rc.compare([t, {**t, "names": np.array(rc.DENSE_NAMES)}])


def test_the_command_runs_the_step_that_is_asked_for(monkeypatch, capsys):
    made = []

    class Check:
        def __init__(self):
            made.append(self.NAMES)

        def trace(self, steps, window):
            k = np.arange(len(self.NAMES), dtype=np.int32)
            return {"kernel_id": k, "start_ns": k * 1000, "end_ns": k * 1000 + 500}

        def step(self):
            return {"count": torch.ones(128, dtype=torch.int32)}

    monkeypatch.setattr(rc, "RankCheck", type("A", (Check,), {"NAMES": rc.NAMES}))
    monkeypatch.setattr(rc, "DenseCheck", type("B", (Check,), {"NAMES": rc.DENSE_NAMES}))
    assert rc.main([]) == 0
    assert "expert-parallel" in capsys.readouterr().out
    assert rc.main(["--dense"]) == 0
    out = capsys.readouterr().out
    assert "cross_entropy_bwd" in out and "expert-parallel" not in out
    assert made == [rc.NAMES, rc.DENSE_NAMES]
