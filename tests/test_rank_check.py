"""The rank check's host side (no GPU needed): the clock of its events, and what
its command does before and after the run."""
import numpy as np
import pytest
import torch

from paper_2606_20374_amd import argus
from paper_2606_20374_amd import rank_check as rc


class Event:
    """A device event on a made-up clock; a difference has 32 bits, in
    milliseconds, like the device's."""
    now_ns = 0

    def __init__(self, enable_timing=False):
        pass

    def record(self, stream=None):
        self.at = Event.now_ns

    def elapsed_time(self, end):
        return float(np.float32((end.at - self.at) / 1e6))


def _trace(monkeypatch, steps, window, run_ns):
    """RankCheck.trace of a step whose operator k takes run_ns[k]."""
    check = object.__new__(rc.RankCheck)
    check.device = torch.device("cuda", 0)

    def step(mark=lambda name: None):
        for name, ns in zip(rc.NAMES, run_ns):
            Event.now_ns += ns
            mark(name)
        return {}

    check.step = step
    Event.now_ns = 0
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: None)
    return check.trace(steps, window, warmup=0)


def test_durations_of_a_long_trace(monkeypatch):
    # a minute of steps: the differences of 32-bit milliseconds are 2^-24 of a
    # duration off, and rounded to whole nanoseconds
    run_ns = [20_011, 15_007, 5_000_003, 12_001, 9_999, 10_007] + [1_000_003] * (len(rc.NAMES) - 6)
    t = _trace(monkeypatch, steps=40, window=100, run_ns=run_ns)
    took = t["end_ns"] - t["start_ns"]
    assert t["end_ns"][-1] > 59e9 and len(took) == 4000 * len(rc.NAMES)
    want = np.tile(run_ns, 4000)
    assert (np.abs(took - want) <= 1 + want * 2.0**-23).all()
    # one operator begins where the one before it ended
    assert (t["start_ns"][1:] == t["end_ns"][:-1]).all()


@pytest.mark.parametrize("ranks", ["7", "0", "-8", "256"])
def test_expert_ranks_that_do_not_divide_the_experts_are_refused_before_the_run(monkeypatch, ranks):
    def none(*args):
        raise AssertionError("the step was run")

    monkeypatch.setattr(rc, "RankCheck", none)
    with pytest.raises(SystemExit) as e:
        rc.main(["--expert-ranks", ranks])
    assert e.value.code == 2
    with pytest.raises(argus.ArgusError):
        rc.expert_load(torch.ones(128, dtype=torch.int32), int(ranks))


def test_ranks_whose_outputs_differ():
    # four ranks of three outputs: one rank alone with its first, two pairs
    # with their second (no majority: all are named), all alike in the third
    d = np.array([[1, 5, 9], [1, 5, 9], [2, 6, 9], [1, 6, 9]], dtype=np.uint64)
    want = [[False, True, False], [False, True, False], [True, True, False], [False, True, False]]
    assert rc.outputs_differ(list(d)).tolist() == want
    assert rc.outputs_differ([d[0]]).tolist() == [[False] * 3]
    with pytest.raises(argus.ArgusError):
        rc.outputs_differ([d[0], d[0][:2]])


def test_digest_tells_bits():
    a = {"x": torch.tensor([1.0, 0.0]), "y": (torch.ones(3, dtype=torch.bfloat16), torch.zeros(2))}
    b = {"x": torch.tensor([1.0, -0.0]), "y": (torch.ones(3, dtype=torch.bfloat16), torch.zeros(2))}
    c = {"x": torch.tensor([1.0, 0.0]), "y": (torch.ones(3, dtype=torch.bfloat16), torch.zeros(2) + 1e-40)}
    da, db, dc = (rc.digest(x) for x in (a, b, c))
    assert (da == rc.digest(a)).all() and (da != db).tolist() == [True, False] and (da != dc).tolist() == [False, True]
