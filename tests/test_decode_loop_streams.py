"""On the CPU: the order in which the decoding loop enqueues -- its stream behind
the program's before the first plan, and the program's behind it at the end,
also where a producer raises.  Streams and steps are stand-ins that keep a log."""
import numpy as np
import pytest
import torch

from paper_2406_11016_amd.decode_loop import DecodeLoop


class Stream:
    device = torch.device("cuda", 0)

    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append(f"{self.name} waits for {other.name}")


class Cache:
    def __init__(self, log):
        self.log, self.counts = log, torch.zeros(2, dtype=torch.int32)

    def plan(self, n, accepted_len=None):
        self.log.append(f"plan {n}")
        self.counts.fill_(n)


class Loop(DecodeLoop):
    def __init__(self, log, cache):
        self.B, self.gamma0, self.gamma_max, self.mode, self.early_exit, self.adapt_gamma = 2, 3, 6, "exact", "never", True
        self.native, self._early_next, self.cache, self.stream = None, False, cache, Stream("loop", log)
        self.acc = torch.full((2,), -1, dtype=torch.int32)
        self._counts_host = torch.zeros(2, dtype=torch.int32)
        self._keep_all, self._unverified = True, False

    def launch(self, gamma, early=False):
        self.stream.log.append("step")
        self._unverified = False

    def collect(self):
        return np.zeros(2, np.int32), np.zeros(2, np.int32)


@pytest.mark.parametrize("with_cache", [True, False])
def test_streams_are_ordered(monkeypatch, with_cache):
    log = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("program", log))
    loop = Loop(log, Cache(log) if with_cache else None)
    loop.run(lambda loop, i, gamma: log.append("producer"), 2)
    steps = ["plan 4", "producer", "step", "plan 3", "producer", "step"]
    assert log == ["loop waits for program", *[x for x in steps if with_cache or not x.startswith("plan")],
                   "program waits for loop"]
    log.clear()

    def fails(loop, i, gamma):
        raise KeyError("producer")

    with pytest.raises(KeyError):
        loop.run(fails, 2)
    assert log[0] == "loop waits for program" and log[-1] == "program waits for loop"
    assert loop.acc.tolist() == [-1, -1]
