"""What beside_prefill reports, on a simulated device of two streams that slow each other down: a step's time beside
encode is that of the steps beside it, not of those before and after.  No GPU."""
import contextlib

import pytest
import torch

from paper_2609_31551_amd import colocate as K


class Device:
    """Streams of work that runs at 1 ms a ms alone, and slower beside the other kind; a host that takes its time."""

    def __init__(self, encode_slow, step_slow):
        self.slow = {"encode": encode_slow, "step": step_slow}
        self.now, self.host, self.streams = 0.0, 0.0, []

    def stream(self):
        s = Stream(self)
        self.streams.append(s)
        return s

    def run(self):
        """Until nothing more can be done; the host waits for that."""
        while True:
            heads = []
            for s in self.streams:
                while s.ops and s.ops[0][1] <= self.now and s.ops[0][0] in ("record", "wait"):
                    kind, _, what = s.ops[0]
                    if kind == "wait" and what.at is None:
                        break
                    if kind == "record":
                        what.at = self.now
                    s.ops.pop(0)
                if s.ops and s.ops[0][0] not in ("record", "wait") and s.ops[0][1] <= self.now:
                    heads.append(s.ops[0])
            later = [s.ops[0][1] for s in self.streams if s.ops and s.ops[0][1] > self.now]
            kinds = {h[0] for h in heads} & {"encode", "step"}
            rate = {k: self.slow[k] if len(kinds) == 2 else 1.0 for k in kinds}
            work = [h for h in heads if h[0] in rate]
            gates = [h for h in heads if h[0] == "gate" and h[2].release is not None]
            ends = [self.now + h[2][0] * rate[h[0]] for h in work] + [max(self.now, g[2].release) for g in gates] + later
            if not ends:
                if any(s.ops and s.ops[0][0] == "wait" and s.ops[0][1] <= self.now and s.ops[0][2].at is not None
                       for s in self.streams):
                    continue
                break
            step = min(ends)
            for h in work:
                h[2][0] -= (step - self.now) / rate[h[0]]
            self.now = step
            for s in self.streams:
                if s.ops and ((s.ops[0] in work and s.ops[0][2][0] <= 1e-9) or (s.ops[0] in gates and s.ops[0][2].release <= self.now)):
                    s.ops.pop(0)
        self.host = max(self.host, self.now)


class Stream:
    def __init__(self, dev):
        self.dev, self.ops = dev, []

    def add(self, kind, what, host_ms=0.0):
        self.dev.host += host_ms
        self.ops.append((kind, self.dev.host, what))

    def wait_event(self, e):
        self.add("wait", e)

    def synchronize(self):
        self.dev.run()


class Event:
    dev = None

    def __init__(self, enable_timing=False):
        self.at = None

    def record(self, stream):
        stream.add("record", self)

    def synchronize(self):
        self.dev.run()
        assert self.at is not None

    def elapsed_time(self, other):
        return other.at - self.at


class Gate(contextlib.AbstractContextManager):
    dev = None

    def __init__(self, n, max_s=10.0):
        self.release = None

    def __enter__(self):
        self.dev.run()
        self.stream = self.dev.stream()
        self.stream.add("gate", self)
        return self

    def __exit__(self, *exc):
        self.release = self.dev.host

    def lapsed(self):
        return False


class Work:
    def __init__(self, ms):
        self.ms = ms

    def step(self, stream):
        stream.add("step", [self.ms], host_ms=0.06)


# sizes in ms; how many times longer either kind takes beside the other
@pytest.mark.parametrize("encode_ms,step_ms,encode_slow,step_slow", [
    (25.0, 0.15, 1.5, 2.0), (1.6, 0.15, 2.5, 1.3), (1.0, 0.5, 2.0, 3.0), (0.4, 1.0, 2.0, 2.0), (5.0, 0.15, 9.0, 1.1),
    (3.0, 0.05, 1.5, 1.5)])
def test_times_beside_are_times_beside(monkeypatch, encode_ms, step_ms, encode_slow, step_slow):
    dev = Device(encode_slow, step_slow)
    streams = {}
    monkeypatch.setattr(K, "_stream", lambda role: streams.setdefault(role, dev.stream()))
    monkeypatch.setattr(K, "CuReservation", type("G", (Gate,), {"dev": dev}))
    monkeypatch.setattr(torch.cuda, "Event", type("E", (Event,), {"dev": dev}))
    monkeypatch.setattr(torch.cuda, "synchronize", dev.run)

    def run(stream):
        stream.add("encode", [encode_ms], host_ms=0.5)
    ms = K.beside_prefill(run, Work(step_ms), reps=2)
    assert ms["prefill_beside"] == pytest.approx(step_ms * step_slow, rel=0.02)
    assert ms["prefill_alone"] == pytest.approx(step_ms, rel=0.02)
    assert ms["encode_alone"] == pytest.approx(encode_ms, rel=0.01)
    assert ms["encode_beside"] == pytest.approx(encode_ms * encode_slow, rel=0.02)
