"""Pipeline.fork() around the library's copy: which trackers move, in which order of streams, and with
what workspace.  CPU only: the copy, the streams and the bank are stand-ins."""
import contextlib
import types

import pytest
import torch


class Stream:
    def __init__(self, name, calls):
        self.name, self.calls, self.seen = name, calls, lambda: None

    def __eq__(self, other):
        return self.name == other.name

    def wait_stream(self, other):
        self.calls.append((self.name, "waits for", other.name, self.seen()))


@pytest.fixture()
def fork(monkeypatch):
    """fork(parent, ...) over pipelines without a GPU; .calls lists what was asked of the library and the streams."""
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import pipeline

    calls = []

    def make(U, first, stream=None):
        p = pipeline.Pipeline.__new__(pipeline.Pipeline)
        p.w, p.device, p.stream = types.SimpleNamespace(U=U), torch.device("cpu"), stream
        p.track = (torch.arange(6 * U, dtype=torch.int32) + first).view(U, 6)
        p.bank = types.SimpleNamespace(U=U, ring_cap=0, copies=torch.full((U,), 3, dtype=torch.int64))
        p.bank.full = []                                   # units that a copy finds no room in
        p.status = torch.zeros(1, dtype=torch.int32)
        return p

    def copy(dst, src, parent, keep, workspace, status, stream=None):
        calls.append(("copy", workspace.numel()))
        assert parent.numel() == dst.U
        assert keep is None or workspace.numel() >= pipeline.rs3.rs3_bank_copy_workspace_bytes(dst.U, keep.shape[1])
        for u in range(dst.U):
            if not -1 <= int(parent[u]) < src.U:
                status.fill_(pipeline.rs3.RS3_EINVAL)
            elif u in dst.full:
                status.fill_(pipeline.rs3.RS3_ECAPACITY)
            elif int(parent[u]) >= 0:
                dst.copies[u] += 1

    monkeypatch.setattr(pipeline.rs3, "rs3_bank_copy", copy)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("current", calls))
    return types.SimpleNamespace(make=make, calls=calls, rs3=pipeline.rs3)


def parents(*p):
    return torch.tensor(p, dtype=torch.int32)


@pytest.mark.parametrize("bad", [3, 4, 1 << 30, (1 << 31) - 1, -2, -(1 << 31)])
def test_a_parent_that_is_no_unit_is_left_to_the_copy(fork, bad):
    """It latches RS3_EINVAL and leaves its unit as it is: no index goes past the trackers for it."""
    a, b = fork.make(3, 100), fork.make(3, 500)
    was = b.track.clone()
    a.fork(parents(2, bad, -1), into=b)
    assert int(b.status) == fork.rs3.RS3_EINVAL
    assert torch.equal(b.track[0], a.track[2]) and torch.equal(b.track[1:], was[1:])


@pytest.mark.parametrize("here,there", [("a", "b"), ("a", None), (None, "b")])
def test_the_target_s_stream_is_waited_for_and_waits(fork, here, there):
    """What the target's stream does goes before the copy, and what it does next after the trackers."""
    a, b = (fork.make(2, n, s and Stream(s, fork.calls)) for n, s in ((100, here), (500, there)))
    seen = lambda: bool(torch.equal(b.track, a.track))
    if b.stream:
        b.stream.seen = seen
    a.fork(parents(0, 1), into=b)
    x, y = here or "current", there or "current"
    first, copy, last = fork.calls
    assert first[:3] == (x, "waits for", y) and copy[0] == "copy" and last[:3] == (y, "waits for", x)
    assert last[3] is (True if there else None)


@pytest.mark.parametrize("name", ["a", None])
def test_one_stream_waits_for_nothing(fork, name):
    a, b = (fork.make(2, n, name and Stream(name, fork.calls)) for n in (100, 500))
    a.fork(parents(0, 1), into=b)
    assert [c[0] for c in fork.calls] == ["copy"]


def test_a_unit_that_the_copy_leaves_keeps_its_tracker(fork):
    a, b = fork.make(3, 100), fork.make(3, 500)
    b.bank.full = [1]
    was = b.track.clone()
    a.fork(parents(0, 2, -1), into=b)
    assert int(b.status) == fork.rs3.RS3_ECAPACITY
    assert torch.equal(b.track[0], a.track[0]) and torch.equal(b.track[1:], was[1:])
    b.bank.full = []
    a.fork(parents(-1, 2, -1), into=b)                     # (a copy counted before is not taken for this one's)
    assert torch.equal(b.track[1], a.track[2]) and torch.equal(b.track[2], was[2])


@pytest.mark.parametrize("U", [1, 2, 5])
def test_a_target_with_another_number_of_units(fork, U):
    """The workspace is the target's, a unit of its own each; trackers go by the parents."""
    a, b = fork.make(3, 100), fork.make(U, 500)
    p = parents(2, 0, -1, 2, 1)[:U]
    was = b.track.clone()
    a.fork(p, torch.ones((U, 5000), dtype=torch.uint8), into=b)
    for u in range(U):
        assert torch.equal(b.track[u], was[u] if p[u] < 0 else a.track[int(p[u])])
    for bad in (p[:-1], torch.cat([p, p])):
        with pytest.raises(ValueError):
            a.fork(bad, into=b)
    assert len(fork.calls) == 1                            # (nothing was copied)
