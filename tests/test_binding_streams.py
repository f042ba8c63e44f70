"""Memory that the calls of a decoding step and the table builds allocate for work on a stream of the caller's, seen on the host with a stand-in
for the library."""
import contextlib

import pytest
import torch

import paper_2410_03355_amd as L
from paper_2410_03355_amd import binding

V, K, N, M = 8, 2, 4, 2
I32 = torch.int32


class _Library:
    def __getattr__(self, name):
        return lambda *args: 4096 if name.endswith("_bytes") else binding.OK


@pytest.fixture
def watched(monkeypatch):
    """(side stream, memory allocated as (address, inside the side stream's context), memory kept for the current stream)."""
    side, made, kept, inside = object(), [], [], [0]

    @contextlib.contextmanager
    def on(stream):
        assert stream is side
        inside[0] += 1
        yield
        inside[0] -= 1

    empty = torch.empty

    def noted(*args, **kwargs):
        t = empty(*args, **kwargs)
        made.append((t.data_ptr(), inside[0]))
        return t

    monkeypatch.setattr(binding, "load", lambda: _Library())
    monkeypatch.setattr(binding, "_marshal", binding._Declines())
    monkeypatch.setattr(binding, "_need_cuda", lambda *a: None)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "current")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t.data_ptr(), s)))
    monkeypatch.setattr(torch, "empty", noted)
    return side, made, kept


def _tensors(got):
    return [t for t in (got.values() if isinstance(got, dict) else got if isinstance(got, tuple) else (got,)) if t is not None]


t, g, tok, table, un = torch.zeros(N, V), torch.zeros(N, V), torch.zeros(N, dtype=I32), torch.zeros(V, K, dtype=I32), torch.zeros(N, 2)
acc, parent = torch.zeros(N, dtype=I32), torch.full((N,), -1, dtype=I32)
CALLS = {
    "verify": lambda s: L.verify(t, g, tok, table, 0.1, un, stream=s),
    "verify_ex": lambda s: L.verify_ex(t, g, tok, table, 0.1, un, stream=s),
    "verify_greedy": lambda s: L.verify_greedy(t, tok, table, 0.1, stream=s, want_path=True),
    "verify_rows": lambda s: L.verify_rows(t, g, acc, tok, table, 0.1, un, stream=s),
    "verify_greedy_rows": lambda s: L.verify_greedy_rows(t, acc, tok, table, 0.1, stream=s),
    "decide_rows": lambda s: L.decide_rows(t, g, None, tok, table, 0.1, un, stream=s, want_path=True),
    "resample_selected": lambda s: L.resample_selected(t, g, None, tok, table, 0.1, un, acc, stream=s),
    "verify_trees": lambda s: L.verify_trees(t, g, None, parent, M, tok, table, 0.1, un, stream=s),
    "verify_trees_sequential": lambda s: L.verify_trees_sequential(t, g, None, parent, M, tok, table, 0.1, un, stream=s),
    "verify_trees_greedy": lambda s: L.verify_trees_greedy(t, None, parent, M, tok, table, 0.1, stream=s),
    "accept_chains": lambda s: L.accept_chains(acc, acc, M, stream=s),
    "accept_trees": lambda s: L.accept_trees(acc, acc, parent, M, stream=s),
    "build_knn": lambda s: L.build_knn(t, K, stream=s),
    "build_random": lambda s: L.build_random(V, K, 1, device="cpu", stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_another_stream(watched, name):
    """It comes from that stream's memory: what the current stream has freed may still be read by work queued there, which the other does not
    wait for.  Outputs are kept until the current stream has passed the place where they are dropped."""
    side, made, kept = watched
    outs = _tensors(CALLS[name](side))
    assert len(made) == len(outs) + (name in ("verify_trees_sequential", "build_knn")) and all(inside for _, inside in made)
    assert sorted(kept) == sorted((o.data_ptr(), "current") for o in outs)
    made.clear()
    kept.clear()
    CALLS[name](None)
    assert made and all(inside == 0 for _, inside in made) and not kept


@pytest.mark.parametrize("name", CALLS)
def test_the_current_stream_by_name(watched, name):
    """Given the current stream itself a call allocates as it does without one."""
    _, made, kept = watched
    CALLS[name]("current")
    assert made and not any(inside for _, inside in made) and not kept


def test_nothing_to_allocate(watched, monkeypatch):
    """With the caller's outputs the streams are not looked at: such calls are captured and timed."""
    side, made, kept = watched
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: pytest.fail("looked at"))
    L.verify(t, g, tok, table, 0.1, un, out_accept=acc, out_resample=acc, stream=side)
    assert not made and not kept
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "current")
    got = L.verify(t, g, tok, table, 0.1, un, out_resample=acc, stream=side)
    assert len(made) == 1 and made[0][1] and got[1] is acc and got[0].data_ptr() == made[0][0]
    got = L.verify(t, g, tok, table, 0.1, un, out_accept=acc, stream=side)
    assert got[0] is acc and got[1].data_ptr() == made[1][0]
