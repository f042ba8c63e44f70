"""What the Python half of the calls around a tree step does before and around the library's calls, seen on the host: the library is a stand-in
that notes its calls, and tensors of host memory are let through."""
import contextlib

import pytest
import torch

import cache_reference as ref
import paper_2410_03355_amd as L
from paper_2410_03355_amd import binding


class _Library:
    def __init__(self):
        self.called, self.workspace = [], 0

    def __getattr__(self, name):
        def call(*args):
            self.called.append((name, args))
            return self.workspace if name.endswith("_bytes") else binding.OK
        return call


@pytest.fixture
def lib(monkeypatch):
    stand_in = _Library()
    monkeypatch.setattr(binding, "load", lambda: stand_in)
    monkeypatch.setattr(binding, "_marshal", binding._Declines())
    monkeypatch.setattr(binding, "_need_here", lambda *a: None)
    monkeypatch.setattr(binding, "_need_cuda", lambda *a: None)
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)
    return stand_in


def _calls(B=2, T=4, Hq=4, Hk=2, D=32):
    """Arguments of each call that are right."""
    gen = torch.Generator().manual_seed(0)
    cache, table = ref.filled_cache(gen, [20 + 10 * b for b in range(B)], Hk, D, 16, True)
    n = torch.tensor([20 + 10 * b for b in range(B)], dtype=torch.int32)
    q, k, v = (torch.zeros(B, T, h, D) for h in (Hq, Hk, Hk))
    pos, freqs = torch.zeros(B, T, 2, dtype=torch.int32), torch.ones(8)
    return {
        "rotate_axes": dict(q=q.flatten(0, 1), k=k.flatten(0, 1), positions=pos.flatten(0, 1), freqs=freqs, sections=(4, 4)),
        "append_cache": dict(cache=cache, table=table, lengths=n, k=k, v=v, positions=pos, freqs=freqs, sections=(4, 4),
                             path=torch.zeros(B, T - 1, dtype=torch.int32), count=torch.zeros(B, dtype=torch.int32)),
        "attend_trees": dict(q=q, k=k, v=v, parent=torch.zeros(B * (T - 1), dtype=torch.int32), cache=cache, table=table, lengths=n),
    }


@pytest.mark.parametrize("name", ["rotate_axes", "append_cache", "attend_trees"])
def test_memory_of_another_stream(lib, monkeypatch, name):
    """With a stream of the caller's, outputs and workspace come from that stream's memory: what the current stream has freed may still be
    read by work that is queued there and that the other stream does not wait for.  Outputs are not given away again before the
    current stream, which reads them, has passed the place where they are dropped."""
    kw, side, state = _calls()[name], object(), {"inside": 0}
    made, kept = [], []

    @contextlib.contextmanager
    def on(stream):
        assert stream is side
        state["inside"] += 1
        yield
        state["inside"] -= 1

    empty = torch.empty

    def noted(*args, **kwargs):
        t = empty(*args, **kwargs)
        made.append((t.data_ptr(), state["inside"]))
        return t

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: "current")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t.data_ptr(), s)))
    monkeypatch.setattr(torch, "empty", noted)
    lib.workspace = 4096
    got = getattr(L, name)(**kw, stream=side)
    outs = got if isinstance(got, tuple) else (got,)
    assert len(made) == len(outs) + (name == "attend_trees") and all(inside for _, inside in made)
    assert all((o.data_ptr(), "current") in kept for o in outs)
    made.clear()
    kept.clear()
    getattr(L, name)(**kw)
    assert all(inside == 0 for _, inside in made) and not kept


FLOATS = {"rotate_axes": ("q", "k", "freqs"), "append_cache": ("k", "v", "freqs"), "attend_trees": ("q", "k", "v")}


@pytest.mark.parametrize("name,which", [(n, w) for n, ws in FLOATS.items() for w in ws])
def test_tangents_are_refused(lib, name, which):
    """A dual tensor would come back without its tangent."""
    kw = _calls()[name]
    with torch.autograd.forward_ad.dual_level():
        plain, kw[which] = kw[which], torch.autograd.forward_ad.make_dual(kw[which], torch.ones_like(kw[which]))
        with pytest.raises(ValueError, match="forward-mode"):
            getattr(L, name)(**kw)
        getattr(L, name)(**{**kw, which: plain})
        with torch.autograd.forward_ad._set_fwd_grad_enabled(False):
            getattr(L, name)(**kw)


@pytest.mark.parametrize("name", ["append_cache", "attend_trees"])
@pytest.mark.parametrize("i,eight", [(0, False), (1, False), (2, True), (3, True)])
def test_a_cache_that_wants_gradients(lib, name, i, eight):
    """Keys, values and scales of a cache have none either: refused where they are recorded, served where nothing is."""
    kw = _calls()[name]
    cache = list(kw["cache"]) if eight else list(L.make_cache(9, 2, 16, 32, torch.bfloat16, "cpu"))
    cache[i] = cache[i].detach().clone().requires_grad_()
    kw["cache"] = tuple(cache)
    with pytest.raises(ValueError, match="no backward pass"):
        getattr(L, name)(**kw)
    assert not any(n == "lantern_" + name for n, _ in lib.called)
    with torch.no_grad():
        getattr(L, name)(**kw)
    assert any(n == "lantern_" + name for n, _ in lib.called)


def test_freqs_that_want_gradients(lib):
    kw = _calls()["append_cache"]
    kw["freqs"] = kw["freqs"].clone().requires_grad_()
    with pytest.raises(ValueError, match="no backward pass"):
        L.append_cache(**kw)
    with torch.no_grad():
        L.append_cache(**kw)


def test_a_path_without_candidates(lib):
    """An empty path has no address, which the library takes for none: the first count rows, none of them, in the place of row 0."""
    kw = _calls(T=1)["append_cache"]
    assert kw["path"].numel() == 0 and kw["path"].data_ptr() == 0
    with pytest.raises(ValueError, match="rows for its candidates"):
        L.append_cache(**kw)
    assert not lib.called
    L.append_cache(**{**kw, "path": None})


def _far(*size, dtype=torch.float32):
    return torch.empty(size, dtype=dtype, device="meta")


FAR = (1 << 32) + 1      # one, when it is cut off to 32 bits
BEYOND = [("rotate_axes", dict(q=_far(FAR, 1, 32), k=None, positions=_far(FAR, 2, dtype=torch.int32))),
          ("rotate_axes", dict(q=_far(8, FAR, 32))), ("rotate_axes", dict(k=_far(8, FAR, 32))), ("rotate_axes", dict(q=_far(8, 1, FAR), k=None)),
          ("rotate_axes", dict(sections=((1 << 32) + 16, -(1 << 32) - 8))),
          ("append_cache", dict(k=_far(2, FAR, 2, 32), v=_far(2, FAR, 2, 32), positions=None, path=None, count=None)),
          ("append_cache", dict(table=_far(2, FAR, dtype=torch.int32))),
          ("append_cache", dict(cache=(_far(FAR, 2, 16, 32, dtype=torch.bfloat16), _far(FAR, 2, 32, 16, dtype=torch.bfloat16), None, None))),
          ("attend_trees", dict(cache=(_far(9, 2, FAR + 15, 32, dtype=torch.bfloat16), _far(9, 2, 32, FAR + 15, dtype=torch.bfloat16), None, None))),
          ("attend_trees", dict(q=_far(2, FAR, 4, 32), k=_far(2, FAR, 2, 32), v=_far(2, FAR, 2, 32), parent=None)),
          ("attend_trees", dict(q=_far(2, 4, FAR + 1, 32))), ("attend_trees", dict(table=_far(2, FAR, dtype=torch.int32)))]


@pytest.mark.parametrize("i", range(len(BEYOND)))
def test_sizes_beyond_32_bits(lib, i):
    """They would be cut off on their way to the library and serve a part of the call."""
    name, kw = BEYOND[i]
    with pytest.raises(ValueError, match="fit 32 bits"):
        getattr(L, name)(**{**_calls()[name], **kw})
    assert not lib.called


def test_workspace_of_sizes_beyond_32_bits(lib):
    cache = _calls()["attend_trees"]["cache"]
    for sizes in ((FAR, 5, 8, 400), (1, FAR, 8, 400), (1, 5, FAR + 7, 400), (1, 5, 8, FAR)):
        with pytest.raises(ValueError, match="fit 32 bits"):
            L.attend_trees_workspace_bytes(torch.bfloat16, *sizes[:3], cache, sizes[3])
    assert not lib.called


def _saved(t):
    """A result whose backward pass wants `t` as it is."""
    return (torch.ones((), requires_grad=True) * t).sum()


def test_written_tensors_have_a_new_version(lib):
    """What a call writes in place may have been saved for a backward pass, which has to notice."""
    kw = _calls()["rotate_axes"]
    later = [_saved(kw["q"]), _saved(kw["k"])]
    L.rotate_axes(**kw)
    assert kw["q"]._version == 0 and kw["positions"]._version == 0
    L.rotate_axes(**kw, out=(kw["q"], kw["k"]))
    for y in later:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    kw = _calls()["append_cache"]
    versions = [t._version for t in kw["cache"]]
    L.append_cache(**kw)
    assert [t._version for t in kw["cache"]] == [n + 1 for n in versions]
    with torch.inference_mode():      # tensors without versions
        kw = _calls()["append_cache"]
        L.append_cache(**kw)
        kw = _calls()["rotate_axes"]
        L.rotate_axes(**kw, out=(kw["q"], kw["k"]))


def test_outputs_that_want_gradients(lib):
    kw = _calls()["rotate_axes"]
    out = kw["q"].clone().requires_grad_(), kw["k"].clone()
    with pytest.raises(ValueError, match="gradients are recorded"):
        L.rotate_axes(**kw, out=out)
    assert not lib.called
    with torch.no_grad():
        L.rotate_axes(**kw, out=out)
