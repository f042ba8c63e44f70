"""Every check that Python makes of the calls around a tree step, one call for each part of it: what would have the kernels read or write out of
range, or take memory for what it is not, is refused with its own words before the library is called.  The library is a stand-in here and tensors
of host memory are let through, so nothing else refuses these calls."""
import pytest
import torch

import paper_2410_03355_amd as L
from paper_2410_03355_amd import binding
from test_cache_binding import _calls, lib  # noqa: F401

HEADS_3 = "q and k must be [N, heads, D]"
POSITIONS = "positions must be contiguous"
GRADIENTS = "gradients are recorded without out and stream"
OUT = "out must hold tensors like q and k"
ROWS = "k and v must be [B, rows, heads, D]"
TABLE = "table must be contiguous"
CACHE = "the cache must be two contiguous tensors"
ALIKE = "the cache's keys and values must have the same"
SCALES = "an 8-bit cache needs k_scale and v_scale"
PATH = "path must be a contiguous int32"
QUERY = "q must be [B, rows, heads, D] like k and v"


def _gaps(t):
    """The same sizes and values with gaps between its elements."""
    return torch.stack([t, t], -1)[..., 0]


def _swap(a, i, t):
    return tuple(t(x) if j == i else x for j, x in enumerate(a))


ROTATE = [
    (lambda c: dict(q=c["q"][0], k=None), ValueError, HEADS_3), (lambda c: dict(k=c["k"][:, 0]), ValueError, HEADS_3),
    (lambda c: dict(k=c["k"][:5]), ValueError, HEADS_3), (lambda c: dict(k=c["k"][..., :16].contiguous()), ValueError, HEADS_3),
    (lambda c: dict(k=c["k"].bfloat16()), ValueError, HEADS_3), (lambda c: dict(q=_gaps(c["q"])), ValueError, HEADS_3),
    (lambda c: dict(k=_gaps(c["k"])), ValueError, HEADS_3),
    (lambda c: dict(q=c["q"].half(), k=c["k"].half()), TypeError, "unsupported dtype"),
    (lambda c: dict(positions=c["positions"].long()), TypeError, "positions must be int32"),
    (lambda c: dict(freqs=c["freqs"].double()), TypeError, "positions must be int32"),
    (lambda c: dict(sections=(), positions=c["positions"][:0], freqs=c["freqs"][:0]), ValueError, POSITIONS),
    (lambda c: dict(sections=(1, 1, 2, 2, 2), positions=torch.zeros(8, 5, dtype=torch.int32, device=c["q"].device)), ValueError, POSITIONS),
    (lambda c: dict(positions=c["positions"][:7]), ValueError, POSITIONS), (lambda c: dict(sections=(4, 2, 2)), ValueError, POSITIONS),
    (lambda c: dict(freqs=c["freqs"][:7]), ValueError, POSITIONS), (lambda c: dict(sections=(4, 5)), ValueError, POSITIONS),
    (lambda c: dict(positions=_gaps(c["positions"])), ValueError, POSITIONS), (lambda c: dict(freqs=_gaps(c["freqs"])), ValueError, POSITIONS),
    (lambda c: dict(out=(c["q"], None)), ValueError, OUT), (lambda c: dict(out=(c["q"][:7], c["k"])), ValueError, OUT),
    (lambda c: dict(out=(c["q"], c["k"][:, :1])), ValueError, OUT), (lambda c: dict(out=(c["q"].bfloat16(), c["k"])), ValueError, OUT),
    (lambda c: dict(out=(c["q"], _gaps(c["k"]))), ValueError, OUT), (lambda c: dict(k=None, out=(c["q"], c["k"])), ValueError, OUT),
    (lambda c: dict(q=c["q"].requires_grad_(), stream=object()), ValueError, GRADIENTS),
    (lambda c: dict(freqs=c["freqs"].requires_grad_()), ValueError, GRADIENTS),
    (lambda c: dict(k=c["k"].requires_grad_(), out=(c["q"], c["k"].detach())), ValueError, GRADIENTS),
]
CACHES = [
    (lambda c: dict(cache=_swap(c["cache"], 0, lambda t: t[0])), ValueError, CACHE), (lambda c: dict(cache=_swap(c["cache"], 1, lambda t: t[0])), ValueError, CACHE),
    (lambda c: dict(cache=_swap(c["cache"], 0, _gaps)), ValueError, CACHE), (lambda c: dict(cache=_swap(c["cache"], 1, _gaps)), ValueError, CACHE),
    (lambda c: dict(cache=_swap(c["cache"], 1, lambda t: t[1:].contiguous())), ValueError, ALIKE),
    (lambda c: dict(cache=_swap(c["cache"], 1, lambda t: t.transpose(2, 3).contiguous())), ValueError, ALIKE),
    (lambda c: dict(cache=_swap(c["cache"], 1, lambda t: t.float().bfloat16())), ValueError, ALIKE),
    (lambda c: dict(cache=_swap(_swap(c["cache"], 0, lambda t: t.float()), 1, lambda t: t.float())), TypeError, "a cache is bfloat16 or"),
] + [(lambda c, i=i, f=f: dict(cache=_swap(c["cache"], i, f)), ValueError, SCALES) for i in (2, 3) for f in (
    lambda t: None, lambda t: t.double(), lambda t: t[1:], lambda t: t[:, :1].contiguous(), _gaps)]
KEPT = [
    (lambda c: dict(k=c["k"][..., None], v=c["v"][..., None]), ValueError, ROWS), (lambda c: dict(v=c["v"][:, :3]), ValueError, ROWS), (lambda c: dict(v=c["v"].bfloat16()), ValueError, ROWS),
    (lambda c: dict(k=c["k"][:, :, :1], v=c["v"][:, :, :1]), ValueError, ROWS), (lambda c: dict(k=c["k"][..., :16], v=c["v"][..., :16]), ValueError, ROWS),
    (lambda c: dict(k=_gaps(c["k"])), ValueError, ROWS), (lambda c: dict(v=_gaps(c["v"])), ValueError, ROWS),
    (lambda c: dict(table=c["table"].long()), TypeError, "table and lengths must be int32"),
    (lambda c: dict(lengths=c["lengths"].long()), TypeError, "table and lengths must be int32"),
    (lambda c: dict(table=c["table"][0]), ValueError, TABLE), (lambda c: dict(table=c["table"][:1]), ValueError, TABLE),
    (lambda c: dict(table=c["table"][:, :0]), ValueError, TABLE), (lambda c: dict(lengths=c["lengths"][:1]), ValueError, TABLE),
    (lambda c: dict(table=_gaps(c["table"])), ValueError, TABLE), (lambda c: dict(lengths=_gaps(c["lengths"])), ValueError, TABLE),
]
APPEND = CACHES + KEPT + [
    (lambda c: dict(k=c["k"].half(), v=c["v"].half()), TypeError, "unsupported dtype"),
    (lambda c: dict(freqs=None), ValueError, "positions come with"), (lambda c: dict(sections=None), ValueError, "positions come with"),
    (lambda c: dict(positions=c["positions"][:, :3].contiguous()), ValueError, POSITIONS),
    (lambda c: dict(path=c["path"].long()), ValueError, PATH), (lambda c: dict(path=c["path"][:, :2].contiguous()), ValueError, PATH),
    (lambda c: dict(path=_gaps(c["path"])), ValueError, PATH), (lambda c: dict(count=c["count"].long()), ValueError, PATH),
    (lambda c: dict(count=c["count"][:1]), ValueError, PATH), (lambda c: dict(count=_gaps(c["count"])), ValueError, PATH),
    (lambda c: dict(count=None), ValueError, "path comes with count"),
]
PARENT = "parent must be a contiguous int32"
ATTEND = CACHES + KEPT + [
    (lambda c: dict(q=c["q"].half(), k=c["k"].half(), v=c["v"].half()), TypeError, "unsupported dtype"),
    (lambda c: dict(q=c["q"][..., None]), ValueError, QUERY), (lambda c: dict(q=c["q"][:1]), ValueError, QUERY), (lambda c: dict(q=c["q"][:, :3]), ValueError, QUERY),
    (lambda c: dict(q=c["q"][..., :16]), ValueError, QUERY), (lambda c: dict(q=c["q"].bfloat16()), ValueError, QUERY), (lambda c: dict(q=_gaps(c["q"])), ValueError, QUERY),
    (lambda c: dict(parent=c["parent"].long()), ValueError, PARENT), (lambda c: dict(parent=c["parent"][:5]), ValueError, PARENT),
    (lambda c: dict(parent=_gaps(c["parent"])), ValueError, PARENT),
    (lambda c: dict(workspace=torch.zeros(512, dtype=torch.uint8, device=c["q"].device)[::2]), ValueError, "workspace must be contiguous"),
]
REFUSED = {"rotate_axes": ROTATE, "append_cache": APPEND, "attend_trees": ATTEND}
ALL = [(name, i) for name, calls in REFUSED.items() for i in range(len(calls))]


@pytest.mark.parametrize("name", ["rotate_axes", "append_cache", "attend_trees"])
def test_the_right_call_goes_through(lib, name):  # noqa: F811
    getattr(L, name)(**_calls()[name])
    assert lib.called[-1][0] == "lantern_" + name


@pytest.mark.parametrize("name,i", ALL)
def test_refused(lib, name, i):  # noqa: F811
    change, kind, words = REFUSED[name][i]
    kw = _calls()[name]
    with pytest.raises(kind) as e:
        getattr(L, name)(**{**kw, **change(kw)})
    assert words in str(e.value), str(e.value)
    assert not lib.called


def test_host_memory():
    """With the checks of the memory in force right calls are refused for it."""
    for name, kw in _calls().items():
        with pytest.raises(ValueError, match="device memory"):
            getattr(L, name)(**kw)


class _Stream:
    def __init__(self, index):
        self.device = torch.device("cuda", index)


def test_other_devices(monkeypatch):
    """Tensors of another device than the current one, and streams of one, are refused: the kernels are launched on the current device."""
    class There:
        is_cuda = True

        def __init__(self, index):
            self.device = torch.device("cuda", index)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    binding._need_here(None, There(0), None)
    binding._need_here(_Stream(0), There(0))
    for stream, tensors in ((None, (There(0), There(1))), (_Stream(1), (There(0),)), (None, (There(1),))):
        with pytest.raises(ValueError, match="current device"):
            binding._need_here(stream, *tensors)


@pytest.mark.parametrize("args,kind", [((4, 2, 16, 32, torch.float16), TypeError), ((4, 2, 16, 32, torch.float32), TypeError), ((4, 2, 24, 32), ValueError),
                                       ((4, 2, 16, 40), ValueError), ((0, 2, 16, 32), ValueError), ((4, 0, 16, 32), ValueError)])
def test_make_cache(args, kind):
    with pytest.raises(kind, match="a cache is|page_tokens must be"):
        L.make_cache(*args, device="cpu")
