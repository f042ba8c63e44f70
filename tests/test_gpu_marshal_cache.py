"""The host half of rotate_axes, append_cache and attend_trees in native code against the way through ctypes: same results for ordinary
calls; declined, and refused or served by Python, what is not one."""
import pytest
import torch

import cache_reference as ref
from paper_2410_03355_amd import binding

pytestmark = pytest.mark.gpu


class _Declines:
    def __getattr__(self, name):
        return lambda *args: None


def _calls(eight, dtype):
    gen = torch.Generator().manual_seed(4)
    B, T, Hq, Hk, D, page = 2, 6, 4, 2, 64, 32
    cache, table = ref.filled_cache(gen, [40, 70], Hk, D, page, eight, rubbish=False)
    heads = ref.normal(gen, B, T, Hq + 2 * Hk, D).to(dtype).cuda()
    q, k, v = heads.split((Hq, Hk, Hk), 2)
    pos = torch.randint(0, 50, (B, T, 2), generator=gen, dtype=torch.int32).cuda()
    freqs, n = torch.rand(20, generator=gen).cuda(), torch.tensor([40, 70], dtype=torch.int32).cuda()
    path = torch.tensor([[0, 2, -1, -1, -1], [1, -1, -1, -1, -1]], dtype=torch.int32).cuda()
    some = torch.tensor([2, 1], dtype=torch.int32).cuda()
    on = ref.on_gpu(cache)
    return on, {
        "rotate_axes": (q.flatten(0, 1), k.flatten(0, 1), pos.flatten(0, 1), freqs, (12, 8), True, False),
        "attend_trees": (q, k, v, ref.tree(gen, B, T - 1).cuda(), on, table.cuda(), n, None, None),
        "append_cache": (on, table.cuda(), n, k, v, pos, freqs, (12, 8), False, path, some),
    }


def _same(a, b):
    a, b = (x if isinstance(x, tuple) else (x,) for x in (a, b))
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_same_results(lantern_gpu, monkeypatch, eight, dtype):
    cache, calls = _calls(eight, dtype)
    start = [None if t is None else t.clone() for t in cache]
    for name, args in calls.items():
        states, outs = [], []
        for general in (False, True):
            for t, s in zip(cache, start):
                if t is not None:
                    t.copy_(s)
            with monkeypatch.context() as m:
                if general:
                    m.setattr(binding, "_marshal", _Declines())
                else:
                    native = getattr(binding._marshal, name)(*args)
                    assert native is not None and native.__class__ is not int, name
                    for t, s in zip(cache, start):
                        if t is not None:
                            t.copy_(s)
                outs.append(getattr(lantern_gpu, name)(*args) if name != "rotate_axes" else lantern_gpu.rotate_axes(*args))
            states.append([None if t is None else t.view(torch.uint8).clone() for t in cache])
        assert _same(*outs), name
        assert all(a is None or torch.equal(a, b) for a, b in zip(*states)), name


def test_declined(lantern_gpu):
    cache, calls = _calls(True, torch.bfloat16)
    m = binding._marshal

    def swapped(name, i, x):
        args = list(calls[name])
        args[i] = x
        return getattr(m, name)(*args)

    q = calls["attend_trees"][0]
    assert swapped("attend_trees", 0, q.half()) is None and swapped("attend_trees", 0, q[..., :32]) is None
    assert swapped("attend_trees", 0, q.cpu()) is None and swapped("attend_trees", 4, list(cache)) is None
    assert swapped("attend_trees", 4, (cache[0], cache[1], None, cache[3])) is None
    assert swapped("attend_trees", 5, calls["attend_trees"][5].long()) is None
    assert swapped("attend_trees", 0, q[:, :, :3]) == binding.E_SHAPE          # three heads over two: the library's own refusal
    with pytest.raises(lantern_gpu.LanternError):
        lantern_gpu.attend_trees(q[:, :, :3], *calls["attend_trees"][1:])
    assert swapped("append_cache", 10, None) is None and swapped("append_cache", 7, (12, 7)) is None
    assert swapped("append_cache", 3, calls["append_cache"][3].transpose(2, 3)) is None
    assert swapped("rotate_axes", 4, [12, 8]) is None and swapped("rotate_axes", 1, None) is None
    a, b = lantern_gpu.rotate_axes(*calls["rotate_axes"][:4], [12, 8], True)       # a list of sections goes the general way
    c, d = lantern_gpu.rotate_axes(*calls["rotate_axes"])
    assert torch.equal(a, c) and torch.equal(b, d)


def test_a_path_without_candidates(lantern_gpu):
    """An empty path has no address: declined, and refused by Python."""
    cache, calls = _calls(True, torch.bfloat16)
    args = list(calls["append_cache"])
    args[3:6] = [x[:, :1].contiguous() for x in args[3:6]]
    args[9] = args[9][:, :0].contiguous()
    before = cache[0].view(torch.uint8).clone()
    assert binding._marshal.append_cache(*args) is None
    with pytest.raises(ValueError, match="rows for its candidates"):
        lantern_gpu.append_cache(*args)
    assert torch.equal(cache[0].view(torch.uint8), before)
