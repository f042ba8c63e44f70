"""Derivatives that the calls around a tree step do not form are refused by the native half too."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


def _calls(lantern, eight):
    gen = torch.Generator().manual_seed(8)
    B, T, Hq, Hk, D = 2, 3, 4, 2, 32
    cache, table = ref.filled_cache(gen, [20, 30], Hk, D, 16, eight, rubbish=False)
    q, k, v = (ref.normal(gen, B, T, h, D).cuda() for h in (Hq, Hk, Hk))
    pos, freqs = torch.zeros(B, T, 1, dtype=torch.int32).cuda(), torch.rand(8, generator=gen).cuda()
    n, table, cache = torch.tensor([20, 30], dtype=torch.int32).cuda(), table.cuda(), ref.on_gpu(cache)
    return {
        "rotate_axes": ([q.flatten(0, 1), k.flatten(0, 1), pos.flatten(0, 1), freqs, (8,)], (0, 1, 3)),
        "append_cache": ([cache, table, n, k, v, pos, freqs, (8,)], (3, 4, 6)),
        "attend_trees": ([q, k, v, None, cache, table, n], (0, 1, 2)),
    }


@pytest.mark.parametrize("name", ["rotate_axes", "append_cache", "attend_trees"])
def test_tangents_are_refused(lantern_gpu, name):
    args, floats = _calls(lantern_gpu, True)[name]
    with torch.autograd.forward_ad.dual_level():
        for i in floats:
            dual = list(args)
            dual[i] = torch.autograd.forward_ad.make_dual(args[i], torch.ones_like(args[i]))
            with pytest.raises(ValueError, match="forward-mode"):
                getattr(lantern_gpu, name)(*dual)
        getattr(lantern_gpu, name)(*args)


@pytest.mark.parametrize("eight", [True, False])
def test_a_cache_that_wants_gradients(lantern_gpu, eight):
    for name, at in (("attend_trees", 4), ("append_cache", 0)):
        args, _ = _calls(lantern_gpu, eight)[name]
        want = getattr(lantern_gpu, name)(*args)
        for i in (2, 3) if eight else (0, 1):
            cache = [t if t is None else t.clone() for t in _calls(lantern_gpu, eight)[name][0][at]]
            cache[i].requires_grad_()
            args[at] = tuple(cache)
            with pytest.raises(ValueError, match="no backward pass"):
                getattr(lantern_gpu, name)(*args)
            with torch.no_grad():
                assert torch.equal(getattr(lantern_gpu, name)(*args), want)


@pytest.mark.parametrize("eight", [True, False])
def test_written_tensors_have_a_new_version(lantern_gpu, eight):
    calls = _calls(lantern_gpu, eight)
    args, _ = calls["append_cache"]
    cache = [t for t in args[0] if t is not None]
    versions = [t._version for t in cache]
    lantern_gpu.append_cache(*args)
    assert [t._version for t in cache] == [n + 1 for n in versions]
    args, _ = calls["rotate_axes"]
    q, k = args[0].clone(), args[1].clone()
    later = (torch.ones((), device="cuda", requires_grad=True) * q).sum()
    lantern_gpu.rotate_axes(q, k, *args[2:], out=(q, k))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        later.backward()
    with torch.inference_mode():
        args, _ = _calls(lantern_gpu, eight)["append_cache"]
        lantern_gpu.append_cache(*args)
