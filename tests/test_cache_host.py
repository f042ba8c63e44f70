"""Refusals of the calls around a tree step: all on the host, before anything is launched (pointers here are never followed)."""
import ctypes
import os

import pytest
import torch

import cache_reference as ref
import paper_2410_03355_amd as L
from paper_2410_03355_amd import binding as B_


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        L.build()
    return L.load()


P = 4096
NUL = None


def _cache(**kw):
    c = dict(k=P, v=P, k_scale=P, v_scale=P, dtype=L.E4M3, pages=9, heads=4, page_tokens=64, D=64)
    c.update(kw)
    return B_._Cache(*c.values())


def _rotation(positions=P, freqs=P, axes=2, pairs=(16, 16, 0, 0), interleaved=0):
    return B_._Rotation(positions, freqs, axes, (ctypes.c_int * 4)(*pairs), interleaved)


S2, S3 = B_._strides(256, 64), B_._strides(8192, 256, 64)
BAD_CACHES = [(dict(dtype=L.F32), "E_DTYPE"), (dict(dtype=7), "E_DTYPE"), (dict(pages=0), "E_SHAPE"), (dict(heads=0), "E_SHAPE"),
              (dict(heads=65536), "E_SHAPE"), (dict(page_tokens=8), "E_SHAPE"), (dict(page_tokens=48), "E_SHAPE"), (dict(page_tokens=256), "E_SHAPE"),
              (dict(D=16), "E_SHAPE"), (dict(D=80), "E_SHAPE"), (dict(D=256), "E_SHAPE"), (dict(k=None), "E_NULL"), (dict(v=None), "E_NULL"),
              (dict(k_scale=None), "E_NULL"), (dict(v_scale=None), "E_NULL"), (dict(k=P + 8), "E_SHAPE"), (dict(v=P + 2), "E_SHAPE")]


def test_rotate_refusals(lib):
    def call(q=P, qs=S2, qh=4, k=P, ks=S2, kh=2, dtype=L.F32, N=3, D=64, rot=_rotation(), oq=P, oqs=S2, ok=P, oks=S2):
        return lib.lantern_rotate_axes(q, qs, qh, k, ks, kh, dtype, N, D, None if rot is None else ctypes.byref(rot), 0, oq, oqs, ok, oks, NUL)

    assert call(dtype=L.E4M3) == B_.E_DTYPE and call(dtype=5) == B_.E_DTYPE
    for kw in (dict(N=-1), dict(qh=0), dict(kh=-1), dict(D=1), dict(D=1025), dict(qh=2 ** 31 - 1), dict(D=62), dict(rot=_rotation(axes=0)),
               dict(rot=_rotation(axes=5)), dict(rot=_rotation(pairs=(0, 0, 9, 9))), dict(rot=_rotation(pairs=(-1, 9, 0, 0))),
               dict(rot=_rotation(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 0, 0))), dict(rot=_rotation(pairs=(17, 16, 0, 0)))):
        assert call(**kw) == B_.E_SHAPE, kw
    for kw in (dict(q=NUL), dict(qs=NUL), dict(oq=NUL), dict(oqs=NUL), dict(k=NUL), dict(ks=NUL), dict(ok=NUL), dict(oks=NUL), dict(rot=None),
               dict(rot=_rotation(positions=None)), dict(rot=_rotation(freqs=None))):
        assert call(**kw) == B_.E_NULL, kw
    assert call(N=0, q=NUL, rot=None) == B_.OK


def test_append_refusals(lib):
    def call(cache=_cache(), table=P, width=9, lengths=P, B=2, T=5, k=P, ks=S3, v=P, vs=S3, dtype=L.BF16, rot=None, path=NUL, count=NUL, out=P + 64):
        return lib.lantern_append_cache(None if cache is None else ctypes.byref(cache), table, width, lengths, B, T, k, ks, v, vs, dtype,
                                        None if rot is None else ctypes.byref(rot), path, count, out, NUL)

    for kw, status in BAD_CACHES:
        assert call(cache=_cache(**kw)) == getattr(B_, status), kw
    assert call(dtype=L.E4M3) == B_.E_DTYPE
    for kw in (dict(B=-1), dict(T=0), dict(width=0), dict(width=2 ** 25), dict(path=P, count=P, T=1), dict(out=P), dict(B=2 ** 30, T=2 ** 12),
               dict(rot=_rotation(pairs=(16, 17, 0, 0)))):
        assert call(**kw) == B_.E_SHAPE, kw
    for kw in (dict(cache=None), dict(table=NUL), dict(lengths=NUL), dict(k=NUL), dict(v=NUL), dict(ks=NUL), dict(vs=NUL), dict(out=NUL), dict(path=P),
               dict(rot=_rotation(positions=None))):
        assert call(**kw) == B_.E_NULL, kw
    assert call(B=0, table=NUL, k=NUL) == B_.OK


def test_attend_refusals(lib):
    def call(q=P, qs=S3, k=P, ks=S3, v=P, vs=S3, dtype=L.BF16, B=2, M=5, Hq=8, parent=P, cache=_cache(), table=P, width=9, lengths=P, scale=0.125, out=P,
             ws=P, ws_bytes=1 << 40):
        return lib.lantern_attend_trees(q, qs, k, ks, v, vs, dtype, B, M, Hq, parent, None if cache is None else ctypes.byref(cache), table, width,
                                        lengths, scale, out, ws, ws_bytes, NUL)

    for kw, status in BAD_CACHES:
        assert call(cache=_cache(**kw)) == getattr(B_, status), kw
    assert call(dtype=L.E4M3) == B_.E_DTYPE
    for kw in (dict(B=-1), dict(M=-1), dict(M=L.MAX_TREE + 1), dict(Hq=0), dict(Hq=-4), dict(Hq=6), dict(width=0), dict(width=2 ** 25),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-1.0), dict(scale=3e38), dict(B=2 ** 28, M=255),
               dict(B=2 ** 22)):      # 2^24 workgroups
        assert call(**kw) == B_.E_SHAPE, kw
    for kw in (dict(cache=None), dict(q=NUL), dict(qs=NUL), dict(k=NUL), dict(ks=NUL), dict(v=NUL), dict(vs=NUL), dict(table=NUL), dict(lengths=NUL),
               dict(out=NUL)):
        assert call(**kw) == B_.E_NULL, kw
    assert call(B=0, q=NUL, ws=NUL, ws_bytes=0) == B_.OK
    size = lib.lantern_attend_trees_workspace_bytes
    need = size(L.BF16, 1, 5, 8, ctypes.byref(_cache()), 400)
    assert need > 0
    for kw in (dict(ws=NUL), dict(ws=P + 64), dict(ws_bytes=need - 1)):
        assert call(B=1, width=400, **kw) == B_.E_WORKSPACE, kw
    assert size(L.E4M3, 1, 5, 8, ctypes.byref(_cache()), 400) == 0 and size(L.BF16, 1, 5, 7, ctypes.byref(_cache()), 400) == 0
    assert size(L.BF16, 0, 5, 8, ctypes.byref(_cache()), 400) == 0


def test_prepare_refusals(lib):
    assert lib.lantern_prepare_cache(L.E4M3, ctypes.byref(_cache())) == B_.E_DTYPE
    assert lib.lantern_prepare_cache(L.BF16, ctypes.byref(_cache(D=8))) == B_.E_SHAPE
    assert lib.lantern_prepare_cache(L.BF16, None) == B_.E_NULL


def test_binding_refusals():
    """Python's checks come before the library's; host tensors are refused."""
    gen = torch.Generator().manual_seed(0)
    cache, table = ref.filled_cache(gen, [20, 30], 2, 32, 16, True)
    n = torch.tensor([20, 30], dtype=torch.int32)
    q, k, v = (torch.zeros(2, 4, h, 32) for h in (4, 2, 2))
    parent = torch.zeros(6, dtype=torch.int32)
    pos, freqs = torch.zeros(2, 4, 2, dtype=torch.int32), torch.ones(8)
    bad = [
        lambda: L.rotate_axes(q[0], k[0], pos[0], freqs, (4, 4)),                    # host memory
        lambda: L.rotate_axes(q[0], k[1].half(), pos[0], freqs, (4, 4)),
        lambda: L.rotate_axes(q, k, pos, freqs, (4, 4)),
        lambda: L.rotate_axes(q[0], k[0, :3], pos[0], freqs, (4, 4)),
        lambda: L.append_cache(cache, table, n, k, v),
        lambda: L.append_cache(cache, table, n, q, v),
        lambda: L.append_cache(cache, table.long(), n, k, v),
        lambda: L.append_cache(cache, table[:1], n, k, v),
        lambda: L.append_cache(cache, table, n, k, v, positions=pos),
        lambda: L.append_cache(cache, table, n, k, v, positions=pos, freqs=freqs, sections=(4, 3)),
        lambda: L.append_cache(cache, table, n, k, v, positions=pos[:, :3], freqs=freqs, sections=(4, 4)),
        lambda: L.append_cache(cache, table, n, k, v, path=torch.zeros(2, 3, dtype=torch.int32)),
        lambda: L.append_cache(cache, table, n, k, v, path=torch.zeros(2, 4, dtype=torch.int32), count=n),
        lambda: L.append_cache((cache[0], cache[1].transpose(2, 3), *cache[2:]), table, n, k, v),
        lambda: L.append_cache((cache[0], cache[1], None, cache[3]), table, n, k, v),
        lambda: L.append_cache((cache[0].float(), cache[1].float(), None, None), table, n, k, v),
        lambda: L.attend_trees(q, k, v, parent, cache, table, n),
        lambda: L.attend_trees(q, k, v, parent[:5], cache, table, n),
        lambda: L.attend_trees(q[..., :16], k, v, parent, cache, table, n),
        lambda: L.attend_trees(q[:, :3], k, v, parent, cache, table, n),
        lambda: L.attend_trees(q.bfloat16(), k, v, parent, cache, table, n),
        lambda: L.make_cache(4, 2, 16, 32, dtype=torch.float16, device="cpu"),
        lambda: L.make_cache(4, 2, 24, 32, device="cpu"),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            f()
            print("not refused:", i)
    c = L.make_cache(4, 2, 16, 32, device="cpu")
    assert c.v.shape == (4, 2, 32, 16) and c.k.dtype == torch.float8_e4m3fn and L.make_cache(4, 2, 16, 32, torch.bfloat16, "cpu").k_scale is None


def test_gradients_that_are_not_formed():
    """Recorded inputs are refused where there is no backward pass, before anything else is done with them."""
    cache, table = ref.filled_cache(torch.Generator().manual_seed(0), [20], 2, 32, 16, True)
    n = torch.tensor([20], dtype=torch.int32)
    x, leaf = torch.zeros(1, 1, 2, 32), torch.zeros(1, 1, 2, 32, requires_grad=True)
    pos, freqs = torch.zeros(1, 2, dtype=torch.int32), torch.ones(8)
    for f in (lambda: L.attend_trees(leaf, x, x, None, cache, table, n), lambda: L.attend_trees(x, leaf, x, None, cache, table, n),
              lambda: L.append_cache(cache, table, n, x, leaf)):
        with pytest.raises(ValueError, match="no backward pass"):
            f()
    for kw in (dict(out=(leaf[0], None)), dict(freqs=freqs.clone().requires_grad_())):
        with pytest.raises(ValueError, match="gradients are recorded"):
            L.rotate_axes(leaf[0], None, pos, kw.pop("freqs", freqs), (4, 4), **kw)


def test_a_workspace_with_gaps():
    cache, table = ref.filled_cache(torch.Generator().manual_seed(0), [20], 2, 32, 16, True)
    x = torch.zeros(1, 1, 2, 32)
    with pytest.raises(ValueError, match="contiguous"):
        L.attend_trees(x, x, x, None, cache, table, torch.tensor([20], dtype=torch.int32), workspace=torch.zeros(512, dtype=torch.uint8)[::2])


def test_workspace_shrinks_with_enough_sequences(lib):
    """Sequences are split only while there are too few of them to fill the device."""
    cache = (torch.zeros(4, 20, 64, 64, dtype=torch.bfloat16), torch.zeros(4, 20, 64, 64, dtype=torch.bfloat16), None, None)
    assert L.attend_trees_workspace_bytes(torch.bfloat16, 64, 60, 20, cache, 12) == 0
    one = L.attend_trees_workspace_bytes(torch.bfloat16, 1, 0, 20, cache, 512)
    assert one % (20 * 66 * 4) == 8 and one > 8      # and where the sequence is cut
