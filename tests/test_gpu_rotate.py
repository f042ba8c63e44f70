"""lantern_rotate_axes against the rotation in 64 bits."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


def _case(seed, N, Hq, Hk, D, sections, dtype, far=600):
    gen = torch.Generator().manual_seed(seed)
    q, k = (ref.normal(gen, N, h, D).to(dtype) for h in (Hq, Hk))
    pos = torch.randint(-3, far, (N, len(sections)), generator=gen, dtype=torch.int32)
    freqs = torch.rand(sum(sections), generator=gen) ** 3
    return q, k, pos, freqs


def _check(got, x, pos, freqs, sections, **kw):
    y, size = ref.rotate(x, pos, freqs, sections, **kw)
    off = (got.double().cpu() - y).abs()
    assert bool((off <= ref.rotate_bound(y, size, x.dtype)).all()), float((off - ref.rotate_bound(y, size, x.dtype)).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("N,Hq,Hk,D,sections", [
    (1, 1, 1, 2, (1,)), (3, 2, 1, 6, (1, 1)), (61, 20, 20, 64, (16, 16)), (130, 5, 3, 100, (17, 9, 24)), (7, 4, 2, 128, (64,)),
    (257, 3, 1, 128, (0, 20, 20, 20)), (5, 2, 2, 96, (3,)), (2, 1, 1, 1024, (256, 256)), (9, 1, 1, 1024, (511,)), (33, 1, 0, 72, (8, 8, 8))])
def test_against_64_bits(lantern_gpu, N, Hq, Hk, D, sections, inter, dtype):
    q, k, pos, freqs = _case(N + D, N, Hq, Hk, D, sections, dtype)
    for inverse in (False, True):
        a, b = lantern_gpu.rotate_axes(q.cuda(), k.cuda() if Hk else None, pos.cuda(), freqs.cuda(), sections, interleaved=inter, inverse=inverse)
        _check(a, q, pos, freqs, sections, interleaved=inter, inverse=inverse)
        if Hk:
            _check(b, k, pos, freqs, sections, interleaved=inter, inverse=inverse)
        else:
            assert b is None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_alignment_and_in_place(lantern_gpu, dtype):
    """Views of one projection's output, rows that begin anywhere, and outputs that are the inputs."""
    sections, D = (12, 20), 64
    q, k, pos, freqs = _case(5, 50, 4, 2, D, sections, dtype)
    for start, more in ((0, 0), (1, 3), (8, 16)):
        room = torch.full((50, start + 6 * D + more), 7.0, dtype=dtype, device="cuda")
        body = room[:, start:start + 6 * D].unflatten(1, (6, D))
        body[:, :4], body[:, 4:] = q.cuda(), k.cuda()
        for inter in (False, True):
            a, b = lantern_gpu.rotate_axes(body[:, :4], body[:, 4:], pos.cuda(), freqs.cuda(), sections, interleaved=inter)
            _check(a, q, pos, freqs, sections, interleaved=inter)
            _check(b, k, pos, freqs, sections, interleaved=inter)
        lantern_gpu.rotate_axes(body[:, :4], body[:, 4:], pos.cuda(), freqs.cuda(), sections, out=(body[:, :4], body[:, 4:]))
        _check(body[:, :4], q, pos, freqs, sections)
        _check(body[:, 4:], k, pos, freqs, sections)
        assert bool((room[:, :start] == 7).all()) and bool((room[:, start + 6 * D:] == 7).all())
    # heads before rows
    turned = q.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    a, _ = lantern_gpu.rotate_axes(turned, None, pos.cuda(), freqs.cuda(), sections)
    _check(a, q, pos, freqs, sections)


def test_far_positions(lantern_gpu):
    """Angles of 2^30 radians and both signs: cosine and sine are those of the exact product."""
    sections = (8,)
    q, _, _, _ = _case(1, 6, 1, 1, 16, sections, torch.float32)
    pos = torch.tensor([[2 ** 30], [-2 ** 30], [2 ** 31 - 1], [-2 ** 31], [10 ** 6 + 1], [0]], dtype=torch.int32)
    freqs = torch.tensor([1.0, 0.5, 0.1, 0.01, 1e-3, 1e-5, 0.0, 2.0 ** -20])
    for inter in (False, True):
        a, _ = lantern_gpu.rotate_axes(q.cuda(), None, pos.cuda(), freqs.cuda(), sections, interleaved=inter)
        _check(a, q, pos, freqs, sections, interleaved=inter)


@pytest.mark.parametrize("inter", [False, True])
def test_gradient_by_formula_and_by_differences(lantern_gpu, inter):
    """The map is linear, so differences are exact up to the outputs' rounding: with steps of one, the derivative of sum(y * g) by
    each element is the difference itself; and it is the inverse of g."""
    sections, D, N = (3, 5), 20, 2
    q, _, pos, freqs = _case(9, N, 1, 1, D, sections, torch.float32)
    g = ref.normal(torch.Generator().manual_seed(4), N, 1, D)
    args = (pos.cuda(), freqs.cuda(), sections)
    grad, _ = lantern_gpu.rotate_axes(g.cuda(), None, *args, interleaved=inter, inverse=True)
    formula, size = ref.rotate(g, pos, freqs, sections, interleaved=inter, inverse=True)
    assert bool(((grad.cpu().double() - formula).abs() <= ref.rotate_bound(formula, size, torch.float32)).all())
    steps = torch.eye(D).repeat(1, 1).view(1, D, D).expand(N, -1, -1)          # D heads, one element moved in each
    up, _ = lantern_gpu.rotate_axes((q + steps).cuda(), None, *args, interleaved=inter)
    down, _ = lantern_gpu.rotate_axes((q - steps).cuda(), None, *args, interleaved=inter)
    by_differences = ((up - down).double().cpu() * g.double()).sum(-1) / 2
    # each y is off by at most 6 * 2^-24 * (|a| + |b| + 2) and q +- 1 by 2^-24 * (|q| + 1)
    room = 16 * 2.0 ** -24 * (q.abs().max() * 2 + 3) * g.abs().sum(-1)
    assert bool(((grad.cpu().double()[:, 0] - by_differences).abs() <= room).all())


def test_streams_nothing_to_do_and_untouched_rest(lantern_gpu):
    sections = (16,)
    q, k, pos, freqs = _case(2, 300, 3, 3, 32, sections, torch.bfloat16)
    want, _ = lantern_gpu.rotate_axes(q.cuda(), None, pos.cuda(), freqs.cuda(), sections)
    side = torch.cuda.Stream()
    qc, kc, pc, fc = q.cuda(), k.cuda(), pos.cuda(), freqs.cuda()
    torch.cuda.synchronize()
    a, b = lantern_gpu.rotate_axes(qc, kc, pc, fc, sections, stream=side)
    side.synchronize()
    assert torch.equal(a, want)
    a, b = lantern_gpu.rotate_axes(qc[:0], kc[:0], pc[:0], fc, sections)
    assert a.shape == (0, 3, 32) and b.shape == (0, 3, 32)
    nan = q.clone()
    nan[5, 1] = float("nan")
    a, _ = lantern_gpu.rotate_axes(nan.cuda(), None, pc, fc, sections)
    assert bool(a[5, 1].isnan().all())
    a[5, 1] = want[5, 1]
    assert torch.equal(a, want)


@pytest.mark.parametrize("inter", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_autograd_turns_back(lantern_gpu, dtype, inter):
    """Gradients of q, of a key head that several share, and of either alone; a gradient without dense heads; twice over."""
    gen = torch.Generator().manual_seed(6)
    N, D, sections = 21, 32, (5, 9)
    pos = torch.randint(-50, 300, (N, 2), generator=gen, dtype=torch.int32).cuda()
    args = (pos, torch.rand(14, generator=gen).cuda(), sections)
    q = ref.normal(gen, N, 3, D).to(dtype).cuda().requires_grad_()
    k = ref.normal(gen, N, 1, D).to(dtype).cuda().requires_grad_()
    gq, gk = ref.normal(gen, N, 3, D).to(dtype).cuda(), ref.normal(gen, N, D, 4).to(dtype).cuda().transpose(1, 2)
    tq, tk = lantern_gpu.rotate_axes(q, k.expand(N, 4, D), *args, interleaved=inter)
    with torch.no_grad():
        wq, wk = lantern_gpu.rotate_axes(q, k.expand(N, 4, D), *args, interleaved=inter)
        bq, bk = lantern_gpu.rotate_axes(gq, gk.contiguous(), *args, interleaved=inter, inverse=True)
    assert torch.equal(tq, wq) and torch.equal(tk, wk) and not wq.requires_grad
    torch.autograd.backward([tq, tk], [gq, gk])
    assert torch.equal(q.grad, bq)
    half = torch.finfo(dtype).eps / 2      # torch's sum over the four heads: in fp32, then rounded once
    room = half * bk.double().sum(1, keepdim=True).abs() + 4 * 2.0 ** -24 * bk.double().abs().sum(1, keepdim=True)
    assert bool(((k.grad.double() - bk.double().sum(1, keepdim=True)).abs() <= room).all())
    alone, none = lantern_gpu.rotate_axes(q, None, *args, interleaved=inter)
    (again,) = torch.autograd.grad(alone, q, gq)
    assert none is None and torch.equal(again, bq)
    only_k = lantern_gpu.rotate_axes(q.detach(), k, *args, interleaved=inter)
    (again,) = torch.autograd.grad(only_k[1], k, gk[:, :1].contiguous())
    assert torch.equal(again, bk[:, :1]) and again.shape == k.shape
