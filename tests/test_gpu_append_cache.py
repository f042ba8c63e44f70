"""lantern_append_cache against the definition in 64 bits: codes and scales equal where keys are not turned."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.cpu().view(torch.uint8 if t.element_size() == 1 else torch.int16 if t.element_size() == 2 else torch.int32)


def _same(got, want):
    for g, w in zip(got, want):
        if w is not None:
            nan = w.float().isnan()
            assert torch.equal(g.cpu().float().isnan(), nan)
            assert torch.equal(torch.where(nan, 0, _bits(g)), torch.where(nan, 0, _bits(w)))


def _rows(gen, B, T, Hk, D, dtype, big=1.0):
    return (ref.normal(gen, B, T, Hk, D) * big).to(dtype), (ref.normal(gen, B, T, Hk, D) * 0.7).to(dtype)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,D,Hk,T,lengths", [
    (16, 32, 1, 1, (0,)), (16, 64, 2, 5, (0, 15, 16, 17)), (32, 96, 3, 70, (31, 0, 5)), (64, 64, 2, 61, (3, 64, 127, -1, 100)),
    (128, 128, 2, 200, (0, 1, 127)), (64, 128, 1, 64, (0, 64, 1))])
def test_prompts(lantern_gpu, eight, dtype, page, D, Hk, T, lengths):
    """Whole and partial pages, pages that hold earlier tokens, every type; the rest of the pages as it was."""
    gen = torch.Generator().manual_seed(page + D + T)
    B = len(lengths)
    k, v = _rows(gen, B, T, Hk, D, dtype)
    cache, table = ref.filled_cache(gen, [max(0, n) + T for n in lengths], Hk, D, page, eight, rubbish=False)
    count = torch.randint(0, T + 1, (B,), generator=gen, dtype=torch.int32)
    for c in (None, count):
        want, ends = ref.append(cache, table, lengths, k, v, count=c)
        dev = ref.on_gpu(cache)
        got = lantern_gpu.append_cache(dev, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), k.cuda(), v.cuda(),
                                       count=None if c is None else c.cuda())
        assert got.tolist() == ends
        _same(dev, want)


@pytest.mark.parametrize("eight", [True, False])
def test_accepted_paths(lantern_gpu, eight):
    """path and count as verify_trees leaves them: row 0, then the accepted candidates; a path of no candidates, a whole branch."""
    gen = torch.Generator().manual_seed(3)
    B, T, Hk, D, page = 5, 9, 2, 64, 16
    lengths = (0, 14, 31, 7, 16)
    path = torch.full((B, T - 1), -1, dtype=torch.int32)
    count = torch.tensor([0, 3, 8, 1, 2], dtype=torch.int32)
    for b in range(B):
        path[b, : count[b]] = torch.randperm(T - 1, generator=gen)[: count[b]].sort().values.to(torch.int32)
    path[4, :2] = 6                                       # the same candidate twice is two tokens
    k, v = _rows(gen, B, T, Hk, D, torch.bfloat16)
    cache, table = ref.filled_cache(gen, [n + T for n in lengths], Hk, D, page, eight, rubbish=False)
    want, ends = ref.append(cache, table, lengths, k, v, path, count)
    dev = ref.on_gpu(cache)
    got = lantern_gpu.append_cache(dev, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), k.cuda(), v.cuda(),
                                   path=path.cuda(), count=count.cuda())
    assert got.tolist() == ends
    _same(dev, want)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("sections,D,eight", [((16, 16), 64, True), ((5, 7), 32, True), ((20, 20, 20), 128, True), ((16,), 32, False)])
def test_rotation_on_the_way(lantern_gpu, sections, D, inter, eight):
    """Keys turned in fp32 and rounded once.  fp32's error (rotate_bound) and half a step of the cache's type: e4m3 2^-4 of the value or
    2^-10 of the scale among the subnormal codes, bf16 2^-8."""
    gen = torch.Generator().manual_seed(D)
    B, T, Hk, page = 3, 40, 2, 32
    lengths = (0, 20, 33)
    k, v = _rows(gen, B, T, Hk, D, torch.bfloat16)
    pos = torch.randint(0, 500, (B, T, len(sections)), generator=gen, dtype=torch.int32)
    freqs = torch.rand(sum(sections), generator=gen)
    cache, table = ref.filled_cache(gen, [n + T for n in lengths], Hk, D, page, eight, rubbish=False)
    dev = ref.on_gpu(cache)
    lantern_gpu.append_cache(dev, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), k.cuda(), v.cuda(), positions=pos.cuda(),
                             freqs=freqs.cuda(), sections=sections, interleaved=inter)
    y, size = ref.rotate(k.flatten(0, 1), pos.flatten(0, 1), freqs, sections, interleaved=inter)
    off32 = ref.rotate_bound(y, size, torch.float32)
    y, off32 = y.view(B, T, Hk, D), off32.view(B, T, Hk, D)
    kp, scale = dev[0].cpu(), None if dev[2] is None else dev[2].cpu()
    for b, n in enumerate(lengths):
        for t in range(T):
            at, slot = int(table[b, (n + t) // page]), (n + t) % page
            got = kp[at, :, slot].double()
            if eight:
                s = scale[at].double()[:, None]
                room = off32[b, t] * 1.1 + 2.0 ** -4 * y[b, t].abs() + 2.0 ** -10 * s
                got = got * s
            else:
                room = off32[b, t] * 1.1 + 2.0 ** -8 * y[b, t].abs()
            assert bool(((got - y[b, t]).abs() <= room).all())
    # values go in as they are
    want, _ = ref.append(cache, table, lengths, k, v)
    _same((dev[1], dev[3]), (want[1], want[3]))


def test_scales_grow_and_codes_are_rounded_again(lantern_gpu):
    """One token after the other of growing size into one page: each step exact; a page begun anew forgets its scale."""
    gen = torch.Generator().manual_seed(8)
    Hk, D, page = 2, 32, 16
    cache, table = ref.filled_cache(gen, [page], Hk, D, page, True, rubbish=False)
    cache[2].fill_(2.0 ** 60)
    dev, tab = ref.on_gpu(cache), table.cuda()
    for n in range(18):
        k, v = _rows(gen, 1, 1, Hk, D, torch.float32, big=4.0 ** (n % 7 - 2))
        want, ends = ref.append(cache, table, (n,), k, v)
        got = lantern_gpu.append_cache(dev, tab, torch.tensor([n], dtype=torch.int32).cuda(), k.cuda(), v.cuda())
        assert got.tolist() == ends
        _same(dev, want)
        cache = want


@pytest.mark.parametrize("values", [(0.0,), (448.0,), (448.1,), (2.0 ** -130, 2.0 ** -149), (3e38,), (math.inf, 1.0), (-math.inf, math.nan, 2.0), (math.nan,)])
def test_extremes(lantern_gpu, values):
    """Nothing but zeros, the borders of a scale, the smallest and largest numbers, and what is not finite."""
    Hk, D, page = 1, 32, 16
    x = torch.zeros(1, 3, Hk, D)
    x[0, 1, 0, : len(values)] = torch.tensor(values)
    for eight in (True, False):
        cache, table = ref.filled_cache(torch.Generator().manual_seed(1), [3], Hk, D, page, eight, rubbish=False)
        want, _ = ref.append(cache, table, (0,), x, x)
        dev = ref.on_gpu(cache)
        lantern_gpu.append_cache(dev, table.cuda(), torch.zeros(1, dtype=torch.int32).cuda(), x.cuda(), x.cuda())
        _same(dev, want)


def test_refused_on_the_device(lantern_gpu):
    """A sequence with a bad page, count, path entry or too narrow a table gets -2 and stays as it was; the others are served."""
    gen = torch.Generator().manual_seed(12)
    T, Hk, D, page = 6, 2, 32, 16
    lengths = (10, 14, 14, 3, 3, 60, 2 ** 31 - 3, 14, -5)
    B = len(lengths)
    cache, table = ref.filled_cache(gen, [63] * B, Hk, D, page, True, rubbish=False)
    pool = cache[0].shape[0]
    path = torch.arange(T - 1, dtype=torch.int32).repeat(B, 1)
    count = torch.full((B,), 5, dtype=torch.int32)
    table[1, 1], table[2, 1] = -1, pool
    count[3], path[4, 2] = -1, T - 1
    count[7] = 6
    k, v = _rows(gen, B, T, Hk, D, torch.bfloat16)
    dev = ref.on_gpu(cache)
    got = lantern_gpu.append_cache(dev, table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), k.cuda(), v.cuda(), path=path.cuda(), count=count.cuda())
    assert got.tolist() == [16, -2, -2, -2, -2, -2, -2, -2, -5]
    want, _ = ref.append(cache, table[:1], lengths[:1], k, v, path, count)
    _same(dev, want)


def test_strides_streams_and_far_pages(lantern_gpu):
    """Views of a projection that begin anywhere; a cache of more than 2^32 elements, written and read behind them."""
    gen = torch.Generator().manual_seed(6)
    Hk, D, page, T = 4, 128, 128, 30
    pages = (1 << 32) // (Hk * page * D) + 40
    k, v = _rows(gen, 1, T, Hk, D, torch.bfloat16)
    small, _ = ref.filled_cache(gen, [T + 100], Hk, D, page, True, rubbish=False, spare=0)
    want, _ = ref.append(small, torch.tensor([[0, 1]]), (110,), k, v)
    big = lantern_gpu.make_cache(pages, Hk, page, D)
    at = [pages - 1, pages - 7]
    for b, s in zip(big, small):
        b[at] = s[:2].cuda()
    table = torch.tensor([at], dtype=torch.int32).cuda()
    for start in (0, 1, 8):
        room = torch.zeros((T, start + 2 * Hk * D + 8), dtype=torch.bfloat16, device="cuda")
        body = room[:, start:start + 2 * Hk * D].unflatten(1, (2 * Hk, D))
        body[:, :Hk], body[:, Hk:] = k[0].cuda(), v[0].cuda()
        for b, s in zip(big, small):
            b[at] = s[:2].cuda()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = lantern_gpu.append_cache(big, table, torch.tensor([110], dtype=torch.int32).cuda(), body[None, :, :Hk], body[None, :, Hk:], stream=side)
        side.synchronize()
        assert got.tolist() == [140]
        _same([t[at] for t in big], [t[:2] for t in want])


@pytest.mark.parametrize("T", [6, 200])
@pytest.mark.parametrize("way", ["path", "rows"])
def test_counts_of_any_value(lantern_gpu, way, T):
    """Counts up to the ends of their type are refused like any that is beyond the rows; the largest that is right is served."""
    gen = torch.Generator().manual_seed(T)
    Hk, D, page = 2, 32, 16
    most = T - 1 if way == "path" else T
    counts = (2 ** 31 - 1, 2 ** 31 - 2, -2 ** 31, most + 1, most, 2 ** 31 - 1 - 12, 0)
    B = len(counts)
    cache, table = ref.filled_cache(gen, [12 + T] * B, Hk, D, page, True, rubbish=False)
    path = torch.arange(T - 1, dtype=torch.int32).repeat(B, 1) if way == "path" else None
    lengths, count = torch.full((B,), 12, dtype=torch.int32), torch.tensor(counts, dtype=torch.int32)
    k, v = _rows(gen, B, T, Hk, D, torch.bfloat16)
    dev = ref.on_gpu(cache)
    got = lantern_gpu.append_cache(dev, table.cuda(), lengths.cuda(), k.cuda(), v.cuda(), path=None if path is None else path.cuda(), count=count.cuda())
    kept = [4, 6]
    want, ends = ref.append(cache, table[kept], [12, 12], k[kept], v[kept], None if path is None else path[kept], count[kept])
    assert got.tolist() == [-2, -2, -2, -2, int(ends[0]), -2, int(ends[1])]
    _same(dev, want)
