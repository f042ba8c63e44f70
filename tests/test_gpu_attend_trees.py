"""lantern_attend_trees against the attention in 64 bits."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


def _case(seed, B, M, G, Hk, D, page, eight, dtype, lengths, odd_scales=False):
    gen = torch.Generator().manual_seed(seed)
    q, k, v = (ref.normal(gen, B, M + 1, h, D).to(dtype) for h in (G * Hk, Hk, Hk))
    cache, table = ref.filled_cache(gen, lengths, Hk, D, page, eight, odd_scales)
    return q, k, v, ref.tree(gen, B, M), cache, table, torch.tensor(lengths, dtype=torch.int32)


def _gpu(lantern, q, k, v, parent, cache, table, lengths, **kw):
    return lantern.attend_trees(q.cuda(), k.cuda(), v.cuda(), None if parent is None else parent.cuda(), ref.on_gpu(cache), table.cuda(), lengths.cuda(), **kw)


def _check(got, want, bound):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), (float((off / bound).max()), int((off > bound).sum()), int(got.isnan().sum()))


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,page,G,Hk,M,lengths", [
    (64, 64, 1, 2, 0, (0, 1, 63, 64, 65, 200, -1)), (64, 16, 1, 2, 60, (0, 1, 15, 16, 17, 500)), (128, 64, 8, 1, 0, (1, 300)),
    (128, 128, 4, 2, 32, (129, 127, 0)), (32, 32, 2, 3, 7, (31, 33, 100)), (96, 64, 1, 1, 15, (64, 1000)), (64, 64, 1, 1, 63, (640,)),
    (64, 64, 1, 1, 64, (10,)), (32, 16, 1, 1, 255, (40,)), (128, 16, 3, 1, 5, (257, 31)), (96, 128, 5, 2, 16, (260, 3))])
def test_against_64_bits(lantern_gpu, eight, dtype, D, page, G, Hk, M, lengths):
    """Lengths around a page and a tile, head groups, trees up to the largest; rubbish in every slot and page that is not seen."""
    case = _case(D + M, len(lengths), M, G, Hk, D, page, eight, dtype, lengths)
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,G,Hk,M,length", [(1, 1, 1, 0, 5000), (1, 2, 2, 20, 3001), (2, 8, 1, 40, 1500)])
def test_split_sequences(lantern_gpu, eight, dtype, B, G, Hk, M, length):
    """Few sequences and heads: their tokens are spread over workgroups and joined; lengths far under the table's as well."""
    D, page = 64, 64
    lengths = tuple(length - 1400 * b for b in range(B))
    case = _case(M + 7, B, M, G, Hk, D, page, eight, dtype, lengths)
    assert lantern_gpu.attend_trees_workspace_bytes(dtype, B, M, G * Hk, ref.on_gpu(case[4]), case[5].shape[1]) > 0
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)
    for few in (0, 1, 65):
        short = case[:6] + (torch.full((B,), few, dtype=torch.int32),)
        cache = [t.clone() if t is not None else None for t in case[4]]
        short = short[:4] + (cache,) + short[5:]
        want, bound = ref.attend(*short)
        _check(_gpu(lantern_gpu, *short), want, bound)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scales_of_any_size(lantern_gpu, dtype):
    """Scales that are no powers of two, pages whose values differ by 2^20, and a page of zeros."""
    case = _case(4, 2, 9, 2, 2, 64, 32, True, dtype, (90, 40), odd_scales=True)
    cache, table = case[4], case[5]
    cache[3][int(table[0, 1])] *= 2.0 ** 20
    cache[3][int(table[0, 0])] *= 2.0 ** -20
    cache[2][int(table[1, 0])] = 2.0 ** -126
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_scores_and_other_scales(lantern_gpu, dtype):
    """Maxima that move in every tile, scores of hundreds, a scale of zero (plain means) and others."""
    case = list(_case(5, 1, 12, 1, 1, 64, 16, False, dtype, (500,)))
    grow = torch.linspace(0.1, 20, 32)
    for w in range(32):
        if 0 <= int(case[5][0, w]) < case[4][0].shape[0]:
            case[4][0][int(case[5][0, w])] *= grow[w].to(torch.bfloat16)
    for scale in (None, 0.0, 1.0, 0.01):
        want, bound = ref.attend(*case, scale=scale)
        _check(_gpu(lantern_gpu, *case, scale=scale), want, bound)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,page,M,lengths,by", [(64, 64, 60, (640, 200), 4), (64, 16, 0, (640, 1000, 63), 8), (128, 128, 20, (700, 65), 8),
                                                 (32, 32, 9, (1200,), 16), (96, 64, 40, (400,), 64)])
def test_maxima_that_rise_along_a_sequence(lantern_gpu, eight, dtype, D, page, M, lengths, by):
    """Scores far apart: a row's largest comes up anywhere in a tile of tokens, after weights that are still to be used."""
    q, *rest = _case(D + by, len(lengths), M, 2, 2, D, page, eight, dtype, lengths)
    case = (q * by, *rest)
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("B,G,Hk,M,D,page", [(20, 1, 20, 32, 32, 32), (23, 2, 12, 40, 64, 64), (10, 1, 20, 70, 128, 64), (25, 3, 16, 10, 96, 128)])
def test_more_sequences_than_fit_at_once(lantern_gpu, eight, B, G, Hk, M, D, page):
    """Sets of rows side by side in a workgroup, the last one empty or not; the last row, a leaf, has a value that is infinite."""
    lengths = [(0, 1, 65, 130, -1, 40)[b % 6] for b in range(B)]
    q, k, v, parent, cache, table, n = _case(B, B, M, G, Hk, D, page, eight, torch.bfloat16, lengths)
    assert lantern_gpu.attend_trees_workspace_bytes(torch.bfloat16, B, M, G * Hk, ref.on_gpu(cache), table.shape[1]) == 0
    want, bound = ref.attend(q, k, v, parent, cache, table, n)
    odd = v.clone()
    odd[:, -1, :, 0] = math.inf
    got = _gpu(lantern_gpu, q, k, odd, parent, cache, table, n)
    _check(got[:, :-1], want[:, :-1], bound[:, :-1])
    there = n >= 0
    assert not bool(got[there][:, -1, :, 0].isfinite().any())
    _check(got[there][:, -1, :, 1:], want[there][:, -1, :, 1:], bound[there][:, -1, :, 1:])


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,G,Hk,M,D", [(30, 1, 20, 24, 32), (12, 2, 22, 27, 64)])
def test_two_tiles_of_rows_without_a_cut(lantern_gpu, eight, dtype, B, G, Hk, M, D):
    """Many short sequences of 25 or 56 rows to a key head: each wavefront takes 32 of them."""
    lengths = [(3, 70, 0, 129)[b % 4] for b in range(B)]
    case = _case(D + B, B, M, G, Hk, D, 32, eight, dtype, lengths)
    assert lantern_gpu.attend_trees_workspace_bytes(dtype, B, M, G * Hk, ref.on_gpu(case[4]), case[5].shape[1]) == 0
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_are_not_there(lantern_gpu, eight, dtype):
    """Candidates with a parent out of range, and those behind them, have zero rows and are seen by nobody, whatever they hold."""
    case = list(_case(6, 3, 20, 2, 1, 64, 64, eight, dtype, (70, 0, -1)))
    q, k, v, parent = case[:4]
    p = parent.view(3, 20)
    p[0, 4], p[0, 11], p[1, 0], p[1, 19] = -2, 11, 0, 400
    p[0, 7] = 4                                  # behind a lost one
    p[1, 1:10] = torch.arange(9)                 # a branch that begins at a lost candidate
    for b in (0, 1):
        _, there = ref.ancestors(p[b], 21)
        assert not all(there) and any(there)
        for i, t in enumerate(there):
            if not t:
                k[b, i], v[b, i], q[b, i] = math.nan, math.inf, math.nan
    k[2], v[2] = math.nan, math.nan
    want, bound = ref.attend(*case)
    got = _gpu(lantern_gpu, *case)
    _check(got, want, bound)
    assert bool((got[2] == 0).all()) and bool((got[0, 5] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_are_not_finite(lantern_gpu, dtype):
    """A candidate's NaN or infinity reaches the rows that see it and no other; its key's likewise."""
    case = list(_case(7, 2, 30, 1, 2, 32, 32, True, dtype, (50, 3)))
    q, k, v, parent = case[:4]
    want, bound = ref.attend(*case)
    v[0, 9, 1, 5], v[0, 3, 0, 7], k[1, 4, 0, 2] = math.nan, -math.inf, math.nan
    got = _gpu(lantern_gpu, *case).cpu()
    hit = torch.zeros_like(got, dtype=torch.bool)
    for b, i, h, d in ((0, 9, 1, 5), (0, 3, 0, 7), (1, 4, 0, slice(None))):
        sees, _ = ref.ancestors(parent.view(2, 30)[b], 31)
        for r in sees[:, i].nonzero().flatten().tolist():
            hit[b, r, h, d] = True
    assert bool(got[hit].isnan().all()) and bool(hit.any()) and not bool(hit.all())
    assert bool(((got.double() - want).abs() <= bound)[~hit].all())


@pytest.mark.parametrize("B,M", [(4, 3), (1, 0)])
def test_bad_pages_and_narrow_tables(lantern_gpu, B, M):
    """A needed page out of range, or a length beyond the table: the sequence's rows are NaN, the others right."""
    lengths = (100, 2000, 70, 30)[:B]
    case = list(_case(11, B, M, 1, 2, 64, 64, True, torch.bfloat16, lengths))
    want, bound = ref.attend(*case)
    table, n = case[5], case[6]
    pool = case[4][0].shape[0]
    table[0, 1] = pool
    if B > 1:
        table[2, 0] = -1
        n[3] = table.shape[1] * 64 + 1
    got = _gpu(lantern_gpu, *case).cpu()
    assert bool(got[0].isnan().all())
    if B > 1:
        assert bool(got[2:].isnan().all())
        _check(got[1:2], want[1:2], bound[1:2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides_alignment_and_chains(lantern_gpu, dtype):
    """Views of one projection's output that begin anywhere, heads before rows, and rows that follow each other."""
    B, T, G, Hk, D = 2, 33, 2, 2, 64
    case = list(_case(13, B, T - 1, G, Hk, D, 32, True, dtype, (77, 5)))
    case[3] = None
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)
    q, k, v, _, cache, table, n = case
    Hq, all_heads = G * Hk, (G + 2) * Hk
    chain = (torch.arange(T - 1, dtype=torch.int32) - 1).repeat(B)
    for start in (0, 3, 16):
        room = torch.full((B, T, start + all_heads * D + 5), math.nan, dtype=dtype, device="cuda")
        body = room[..., start:start + all_heads * D].unflatten(-1, (all_heads, D))
        body[:, :, :Hq], body[:, :, Hq:Hq + Hk], body[:, :, Hq + Hk:] = q.cuda(), k.cuda(), v.cuda()
        got = lantern_gpu.attend_trees(body[:, :, :Hq], body[:, :, Hq:Hq + Hk], body[:, :, Hq + Hk:], chain.cuda(), ref.on_gpu(cache), table.cuda(), n.cuda())
        _check(got, want, bound)
    turned = [t.cuda().transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v)]
    _check(lantern_gpu.attend_trees(*turned, None, ref.on_gpu(cache), table.cuda(), n.cuda()), want, bound)


def test_same_call_same_bits_on_any_stream(lantern_gpu):
    case = _case(17, 2, 60, 1, 4, 64, 64, True, torch.bfloat16, (3000, 200))
    dev = [t.cuda() for t in case[:4]] + [ref.on_gpu(case[4]), case[5].cuda(), case[6].cuda()]
    want = lantern_gpu.attend_trees(*dev)
    need = lantern_gpu.attend_trees_workspace_bytes(torch.bfloat16, 2, 60, 4, dev[4], dev[5].shape[1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty(max(need, 256), dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    got = [lantern_gpu.attend_trees(*dev, workspace=w, stream=s) for _ in range(3) for s, w in zip(streams, spaces)]
    got += [lantern_gpu.attend_trees(*dev, stream=streams[0])]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    if need:
        with pytest.raises(lantern_gpu.LanternError):
            lantern_gpu.attend_trees(*dev, workspace=spaces[0][:need - 1])


def test_far_pages(lantern_gpu):
    """A cache of more than 2^32 bytes, read behind them."""
    Hk, D, page = 4, 128, 128
    case = _case(19, 1, 4, 2, Hk, D, page, True, torch.bfloat16, (300,))
    want, bound = ref.attend(*case)
    q, k, v, parent, cache, table, n = case
    pages = (1 << 32) // (Hk * page * D) + 40
    big = lantern_gpu.make_cache(pages, Hk, page, D)
    used = -(-300 // page)
    at = [pages - 1 - 5 * i for i in range(used)]
    for b, s in zip(big, cache):
        b[at] = s[table[0, :used].long()].cuda()
    got = lantern_gpu.attend_trees(q.cuda(), k.cuda(), v.cuda(), parent.cuda(), big, torch.tensor([at], dtype=torch.int32).cuda(), n.cuda())
    _check(got, want, bound)
