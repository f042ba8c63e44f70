"""lantern_attend_trees with more sequences than a wavefront has lanes, of which the long ones are cut into parts: one key head, as on one GPU of
several that share a model's heads."""
import pytest
import torch

import cache_reference as ref
from test_gpu_attend_trees import _case, _check, _gpu

pytestmark = pytest.mark.gpu


def _uneven(B, longest):
    """Nothing, no sequence, and short ones, with long ones among the first 64, the next and the last."""
    n = [(0, -1, 1, 33, 65, 400)[b % 6] for b in range(B)]
    for b, length in ((3, longest - 100), (63, 700), (64, longest - 1), (B - 2, longest // 2), (B - 1, longest)):
        n[b] = length
    return tuple(n)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("dtype,B,G,M", [(torch.bfloat16, 65, 1, 0), (torch.bfloat16, 100, 2, 1), (torch.bfloat16, 129, 4, 3), (torch.bfloat16, 384, 1, 0),
                                         (torch.float32, 65, 1, 0), (torch.float32, 100, 2, 1), (torch.float32, 250, 1, 0)])
def test_long_ones_among_many(lantern_gpu, eight, dtype, B, G, M):
    page, D = 64, 32
    case = _case(B + M, B, M, G, 1, D, page, eight, dtype, _uneven(B, 4090))
    assert lantern_gpu.attend_trees_workspace_bytes(dtype, B, M, G, ref.on_gpu(case[4]), case[5].shape[1]) > 0
    want, bound = ref.attend(*case)
    _check(_gpu(lantern_gpu, *case), want, bound)


def test_bad_pages_among_many(lantern_gpu):
    """A page that is none, in the first, a middle and the last part of sequences of each round of 64, and a table too narrow: these rows alone are NaN."""
    B, page = 200, 64
    lengths = list(_uneven(B, 4090))
    case = _case(9, B, 0, 1, 1, 64, page, True, torch.bfloat16, lengths)
    assert lantern_gpu.attend_trees_workspace_bytes(torch.bfloat16, B, 0, 1, ref.on_gpu(case[4]), case[5].shape[1]) > 0
    want, bound = ref.attend(*case)
    bad = {3: 0, 64: 30, B - 1: 63}
    for b, w in bad.items():
        case[5][b, w] = -1
    n = case[6].clone()
    n[130] = page * case[5].shape[1] + 1
    got = _gpu(lantern_gpu, *case[:6], n)
    lost = torch.zeros(B, dtype=torch.bool)
    lost[[*bad, 130]] = True
    assert bool(got[lost.cuda()].isnan().all())
    _check(got[~lost.cuda()], want[~lost], bound[~lost])


def test_captured_with_other_lengths(lantern_gpu):
    """The cuts follow the lengths that a replay finds; every replay beside the eager call."""
    B, page, Hk = 150, 64, 1
    case = _case(2, B, 2, 2, Hk, 32, page, True, torch.bfloat16, _uneven(B, 2500))
    cache, table = ref.filled_cache(torch.Generator().manual_seed(1), [2500] * B, Hk, 32, page, True, rubbish=False)
    cache, table = ref.on_gpu(cache), table.cuda()
    assert lantern_gpu.attend_trees_workspace_bytes(torch.bfloat16, B, 2, 2, cache, table.shape[1]) > 0
    q, k, v, parent = (t.cuda() for t in case[:4])
    lengths = case[6].cuda()
    lantern_gpu.prepare_cache(torch.bfloat16, cache)
    others = [torch.tensor(n, dtype=torch.int32).cuda() for n in ([0] * B, [2500] * B, list(_uneven(B, 2500))[::-1], [-1] * (B - 1) + [2499])]
    want = [lantern_gpu.attend_trees(q, k, v, parent, cache, table, n) for n in others]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = lantern_gpu.attend_trees(q, k, v, parent, cache, table, lengths)
    for _ in range(3):
        for n, w in zip(others, want):
            lengths.copy_(n)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)
            assert torch.equal(lantern_gpu.attend_trees(q, k, v, parent, cache, table, n), w)
