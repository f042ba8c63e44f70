"""Calls around a tree step on a stream of the caller's, beside work that is still queued on the current one."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu


def _stream_of(t):
    """The stream whose memory a tensor lies in."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


def test_outputs_and_workspace_lie_in_the_streams_own_memory(lantern_gpu):
    """What the current stream has freed, but has not read yet, is not given to a call on another stream; the results are the current stream's."""
    gen = torch.Generator().manual_seed(3)
    Hq, Hk, D, n, T = 4, 2, 64, 1500, 5
    start, table = ref.filled_cache(gen, [n + T], Hk, D, 64, True)
    x = ref.normal(gen, 1, T, Hq + 2 * Hk, D).bfloat16().cuda()
    q, k, v = x.split((Hq, Hk, Hk), 2)
    parent, lengths, table = ref.tree(gen, 1, T - 1).cuda(), torch.tensor([n], dtype=torch.int32).cuda(), table.cuda()
    pos, freqs = torch.arange(T, dtype=torch.int32).cuda()[:, None], torch.rand(32, generator=gen).cuda()
    cache = ref.on_gpu(start)
    need = lantern_gpu.attend_trees_workspace_bytes(q.dtype, 1, T - 1, Hq, cache, table.shape[1])
    assert need > 0
    calls = (lambda s: lantern_gpu.attend_trees(q, k, v, parent, cache, table, lengths, stream=s),
             lambda s: lantern_gpu.rotate_axes(q[0], k[0], pos, freqs, (32,), stream=s),
             lambda s: lantern_gpu.append_cache(cache, table, lengths, k, v, stream=s))
    side = torch.cuda.Stream()
    for call in calls:
        want = call(None)
        want = want if isinstance(want, tuple) else (want,)
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        # queued on the current stream behind long work: copies of tensors that are then dropped, as large as outputs and workspace
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            busy = busy @ busy * 1e-3
        lent = [torch.full((nbytes,), i, dtype=torch.uint8, device="cuda") for i, nbytes in enumerate((need, 20, 2560, 5120, 4 * T * Hq * D))]
        copies = [t.clone() for t in lent]
        del lent
        got = call(side)
        got = got if isinstance(got, tuple) else (got,)
        assert all(_stream_of(t) == side.cuda_stream for t in got)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(bool((c == i).all()) for i, c in enumerate(copies))
