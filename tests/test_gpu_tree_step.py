"""A tree step as a user runs it: turn, attend, verify, append; eager and as a replayed graph."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from parity_utils import random_table
from synth import trees, workloads

pytestmark = pytest.mark.gpu

SECTIONS, D, HEADS, KEY_HEADS, PAGE = (16, 16), 64, 4, 2, 16


class Step:
    """Static buffers of a batch of trees, and the calls on them."""

    def __init__(self, lantern, eight, dtype):
        self.lantern, self.dtype = lantern, dtype
        self.B, self.M = 3, 12
        self.cfg = workloads.with_overrides(workloads.CONFIGS["tiny"], delta=0.3)
        self.knn = torch.from_numpy(random_table(self.cfg.V, self.cfg.k, seed=2)).cuda()
        self.lengths = torch.tensor([30, 0, 15], dtype=torch.int32).cuda()
        gen = torch.Generator().manual_seed(1)
        cache, table = ref.filled_cache(gen, self.lengths.tolist(), KEY_HEADS, D, PAGE, eight, rubbish=False, spare=60)
        free = [i for i in range(cache[0].shape[0]) if i not in table.flatten().tolist()]
        more = torch.tensor(free[: self.B * 18], dtype=torch.int32).view(self.B, 18)
        self.cache = ref.on_gpu(cache)
        self.table = torch.cat([table, more], 1).cuda().contiguous()
        self.freqs = torch.rand(sum(SECTIONS), generator=gen).cuda()
        T = self.M + 1
        self.heads = torch.zeros((self.B, T, HEADS + 2 * KEY_HEADS, D), dtype=dtype, device="cuda")
        self.positions = torch.zeros((self.B, T, 2), dtype=torch.int32, device="cuda")
        self.parent = torch.zeros(self.B * self.M, dtype=torch.int32, device="cuda")
        self.rows = torch.zeros(self.B * self.M, dtype=torch.int32, device="cuda")
        self.tokens = torch.zeros(self.B * self.M, dtype=torch.int32, device="cuda")
        self.logits = [torch.zeros((self.B * T, self.cfg.V), device="cuda") for _ in range(2)]
        self.uniforms = torch.zeros((self.B * self.M, 2), device="cuda")

    def load(self, n):
        gen = torch.Generator().manual_seed(100 + n)
        parent = trees.random_trees(np.random.default_rng(n), self.B, self.M)
        st, row, tok, un = trees.tree_step(self.cfg, parent, step=n, device="cpu")
        self.heads.copy_(ref.normal(gen, *self.heads.shape).to(self.dtype))
        self.positions.copy_(torch.randint(0, 200, self.positions.shape, generator=gen, dtype=torch.int32))
        self.parent.copy_(torch.from_numpy(parent.reshape(-1)))
        self.rows.copy_(torch.from_numpy(row))
        self.tokens.copy_(torch.from_numpy(tok))
        self.logits[0].copy_(st.target_logits)
        self.logits[1].copy_(st.draft_logits)
        self.uniforms.copy_(un)

    def __call__(self):
        L, B, T = self.lantern, self.B, self.M + 1
        q, k, v = self.heads.split((HEADS, KEY_HEADS, KEY_HEADS), 2)
        tq, tk = L.rotate_axes(q.flatten(0, 1), k.flatten(0, 1), self.positions, self.freqs, SECTIONS)
        out = L.attend_trees(tq.view(B, T, HEADS, D), tk.view(B, T, KEY_HEADS, D), v, self.parent, self.cache, self.table, self.lengths)
        accept, n, path, nxt = L.verify_trees(*self.logits, self.rows, self.parent, self.M, self.tokens, self.knn, self.cfg.delta, self.uniforms)
        new = L.append_cache(self.cache, self.table, self.lengths, k, v, positions=self.positions, freqs=self.freqs, sections=SECTIONS,
                             path=path, count=n)
        self.lengths.copy_(new)
        return tq, tk, out, n, path, nxt


@pytest.mark.parametrize("eight,dtype", [(True, torch.bfloat16), (False, torch.float32)])
def test_steps_one_after_the_other(lantern_gpu, eight, dtype):
    """Each step against 64 bits on what the cache held before it; the cache after it against what was accepted."""
    step = Step(lantern_gpu, eight, dtype)
    moved = 0
    for n in range(5):
        step.load(n)
        before, lengths = [None if t is None else t.cpu().clone() for t in step.cache], step.lengths.tolist()
        tq, tk, out, count, path, nxt = step()
        B, T = step.B, step.M + 1
        q, k, v = step.heads.cpu().split((HEADS, KEY_HEADS, KEY_HEADS), 2)
        want, bound = ref.attend(tq.view(B, T, HEADS, D), tk.view(B, T, KEY_HEADS, D), v, step.parent.cpu(), before, step.table.cpu(), lengths)
        assert bool(((out.double().cpu() - want).abs() <= bound).all())
        assert bool((nxt >= -1).all())
        # values as they are: bit for bit; keys: the turned ones, up to half a step of the cache's type
        after, ends = ref.append(before, step.table.cpu(), lengths, torch.zeros_like(k), v, path.cpu(), count.cpu())
        assert step.lengths.tolist() == ends
        assert torch.equal(step.cache[1].cpu().view(torch.uint8), after[1].view(torch.uint8))
        y, size = ref.rotate(k.flatten(0, 1), step.positions.cpu().flatten(0, 1), step.freqs.cpu(), SECTIONS)
        y, off = y.view(B, T, KEY_HEADS, D), ref.rotate_bound(y, size, torch.float32).view(B, T, KEY_HEADS, D)
        for b in range(B):
            for i, row in enumerate(ref.rows_of(path.cpu(), count.cpu(), b, T)):
                at, slot = int(step.table[b, (lengths[b] + i) // PAGE]), (lengths[b] + i) % PAGE
                got = step.cache[0][at, :, slot].double().cpu()
                s = step.cache[2][at].double().cpu()[:, None] if eight else torch.zeros(KEY_HEADS, 1)
                got = got * s if eight else got
                room = (2.0 ** -4 if eight else 2.0 ** -8) * y[b, row].abs() + 2.0 ** -10 * s + 1.1 * off[b, row]
                assert bool(((got - y[b, row]).abs() <= room).all())
                moved += 1
    assert moved > 15


def test_captured_step_replays(lantern_gpu):
    """The whole step in a graph, its first replay included, with eager work between the replays; against the eager step."""
    eager, replayed = Step(lantern_gpu, True, torch.bfloat16), Step(lantern_gpu, True, torch.bfloat16)
    lantern_gpu.prepare(torch.float32, eager.cfg.V, eager.cfg.k)
    lantern_gpu.prepare_cache(torch.bfloat16, eager.cache)
    graph = torch.cuda.CUDAGraph()
    replayed.load(0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outs = replayed()
    for n in range(6):
        eager.load(n)
        replayed.load(n)
        want = eager()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
        for a, b in zip(replayed.cache, eager.cache):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(replayed.lengths, eager.lengths)


@pytest.mark.parametrize("dtype,eight,width,rows", [(torch.float32, True, 128, 3), (torch.float32, False, 96, 40), (torch.bfloat16, True, 128, 40)])
def test_wide_heads_captured_on_their_first_call(lantern_gpu, dtype, eight, width, rows):
    """prepare_cache before the capture is all that heads need whose tiles take more than 64 KiB of LDS."""
    gen = torch.Generator().manual_seed(rows)
    lengths = [700, 0]
    cache, table = ref.filled_cache(gen, lengths, 1, width, 32, eight)
    dev, tab = ref.on_gpu(cache), table.cuda()
    n = torch.tensor(lengths, dtype=torch.int32).cuda()
    lantern_gpu.prepare_cache(dtype, dev)
    q, k, v = (ref.normal(gen, 2, rows, 1, width).to(dtype).cuda() for _ in range(3))
    parent = torch.from_numpy(trees.random_trees(np.random.default_rng(5), 2, rows - 1).reshape(-1)).int().cuda()
    need = lantern_gpu.attend_trees_workspace_bytes(dtype, 2, rows - 1, 1, dev, tab.shape[1])
    space = torch.empty(need, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lantern_gpu.attend_trees(q, k, v, parent, dev, tab, n, workspace=space)
    for turn in range(3):
        q.copy_(ref.normal(gen, 2, rows, 1, width))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, lantern_gpu.attend_trees(q, k, v, parent, dev, tab, n))


def test_two_graphs_with_workspaces_of_their_own(lantern_gpu):
    """Split sequences captured twice, replayed at the same time on two streams."""
    gen = torch.Generator().manual_seed(3)
    lengths = (4000,)
    cache, table = ref.filled_cache(gen, lengths, 1, 64, 64, True)
    dev, tab, n = ref.on_gpu(cache), table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    graphs, outs, wants, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    for s in range(2):
        q, k, v = (ref.normal(gen, 1, 1, h, 64).to(torch.bfloat16).cuda() for h in (2, 1, 1))
        wants.append(lantern_gpu.attend_trees(q, k, v, None, dev, tab, n))
        need = lantern_gpu.attend_trees_workspace_bytes(torch.bfloat16, 1, 0, 2, dev, tab.shape[1])
        assert need > 0
        space = torch.empty(need, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(lantern_gpu.attend_trees(q, k, v, None, dev, tab, n, workspace=space))
        outs.append((q, k, v, space))
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], wants[0]) and torch.equal(outs[2], wants[1])
