"""The operators around a tree step in 64 bits, from their definitions, on the CPU; inputs for their tests; bounds on their errors."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # relative half step of a rounding
LARGEST = 448.0


def rotate(x, positions, freqs, sections, interleaved=False, inverse=False):
    """x [N, heads, D], positions [N, axes] -> (turned, sum of magnitudes of the terms of each element), fp64."""
    x = x.double().cpu()
    y, size = x.clone(), x.abs()
    P, j = sum(sections), 0
    for axis, n in enumerate(sections):
        for _ in range(n):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + P)
            phi = positions[:, axis].cpu().double() * float(freqs[j]) * (-1.0 if inverse else 1.0)
            c, s = phi.cos()[:, None], phi.sin()[:, None]
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., a] * s + x[..., b] * c
            size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
            j += 1
    return y, size


def rotate_bound(y, size, dtype):
    """cos and sin rounded once (2^-24), product and sum once each: 3 half steps of the terms, and one for the second order; then
    the output's rounding.  The angle's own error (2^-52 of it, below 2^30 in the tests) is under 2^-22 of an element."""
    return 4 * 2.0 ** -24 * size + 2.0 ** -22 * 2.0 ** -4 * size + (HALF[dtype] * y.abs() if dtype != torch.float32 else 0.0) + 1e-37


def scale_for(largest):
    if largest == 0:
        return 2.0 ** -126
    m, e = math.frexp(largest)
    return 2.0 ** max(-126, e - 9 + (m > 0.875))


def quantise(x, scale):
    """Values (fp64) as e4m3 codes of a scale: what is not finite becomes NaN."""
    q = (x / scale).clamp(-LARGEST, LARGEST)
    return torch.where(x.isfinite(), q, torch.full_like(q, math.nan)).float().to(torch.float8_e4m3fn)


def rows_of(path, count, b, T):
    if path is None:
        return list(range(T if count is None else int(count[b])))
    return [0] + [int(p) + 1 for p in path[b, : int(count[b])]]


def append(cache, table, lengths, k, v, path=None, count=None):
    """Cache tensors after k, v [B, T, heads, D] (already turned) went in, and the new lengths.  On CPU copies."""
    kp, vp, ks, vs = (None if t is None else t.cpu().clone() for t in cache)
    page = kp.shape[2]
    ends = []
    for b in range(len(lengths)):
        start = int(lengths[b])
        if start < 0:
            ends.append(start)
            continue
        rows = rows_of(path, count, b, k.shape[1])
        ends.append(start + len(rows))
        for w in range(start // page, -(-ends[-1] // page)):
            lo, hi, at = max(start, w * page), min(ends[-1], (w + 1) * page), int(table[b, w])
            for pages, scales, x in ((kp, ks, k), (vp.transpose(2, 3), vs, v)):
                for h in range(kp.shape[1]):
                    new = x[b, rows[lo - start:hi - start], h].double().cpu()
                    slots = slice(lo - w * page, hi - w * page)
                    if scales is None:
                        pages[at, h, slots] = new.to(torch.float32).to(torch.bfloat16)
                        continue
                    fine = new[new.isfinite()]
                    scale = scale_for(float(fine.abs().max()) if fine.numel() else 0.0)
                    if lo > w * page:
                        was = float(scales[at, h])
                        scale = max(scale, was)
                        old = slice(0, lo - w * page)
                        pages[at, h, old] = quantise(pages[at, h, old].double() * was, scale)
                    pages[at, h, slots] = quantise(new, scale)
                    scales[at, h] = scale
    return (kp, vp, ks, vs), ends


def ancestors(parent, T):
    """sees [T, T] and which rows are there, of one tree of T - 1 candidates (parent None: a chain)."""
    sees, there = torch.zeros((T, T), dtype=torch.bool), [True] * T
    sees[0, 0] = True
    for i in range(1, T):
        p = i - 2 if parent is None else int(parent[i - 1])
        there[i] = -1 <= p < i - 1 and there[p + 1]
        if there[i]:
            sees[i] = sees[p + 1]
            sees[i, i] = True
    return sees, there


def attend(q, k, v, parent, cache, table, lengths, scale=None):
    """(out, bound on a kernel's error) [B, T, heads, D], fp64.  The bound: a score's exponent is off by the fp32 sum over D
    terms, and by two roundings of its scale; exp2 by 2^-22; the sums over n weights by n half steps each; bf16 rounds every
    weight w by 2^-8 of it: with w' in both sums, o' - o = sum (w' - w)(v - o) / sum w', at most 2^-8 sum p |v - o|; then the output's
    rounding."""
    dtype = q.dtype
    half = HALF[dtype]
    B, T, Hq, D = q.shape
    kp, vp, ks, vs = (None if t is None else t.cpu() for t in cache)
    Hk, page = kp.shape[1], kp.shape[2]
    G = Hq // Hk
    scale = D ** -0.5 if scale is None else scale
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    out, bound = torch.zeros((B, T, Hq, D), dtype=torch.float64), torch.zeros((B, T, Hq, D), dtype=torch.float64)
    for b in range(B):
        n = int(lengths[b])
        if n < 0:
            continue
        sees, there = ancestors(None if parent is None else parent.view(B, T - 1)[b], T)
        pages = table[b, : -(-n // page)].cpu().long()
        for h in range(Hk):
            ck, cv = kp[pages, h].double(), vp[pages, h].double()
            if ks is not None:
                ck, cv = ck * ks[pages, h].double()[:, None, None], cv * vs[pages, h].double()[:, None, None]
            ck, cv = ck.reshape(-1, D)[:n], cv.transpose(1, 2).reshape(-1, D)[:n]
            for i in range(T):
                if not there[i]:
                    continue
                rows = sees[i].nonzero().flatten()
                kk, vv = torch.cat([ck, k[b, rows, h]]), torch.cat([cv, v[b, rows, h]])
                qq = q[b, i, h * G:(h + 1) * G]
                s = qq @ kk.t() * scale
                p = torch.softmax(s, -1)
                o = p @ vv
                out[b, i, h * G:(h + 1) * G] = o
                reach = (qq.abs() @ kk.abs().t() * scale).amax(-1, keepdim=True)
                much = 2 * 2.0 ** -24 * (D + 8) * reach + 2 * 2.0 ** -22 + 2 * 2.0 ** -24 * (len(kk) + 8)
                room = much * (p @ vv.abs()) + half * o.abs() + 1e-37
                if dtype == torch.bfloat16:
                    room = room + 2.0 ** -8 * (p @ vv.abs() + o.abs())
                bound[b, i, h * G:(h + 1) * G] = room
    return out, bound


def normal(gen, *size):
    return torch.randn(*size, generator=gen)


def tree(gen, B, M):
    """parent [B*M] int32, every candidate behind a random one before it."""
    p = torch.rand(B, M, generator=gen) * torch.arange(1, M + 1)
    return (p.floor().to(torch.int32) - 1).reshape(-1).contiguous()


def filled_cache(gen, tokens, Hk, D, page, eight, odd_scales=False, spare=2, rubbish=True):
    """(cache, table) on the CPU for sequences of `tokens` cached tokens each, room for one page more; slots behind the ends, other
    pages and table entries that are not needed hold rubbish."""
    B = len(tokens)
    width = max(max(tokens), 0) // page + 1
    pool = B * width + spare
    table = torch.randperm(pool, generator=gen)[: B * width].view(B, width).to(torch.int32)
    x, y = normal(gen, pool, Hk, page, D), normal(gen, pool, Hk, D, page) * 1.5
    cache = [x.to(torch.bfloat16), y.to(torch.bfloat16), None, None]
    if eight:
        cache = []
        for t in (x, y):
            s = torch.tensor([scale_for(float(m)) for m in t.abs().amax((2, 3)).flatten()]).view(pool, Hk)
            if odd_scales:
                s = t.abs().amax((2, 3)) / LARGEST * 1.01
            cache.append((t / s[..., None, None]).to(torch.float8_e4m3fn))
            cache.append(s.contiguous())
        cache = [cache[0], cache[2], cache[1], cache[3]]
    if rubbish:
        nan = torch.tensor(math.nan).to(cache[0].dtype)
        used = set()
        for b, n in enumerate(tokens):
            for w in range(width):
                at, keep = int(table[b, w]), min(page, max(0, n - w * page))
                used.add(at)
                cache[0][at, :, keep:], cache[1][at, :, :, keep:] = nan, nan
                if keep == 0:
                    table[b, w] = (-1, pool + 7, 1 << 30)[(b + w) % 3]
        for at in set(range(pool)) - used:
            cache[0][at], cache[1][at] = nan, nan
    return cache, table.contiguous()


def on_gpu(cache):
    return tuple(None if t is None else t.cuda() for t in cache)
