"""Plain restatements, in float64, of the bounds of blocks, their selection and attention over chosen blocks."""
import math

import torch

from tests.cache_helpers import attend_ref, attend_tol, rows_of, scale_of


def unit_of(amax):
    """Least power of two u >= 2^-126 with amax <= 127 u, by search."""
    e = -126
    while amax > 127 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def bounds_ref(keys):
    """keys [page][dh] -> (lo, hi as whole numbers of the unit, unit); an infinity or a NaN: zeros and infinity."""
    k = keys.double()
    if not torch.isfinite(k).all():
        z = torch.zeros(k.shape[1], dtype=torch.float64, device=k.device)
        return z, z, math.inf
    u = unit_of(float(k.abs().max()))
    return torch.floor(k.amin(0) / u), torch.ceil(k.amax(0) / u), u


def check_bounds(cache, layer, pages):
    """The bounds of these pages are those of their keys."""
    for p in pages:
        for h in range(cache.kv_heads):
            lo, hi, u = bounds_ref(cache.k[layer, p, h])
            assert float(cache.scales[layer, p, h]) == u, (p, h)
            assert torch.equal(cache.codes[layer, p, h, 0].double(), lo), (p, h)
            assert torch.equal(cache.codes[layer, p, h, 1].double(), hi), (p, h)


def select_ref(cache, m, layer, x, q, n, first=1, last=1):
    """Lists [T][kv_heads][n] from the cache's bounds, one token and head at a time."""
    rep, dh = cache.q_heads // cache.kv_heads, cache.head_dim
    out = torch.full((sum(q), cache.kv_heads, n), -1, dtype=torch.int32)
    codes, scales = cache.codes[layer].cpu().double(), cache.scales[layer].cpu().double()
    x = x.cpu().double().view(-1, cache.kv_heads, rep, dh)
    t = 0
    for s, new in enumerate(q):
        full = (m.len[s] - new) // cache.page
        ids = m.own[s][:full]
        for _ in range(new):
            for g in range(cache.kv_heads):
                if full <= n:
                    out[t, g, :full] = torch.arange(full)
                    continue
                best = torch.full((full,), -math.inf, dtype=torch.float64)
                for r in range(rep):
                    v = x[t, g, r]
                    if not torch.isfinite(v).all():
                        best = best.maximum(torch.zeros(()).double())
                        continue
                    u = unit_of(float(v.abs().max()))
                    c = torch.round(v / u)
                    best = best.maximum(torch.maximum(c * codes[ids, g, 0], c * codes[ids, g, 1]).sum(-1) * u)
                score = torch.where(torch.isinf(scales[ids, g]), math.inf, best * scales[ids, g].nan_to_num(posinf=0.0))
                always = list(range(first)) + list(range(full - last, full))
                rest = [b for b in range(first, full - last)]
                rest.sort(key=lambda b: (-float(score[b]), b))
                out[t, g] = torch.tensor(sorted(always + rest[:n - first - last]), dtype=torch.int32)
            t += 1
    return out


def check_blocks(cache, m, x, q, blocks, out, layer, tree=None, scale=None, heads=None, tokens=None):
    """attend_blocks against attend_ref, token by token (heads, tokens: those that are looked at)."""
    dh, rep, page = cache.head_dim, cache.q_heads // cache.kv_heads, cache.page
    lists = blocks.cpu().tolist()
    t = 0
    for s, new in enumerate(q):
        kv = m.len[s]
        base = kv - new
        if new:
            k, v = rows_of(cache.k[layer], m, s, kv), rows_of(cache.v[layer], m, s, kv)
        for i in range(new):
            for g in (heads or range(cache.kv_heads)) if tokens is None or t in tokens else ():
                seen = torch.zeros(1, kv, dtype=torch.bool, device=x.device)
                for b in lists[t][g]:
                    if b >= 0:
                        seen[0, b * page:(b + 1) * page] = True
                seen[0, base // page * page:base] = True
                if tree is None:
                    seen[0, base:base + i + 1] = True
                else:
                    for j in range(new):
                        seen[0, base + j] = bool(int(tree[t]) >> j & 1)
                at = slice(g * rep, (g + 1) * rep)
                ref, mag = attend_ref(x[t].view(-1, dh)[at][None], k[g:g + 1], v[g:g + 1], seen, scale or scale_of(dh))
                got = out[t].view(-1, dh)[at][None].double()
                assert torch.equal(torch.isnan(got), torch.isnan(ref)), (s, i, g)
                err = torch.where(torch.isfinite(ref), (got - ref).abs() - attend_tol(ref, mag), -1.0)
                assert float(err.max()) <= 0, (s, i, g, float(err.max()))
            t += 1
