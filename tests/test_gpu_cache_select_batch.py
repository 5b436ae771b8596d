"""Selection of blocks for many single tokens (GPU): scores by warps that share all blocks of a step, a choice per list,
slices of a step; what chunks and long tables fall back to.  Every case says how many launches it is, so that none of them
moves to another kernel unseen."""
import math

import pytest
import torch

from tests.test_gpu_cache import DEV
from tests.test_gpu_cache_blocks import with_bounds

pytestmark = pytest.mark.gpu


def units(amax):
    """The least power of two u >= 2^-126 with amax <= 127 u, of each value (float64)."""
    e = torch.ceil(torch.log2((amax / 127).clamp(min=2.0 ** -126)))
    e = torch.where(127 * torch.exp2(e - 1) >= amax, e - 1, e)
    return torch.exp2(torch.where(127 * torch.exp2(e) < amax, e + 1, e).clamp(min=-126))


def lists_ref(cache, m, layer, x, q, n, first=1, last=1):
    """Lists [T][kv_heads][n] from the cache's bounds: a stable sort of all scores in float64, a sequence at a time."""
    hkv, rep, dh = cache.kv_heads, cache.q_heads // cache.kv_heads, cache.head_dim
    out = torch.full((sum(q), hkv, n), -1, dtype=torch.int32, device=DEV)
    t = 0
    for s, new in enumerate(q):
        full = (m.len[s] - new) // cache.page
        if new and 0 < full <= n:
            out[t:t + new, :, :full] = torch.arange(full, dtype=torch.int32, device=DEV)
        elif new and full:
            ids = torch.tensor(m.own[s][:full], device=DEV)
            c = x[t:t + new].double().view(new, hkv, rep, dh)
            u = units(c.abs().amax(-1, keepdim=True))
            c = torch.round(c / u)
            lo, hi = cache.codes[layer][ids].double().unbind(2)      # [full][hkv][dh]
            score = torch.einsum("tgrd,fgd->tgrf", c.clamp(max=0), lo) + torch.einsum("tgrd,fgd->tgrf", c.clamp(min=0), hi)
            score = (score * u).amax(2) * cache.scales[layer][ids].double().t()
            rest = torch.argsort(-score[..., first:full - last], dim=-1, stable=True)[..., :n - first - last] + first
            ends = torch.cat([torch.arange(first, device=DEV), torch.arange(full - last, full, device=DEV)])
            out[t:t + new] = torch.cat([ends.expand(new, hkv, -1), rest], -1).sort(-1)[0].int()
        t += new
    return out


def check(c, m, x, q, n, launches, first=1, last=1, layer=1):
    before = c.stats()["launches"]
    got = c.select(layer, x, n, first=first, last=last)
    assert c.stats()["launches"] - before == launches
    assert torch.equal(got, lists_ref(c, m, layer, x, q, n, first, last))
    assert c.stats()["status"] == 0


# Query heads, key/value heads: 1, 2, 3, 7, 20 and 128 heads to a key/value head.
SHAPES = [(8, 8), (8, 4), (9, 3), (14, 2), (40, 2), (128, 1)]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads", SHAPES)
@pytest.mark.parametrize("page", [16, 64])
def test_tokens_of_mixed_lengths(heads, dh, page):
    """Sequences of all lengths beside those whose blocks all fit, fresh ones and ones without a token."""
    n = 6
    ctx = [0, 3 * page, 700 * page // 16, page * n, page * n + page, 5, 333 * page // 16 + 1, 2000 * page // 16, 0, 17 * page, 40 * page] * 6
    q = [int(i % 9 != 4) for i in range(len(ctx))]
    c, m, x = with_bounds(heads + (dh,), page, ctx, q, layers=2, seed=dh + page)
    c.summarize(1, whole=True)
    small = sum(q) * heads[1] <= 64 and c.max_pages <= 1024
    check(c, m, x, q, n, 1 if small else 2)
    check(c, m, x, q, n, 1 if small else 2, first=0, last=0)
    check(c, m, x, q, n, 1 if small else 2, first=2, last=4)


@pytest.mark.parametrize("page,heads,dh,columns,n", [(16, (8, 2), 64, 2047, 40), (16, (4, 4), 128, 2049, 300), (16, (2, 1), 64, 9000, 1000),
                                                     (16, (20, 1), 128, 4100, 2100)])
def test_long_sequences(page, heads, dh, columns, n):
    """More blocks than a choice holds in registers (2048), beside shorter ones."""
    ctx = [columns * page, columns * page // 2 + 3, 50 * page]
    c, m, x = with_bounds(heads + (dh,), page, ctx, [1] * 3)
    c.summarize(1, whole=True)
    check(c, m, x, [1] * 3, n, 2)
    check(c, m, x, [1] * 3, n, 2, first=5, last=0)


@pytest.mark.parametrize("spread", ["equal", "clusters", "magnitudes", "zero"])
@pytest.mark.parametrize("columns,n", [(1500, 700), (2500, 60)])
def test_clustered_scores(columns, n, spread):
    """Hundreds of equal keys around the last one taken, in registers and behind them."""
    q = [1] * 40
    ctx = [columns * 16 + 5, 300 * 16] + [100 * 16] * 38
    c, m, x = with_bounds((4, 2, 64), 16, ctx, q, poison=False, seed=n)
    g = torch.Generator(device=DEV).manual_seed(n)
    one = torch.randn((1, 1, 16, 64), generator=g, device=DEV)
    for s in (0, 1):
        ids = m.own[s][:ctx[s] // 16]
        k = len(ids)
        if spread == "clusters":
            f = torch.tensor([1.0, 1.0, 1.0078125, -3.0], device=DEV)[torch.randint(0, 4, (k,), generator=g, device=DEV)]
        elif spread == "magnitudes":
            f = torch.exp2(torch.randint(-60, 60, (k,), generator=g, device=DEV).float()) * torch.randint(-1, 2, (k,), generator=g, device=DEV)
        else:
            f = torch.full((k,), float(spread == "equal"), device=DEV)
        c.k[1, ids] = (one * f.view(-1, 1, 1, 1)).expand(k, 2, 16, 64).bfloat16()
    c.summarize(1, whole=True)
    check(c, m, x, q, n, 2)
    check(c, m, x, q, n, 2, first=0, last=0)


def test_slices_of_many_tokens():
    """More than 1024 tokens are scored and chosen for 1024 at a time."""
    ctx = [16 * (i * 7 % 45) + i % 16 for i in range(1000)]
    q = [1 + i % 2 for i in range(1000)]
    c, m, x = with_bounds((4, 2, 64), 16, ctx, q, layers=2)
    c.summarize(1, whole=True)
    assert sum(q) == 1500
    check(c, m, x, q, 8, 4)


def test_slices_of_long_tables():
    """Scores are held for 8 M blocks at a time: 3 tokens here."""
    columns = 1 << 20
    ctx, q = [16 * 300, 16 * 500, 0, 16 * 40, 16 * 900, 16 * 77, 16 * 60, 16 * 61], [1] * 7 + [2]
    c, m, x = with_bounds((4, 2, 64), 16, ctx, q, width=columns - 902)
    c.summarize(1, whole=True)
    most = (8 << 20) // (-(-c.max_pages // 4) * 4 * 2)
    assert most == 3 or most == 4
    check(c, m, x, q, 7, 2 * -(-9 // most))


@pytest.mark.parametrize("heads,dh", [((8, 2), 128), ((12, 12), 64), ((7, 1), 64)])
def test_chunks_in_long_tables(heads, dh):
    """Eight tokens' scores over all columns of the table do not fit in shared memory: token by token."""
    ctx, q = [16 * 700 + 3, 16 * 90], [70, 33]
    c, m, x = with_bounds(heads + (dh,), 16, ctx, q, width=4000)
    c.summarize(1, whole=True)
    check(c, m, x, q, 20, 2)
    narrow, m2, x2 = with_bounds(heads + (dh,), 16, ctx, q)
    narrow.summarize(1, whole=True)
    check(narrow, m2, x2, q, 20, 1)
    assert math.prod(narrow.k.shape) == math.prod(c.k.shape)


@pytest.mark.parametrize("q,launches", [([1, 1], 1), ([1] * 40, 2), ([20, 9], 1)])
@pytest.mark.parametrize("keys,queries", [(100, 100), (-100, -90), (120, -120), (60, -126), (-126, 30)])
def test_scores_outside_of_single_precision(q, launches, keys, queries):
    """A score is the product of a sum, the query's unit and the block's scale, each step in fp32: infinite above its range,
    coarser or zero below, and of equal ones the lower columns are taken."""
    ctx = [16 * 200, 16 * 90] + [16 * 30] * (len(q) - 2)
    c, m, x = with_bounds((4, 2, 64), 16, ctx, q, poison=False)
    g = torch.Generator(device=DEV).manual_seed(3)
    lift = torch.exp2(torch.randint(keys - 6, keys + 1, (c.n_pages, 2, 1, 1), generator=g, device=DEV).double())
    c.k[1] = (torch.randn(c.k[1].shape, generator=g, device=DEV).double().clamp(-3.9, 3.9) * lift).bfloat16()
    x.copy_((torch.randn(x.shape, generator=g, device=DEV).double().clamp(-3.9, 3.9) * 2.0 ** queries).bfloat16())
    c.summarize(1, whole=True)
    before = c.stats()["launches"]
    got = c.select(1, x, 9)
    assert c.stats()["launches"] - before == launches
    t = 0
    for s, new in enumerate(q):
        full = ctx[s] // 16
        ids = torch.tensor(m.own[s][:full], device=DEV)
        y = x[t:t + new].double().view(new, 2, 2, 64)
        u = units(y.abs().amax(-1, keepdim=True))
        y = torch.round(y / u)
        lo, hi = c.codes[1][ids].double().unbind(2)
        whole = torch.einsum("tgrd,fgd->tgrf", y.clamp(max=0), lo) + torch.einsum("tgrd,fgd->tgrf", y.clamp(min=0), hi)
        score = (whole.float() * u.float()).amax(2) * c.scales[1][ids].t()
        rest = torch.argsort(-score[..., 1:full - 1], dim=-1, stable=True)[..., :7] + 1
        ends = torch.tensor([0, full - 1], device=DEV).expand(new, 2, 2)
        assert torch.equal(got[t:t + new], torch.cat([ends, rest], -1).sort(-1)[0].int()), s
        t += new
    assert c.stats()["status"] == 0
