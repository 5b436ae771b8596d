"""Paths of the paged cache that ordinary cases seldom reach.  Where a path hangs on the step's plan, the test first says,
by the step's rules, that its sizes give that plan."""
import random

import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.cache_helpers import CacheModel
from tests.test_gpu_cache import DEV, check_attend, filled

pytestmark = pytest.mark.gpu


def plan_of(shapes, ctx, q):
    """The work list of a step: cost and tokens of each group, and whether whole items are drawn."""
    hq, hkv, _ = shapes
    tt = 128 // (hq // hkv)
    groups = []
    for c, n in zip(ctx, q):
        for first in range(0, n, 2 * tt):
            m = min(2 * tt, n - first)
            keys = c + n if n <= 64 else c + first + m
            groups.append((-(-keys // 128) + 1 << (m > tt), m))
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    total = hkv * sum(g[0] for g in groups)
    return dict(groups=len(groups), whole=2 * max(g[0] for g in groups) * sms <= total,
                pairs=any(g[1] > tt for g in groups), items=len(groups) * hkv, sms=sms)


@pytest.mark.parametrize("shapes,page", [((4, 4, 64), 16), ((4, 4, 128), 32), ((8, 4, 64), 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_first_tile_by_hand_behind_a_joined_item(shapes, page, bad):
    """A CTA draws several one-tile items.  The slots of the earlier ones read each other's sums; in the later ones a
    slot's first tile has a value that is not finite and that only the last token sees, so that the softmax warps add
    it themselves, where the other slot may still read."""
    n = 260
    long = [200 + (i * 53) % 180 for i in range(n // 2)]                    # two or three tiles, both slots
    short = [20 + (i * 41) % 100 if i % 2 else 130 + (i * 17) % 100 for i in range(n - n // 2)]   # tile 0, or tile 1
    ctx, q = long + short, [1] * len(long) + [3] * len(short)
    plan = plan_of(shapes, ctx, q)
    assert plan["whole"] and not plan["pairs"] and plan["items"] > 3 * plan["sms"]
    cache, m, x = filled(shapes, page, ctx, q, seed=23)
    for s in range(len(long), n):
        a, b = m.row(s, m.len[s] - 1)
        cache.v[1, a, :, b, 1::3] = bad
    first = cache.attend(1, x)
    check_attend(cache, m, x, q, first, 1)
    rows = torch.arange(sum(q), device=DEV) - len(long)
    seen = (rows >= 0) & (rows % 3 == 2)
    assert torch.equal(torch.isfinite(first.float()).all(1), ~seen)
    for _ in range(30):
        assert torch.equal(cache.attend(1, x).view(torch.int16), first.view(torch.int16))
    assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,page", [((8, 8, 128), 64), ((8, 8, 64), 32)])
def test_whole_items_of_two_query_tiles(shapes, page):
    """Many prompts of like length: every CTA draws whole items, most of them of two query tiles."""
    q = [257 + (i * 29) % 70 for i in range(40)]
    ctx = [(i * 61) % 90 if i % 3 == 0 else 0 for i in range(40)]
    plan = plan_of(shapes, ctx, q)
    assert plan["whole"] and plan["pairs"] and plan["items"] > plan["sms"]
    cache, m, x = filled(shapes, page, ctx, q, seed=37)
    out = cache.attend(1, x)
    check_attend(cache, m, x, q, out, 1)
    assert torch.equal(cache.attend(1, x), out) and cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,page,ctx,q,whole", [
    ((64, 1, 64), 64, [0] * 15, [300] * 15, True),                           # groups of 4 tokens
    ((64, 1, 128), 128, [0, 700] + [0] * 15, [250, 260] + [270] * 15, True),
    ((32, 1, 128), 64, [9000] + [0] * 100, [3] + [100] * 100, False),        # groups of 8, one of them long
    ((32, 1, 64), 16, [0] * 100 + [9000], [100] * 100 + [3], False)])
def test_more_groups_than_threads(shapes, page, ctx, q, whole):
    """The step's block has 1024 threads; beyond as many groups it makes the work list in rounds."""
    plan = plan_of(shapes, ctx, q)
    assert plan["groups"] > 1024 and plan["whole"] == whole
    cache, m, x = filled(shapes, page, ctx, q, seed=41)
    out = cache.attend(0, x)
    check_attend(cache, m, x, q, out, 0)
    assert torch.equal(cache.attend(0, x), out) and cache.stats()["device_error"] == 0


def test_more_fresh_pages_than_threads():
    """A step that takes more than 1024 pages, found in several rounds over a pool that is mostly taken, with a shared last
    page to copy among the later ones."""
    n_pages, page = 9000, 16
    c = B.PagedCache.empty(2, n_pages, 2, 1, 64, page, 4, 1100, T_max=17500)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))
    m = CacheModel(n_pages, 4, 1100, page)
    m.ref = [int(i % 5 != 2) for i in range(n_pages)]                  # 1800 free
    c.ref.copy_(torch.tensor(m.ref, dtype=torch.int32))
    for seq, q in (([0], [40]), ([3], [7])):
        c.step(seq, q)
        assert m.step(seq, q) == []
    c.fork([0], [2])
    m.fork([0], [2])
    seq, q = [1, 0, 3], [16500, 5, 900]
    k, v = c.k.clone(), c.v.clone()
    c.step(seq, q)
    copies = m.step(seq, q)
    assert len(copies) == 1 and len(m.own[1]) > 1024                   # the copy's page is taken behind these
    for a, b in copies:
        k[:, b], v[:, b] = k[:, a], v[:, a]
    assert torch.equal(c.table.cpu(), m.table()) and c.length.tolist() == m.len and c.ref.tolist() == m.ref
    assert torch.equal(c.k, k) and torch.equal(c.v, v)
    qkv = torch.randn((sum(q), 4 * 64), device=DEV).to(torch.bfloat16)
    c.append(1, qkv, theta=0.0)
    at = 0
    for s, n in zip(seq, q):
        pos = torch.arange(m.len[s] - n, m.len[s], device=DEV)
        pages = c.table[s].long()[pos // page]
        k[1, pages, 0, pos % page] = qkv[at:at + n, 128:192]
        v[1, pages, 0, pos % page] = qkv[at:at + n, 192:]
        at += n
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and c.stats()["status"] == 0


@pytest.mark.parametrize("page,dh,seed", [(16, 64, 1), (16, 128, 2), (64, 128, 3), (128, 64, 4)])
def test_long_accepted_paths(page, dh, seed):
    """Paths longer than the lanes that move a row (8 or 16), up to the 64 that a tree has."""
    rng = random.Random(seed)
    layers, hkv, seqs = 2, 3, 6
    c = B.PagedCache.empty(layers, 90, hkv, hkv, dh, page, seqs, 12, T_max=400)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))
    m = CacheModel(90, seqs, 12, page)
    lens = [0, 1, 15, 16, 31, 100]
    for q in (lens, [64] * seqs):
        c.step(range(seqs), q)
        m.step(range(seqs), q)
    k, v = c.k.clone(), c.v.clone()
    n_acc = [64, 63, 40, 17, 9, 33]
    path = [sorted(rng.sample(range(64), n)) + [-1] * (64 - n) for n in n_acc]
    path[5] = list(range(31, 64)) + [7] * 31                           # the last 33 in a row
    c.accept(range(seqs), torch.tensor(n_acc, dtype=torch.int32, device=DEV), torch.tensor(path, dtype=torch.int32, device=DEV))
    for moves in m.accept(range(seqs), n_acc, path):
        for a, b in moves:
            k[:, b[0], :, b[1]], v[:, b[0], :, b[1]] = k[:, a[0], :, a[1]], v[:, a[0], :, a[1]]
    assert torch.equal(c.table.cpu(), m.table()) and c.length.tolist() == m.len and c.ref.tolist() == m.ref
    assert torch.equal(c.k, k) and torch.equal(c.v, v) and c.stats()["status"] == 0
