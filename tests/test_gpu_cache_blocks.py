"""Blocks of the paged cache: bounds of their keys, their selection, attention over chosen ones (GPU) against plain
restatements in float64."""
import random

import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.blocks_helpers import check_blocks, check_bounds, select_ref, unit_of
from tests.cache_helpers import CacheModel
from tests.test_gpu_cache import DEV, check_attend, filled

pytestmark = pytest.mark.gpu


def with_bounds(shapes, page, ctx, q, **kw):
    """``filled`` with bounds, all of them set to values that no call writes."""
    cache, m, x = filled(shapes, page, ctx, q, **kw)
    cache.set_bounds(torch.full(cache.k.shape[:3] + (2, shapes[2]), 77, dtype=torch.int8, device=DEV),
                     torch.full(cache.k.shape[:3], -3.0, device=DEV))
    return cache, m, x


def filled_pages(m, q, whole=False):
    return [p for s, n in enumerate(q) for p in m.own[s][0 if whole else (m.len[s] - n) // m.page:m.len[s] // m.page]]


@pytest.mark.parametrize("shapes,page,ctx,q", [
    ((8, 2, 128), 64, [0, 63, 64, 65, 700, 127], [200, 1, 1, 62, 1, 129]),
    ((3, 3, 64), 16, [0, 15, 16, 31, 100], [1, 1, 1, 0, 45]),
    ((4, 1, 128), 16, [15, 30, 47], [1, 1, 1]),
    ((4, 4, 64), 128, [0, 300], [385, 1]),
    ((2, 2, 128), 32, [(i * 7) % 90 for i in range(90)], [1 + i % 3 for i in range(90)])])
def test_bounds(shapes, page, ctx, q):
    c, m, _ = with_bounds(shapes, page, ctx, q)
    mine = filled_pages(m, q)
    c.summarize(1)
    check_bounds(c, 1, mine)
    others = [p for p in range(c.n_pages) if p not in mine]
    assert (c.codes[1, others] == 77).all() and (c.scales[1, others] == -3.0).all()
    assert (c.codes[0] == 77).all() and (c.scales[0] == -3.0).all()
    c.summarize(0, whole=True)
    check_bounds(c, 0, filled_pages(m, q, whole=True))
    assert c.stats()["status"] == 0


def test_bounds_of_odd_values():
    """Zeros, the smallest and largest numbers, powers of two and their neighbours, infinities and NaN."""
    c, m, _ = with_bounds((1, 1, 64), 16, [0], [16 * 12], poison=False)
    k = c.k[0, m.own[0], 0]
    tiny, big = 2.0 ** -133, 3.3895313892515355e38
    k[0] = 0
    k[1] = 0
    k[1, 3, 5] = -tiny
    k[2] = tiny
    k[3] = big
    k[3, 0, 0] = -big
    k[4] = 127.0
    k[5] = 127.5
    k[6] = -128.0
    k[7] = 1.0
    k[7, 2, 2] = tiny                               # outwards by a whole unit, however small
    k[7, :, 3] = -tiny
    k[8, 1, 1] = float("inf")
    k[9, 2, 63] = float("-inf")
    k[10, 15, 0] = float("nan")
    k[11] = -0.0
    c.k[0, m.own[0], 0] = k
    c.summarize(0)
    check_bounds(c, 0, m.own[0][:12])
    assert c.codes[0, m.own[0][7], 0, :, 2].tolist() == [0 if k[7, :, 2].min() >= 0 else -1, 64]
    assert c.codes[0, m.own[0][7], 0, :, 3].tolist() == [-1, 0]
    assert unit_of(127.0) == 1.0 and unit_of(127.5) == 2.0


def sequence_pages(c, s, length):
    return c.table[s, :length // c.page].tolist()


@pytest.mark.parametrize("page,dh", [(16, 64), (32, 128)])
def test_bounds_follow_accepted_drafts_and_moved_pages(page, dh):
    """Drafts, an accepted path, further tokens, a fork, compaction: what select would read is always right."""
    c = B.PagedCache.empty(2, 60, 4, 2, dh, page, 4, 12, T_max=300, bounds=True)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))

    def check(seqs):
        for s in seqs:
            for layer in (0, 1):
                check_bounds(c, layer, sequence_pages(c, s, int(c.length[s])))

    def step(seq, q):
        c.step(seq, q)
        for layer in (0, 1):
            c.summarize(layer)

    step([0, 1, 3], [3 * page + 5, page - 1, 2 * page])
    check([0, 1, 3])
    step([0, 1], [60, 40])                          # drafts fill pages
    check([0, 1])
    path = torch.tensor([[1, 4, 5, 6] + list(range(20, 56)), list(range(3, 30)) + [0] * 13], dtype=torch.int32, device=DEV)
    c.accept([0, 1], torch.tensor([40, 17], dtype=torch.int32, device=DEV), path)
    assert c.length.tolist()[:2] == [3 * page + 45, page + 16]
    check([0, 1])                                   # whole pages that the path came to lie in
    step([0, 1], [page, 1])
    check([0, 1])
    c.fork([0], [2])
    step([0, 2], [page, page + 3])                  # the shared last page becomes each one's own
    check([0, 1, 2])
    c.truncate([3, 1], [0, 7])
    c.compact()
    step([0, 1, 2], [1, page, 2])
    check([0, 1, 2])
    assert c.stats()["status"] == 0


SELECT = {
    # shapes, page, ctx, q, n, first, last
    "one": ((8, 2, 128), 16, [1000], [1], 9, 1, 1),
    "short": ((8, 2, 128), 64, [0, 63, 64, 500, 640, 641], [1] * 6, 8, 1, 1),
    "none_forced": ((12, 12, 64), 16, [333, 170], [1, 3], 5, 0, 0),
    "all_forced": ((4, 2, 128), 16, [333, 170], [1, 3], 5, 3, 2),
    "single": ((4, 4, 64), 16, [400, 0, 17], [2, 1, 1], 1, 0, 0),
    "heads_20": ((40, 2, 64), 32, [900], [2], 7, 1, 2),
    "heads_128": ((128, 1, 128), 16, [700], [1], 12, 1, 1),
    "chunk": ((8, 2, 128), 16, [700, 90], [40, 33], 6, 1, 1),
    "chunk_runs": ((4, 4, 64), 16, [300, 20, 200, 150, 400], [3, 9, 1, 2, 17], 5, 1, 1),
    "chunk_heads_2": ((4, 2, 128), 16, [300, 200, 400], [3, 8, 14], 5, 0, 1),
    "chunk_heads_3": ((6, 2, 64), 32, [300, 200, 800], [5, 8, 11], 4, 1, 0),
    "chunk_heads_7": ((7, 1, 128), 16, [300, 400], [5, 12], 4, 1, 1),
    "heads_3": ((3, 1, 128), 16, [300, 400], [1, 2], 4, 1, 1),
    "many_blocks": ((4, 1, 64), 16, [20000], [1], 100, 1, 1),
    "some_without_tokens": ((4, 2, 128), 128, [1500, 900, 2000], [1, 0, 1], 3, 1, 1),
}


@pytest.mark.parametrize("name", SELECT)
def test_select(name):
    shapes, page, ctx, q, n, first, last = SELECT[name]
    c, m, x = with_bounds(shapes, page, ctx, q)
    c.summarize(1, whole=True)
    got = c.select(1, x, n, first=first, last=last)
    assert torch.equal(got.cpu(), select_ref(c, m, 1, x, q, n, first, last))
    assert c.stats()["status"] == 0


def test_select_ties_and_odd_scores():
    """Equal blocks: the lower columns; blocks with an infinity come first; a head with a NaN scores 0; all zero."""
    c, m, x = with_bounds((4, 2, 64), 16, [640], [4], poison=False)
    ids = m.own[0]
    c.k[0, ids[:40]] = c.k[0, ids[:1]]                              # 40 equal blocks
    c.k[0, ids[17], 1, 3, 3] = float("inf")
    c.k[0, ids[30]] *= -2
    x[1] = 0
    x[2, :64] = float("nan")
    x[3, 2 * 64:] = float("inf")
    c.summarize(0, whole=True)
    got = c.select(0, x, 6)
    assert torch.equal(got.cpu(), select_ref(c, m, 0, x, [4], 6))
    assert got[1, 0].tolist() == [0, 1, 2, 3, 4, 39] and 17 in got[1, 1].tolist()
    # queries and keys of every magnitude: scores are exact
    c.k[0, ids[:40]] = torch.randn_like(c.k[0, ids[:40]]) * torch.exp2(torch.randint(-40, 40, (40, 2, 1, 1), device=DEV).bfloat16())
    x.copy_(torch.randn_like(x) * torch.exp2(torch.randint(-20, 20, (4, 1), device=DEV).bfloat16()))
    c.summarize(0, whole=True)
    assert torch.equal(c.select(0, x, 11).cpu(), select_ref(c, m, 0, x, [4], 11))


@pytest.mark.parametrize("q", [2, 9])
@pytest.mark.parametrize("n", [5, 60, 200, 390])
def test_select_clustered_scores(q, n):
    """Hundreds of equal blocks, scores in few tight clusters, scores of all magnitudes and both signs, all zero."""
    c, m, x = with_bounds((2, 1, 64), 16, [400 * 16 + 3], [q], poison=False, seed=n)
    ids, g = m.own[0][:400], torch.Generator(device=DEV).manual_seed(n)
    one = torch.randn((1, 1, 16, 64), generator=g, device=DEV).bfloat16()
    kinds = torch.randint(0, 4, (400,), generator=g, device=DEV)
    for keys in (one.expand(400, 1, 16, 64), one * torch.tensor([1.0, 1.0, 1.0078125, -3.0], device=DEV)[kinds].view(-1, 1, 1, 1),
                 one * torch.exp2(torch.randint(-60, 60, (400, 1, 1, 1), generator=g, device=DEV).float()) *
                 torch.randint(-1, 2, (400, 1, 1, 1), generator=g, device=DEV), one * 0):
        c.k[0, ids] = keys.bfloat16()
        c.summarize(0, whole=True)
        assert torch.equal(c.select(0, x, n).cpu(), select_ref(c, m, 0, x, [q], n))
        assert torch.equal(c.select(0, x, n, first=0, last=0).cpu(), select_ref(c, m, 0, x, [q], n, 0, 0))
    assert c.stats()["status"] == 0


def lists_of(m, q, n, kv_heads, seed=0, fill=None):
    """Random ascending columns before the step, -1 behind."""
    rng = random.Random(seed)
    out = []
    for s, new in enumerate(q):
        full = (m.len[s] - new) // m.page
        for _ in range(new):
            for _ in range(kv_heads):
                k = min(full, n if fill is None else rng.randint(0, n))
                out.append(sorted(rng.sample(range(full), k)) + [-1] * (n - k))
    return torch.tensor(out, dtype=torch.int32, device=DEV).view(sum(q), kv_heads, n)


BLOCKS = {
    "one": ((8, 2, 128), 64, [5000], [1], 12),
    "one_page16": ((8, 2, 128), 16, [5000], [1], 50),
    "one_d64": ((12, 12, 64), 32, [3000], [1], 20),
    "edges": ((8, 2, 128), 16, [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129], [1] * 11, 3),
    "edges_page128": ((4, 1, 128), 128, [0, 1, 63, 64, 127, 128, 129, 500], [1] * 8, 2),
    "edges_page64_d64": ((4, 4, 64), 64, [0, 63, 64, 65, 300], [1, 2, 1, 1, 3], 2),
    "no_blocks": ((8, 2, 128), 32, [100, 0, 64], [1, 20, 3], 0),
    "heads_5": ((10, 2, 128), 64, [900, 70], [1, 2], 6),
    "heads_9": ((9, 1, 64), 16, [900], [2], 9),
    "heads_17": ((17, 1, 128), 32, [500], [1], 7),
    "heads_128": ((128, 1, 128), 64, [700], [1], 5),
    "chunk": ((8, 2, 128), 16, [600, 0, 40], [70, 33, 9], 10),
    "chunk_page128": ((4, 2, 64), 128, [1000], [150], 4),
    "some_without_tokens": ((8, 2, 128), 64, [300, 700, 400], [1, 0, 1], 3),
    "batch": ((4, 4, 64), 16, [(i * 37) % 500 for i in range(120)], [1] * 120, 8),
}


@pytest.mark.parametrize("fill", [None, "some"])
@pytest.mark.parametrize("name", BLOCKS)
def test_attend_blocks(name, fill):
    shapes, page, ctx, q, n = BLOCKS[name]
    cache, m, x = filled(shapes, page, ctx, q)
    blocks = lists_of(m, q, n, shapes[1], fill=fill)
    out = cache.attend_blocks(1, x, blocks)
    check_blocks(cache, m, x, q, blocks, out, 1, heads=None if sum(q) < 40 else [0, shapes[1] - 1])
    assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,page", [((8, 2, 128), 64), ((6, 6, 64), 16), ((40, 2, 128), 128)])
def test_attend_blocks_tree(shapes, page):
    ctx, q = [0, 127, 300, 100, 64, 1000], [17, 64, 1, 40, 64, 33]
    cache, m, x = filled(shapes, page, ctx, q, seed=3)
    rng = random.Random(5)
    words = [rng.getrandbits(64) for _ in range(sum(q))]
    words[81] = 0
    words[0] = 0                                     # no prefix, sees nothing
    words[5] = -1 & (1 << 64) - 1                    # bits past the drafts say nothing
    tree = torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)
    blocks = lists_of(m, q, 3, shapes[1], fill="some")
    out = cache.attend_blocks(0, x, blocks, tree=tree)
    check_blocks(cache, m, x, q, blocks, out, 0, tree=words, heads=[0, shapes[1] - 1])
    assert (out[0] == 0).all()
    assert cache.stats()["device_error"] == 0


def test_all_blocks_are_attend():
    """Lists of every page before the step: the same as attend, also with values that are not finite."""
    shapes, page, ctx, q = (8, 2, 128), 32, [700, 33, 512], [5, 1, 30]
    cache, m, x = filled(shapes, page, ctx, q, seed=9)
    cache.v[0, m.own[0][2], 1, 5, 7] = float("inf")
    cache.k[0, m.own[2][3], 0, 1, 1] = float("nan")
    blocks = lists_of(m, q, 30, 2)
    check_attend(cache, m, x, q, cache.attend_blocks(0, x, blocks), 0)
    check_blocks(cache, m, x, q, blocks, cache.attend_blocks(0, x, blocks, scale=0.03), 0, scale=0.03)


# Prompts whose lists are masks of an attention over all pages (many listed positions a token, against the sequence's
# length), and one whose lists are followed.
MANY = {
    "page64": ((8, 2, 128), 64, [1500, 900, 64], [400, 300, 100], 16),
    "page16_d64": ((6, 6, 64), 16, [2000, 37], [200, 50], 80),
    "page32_heads_17": ((17, 1, 128), 32, [2500, 131], [400, 100], 50),
    "page128_d64": ((4, 2, 64), 128, [3000], [700], 12),
    "heads_3": ((6, 2, 128), 16, [1000, 700, 15], [331, 1, 400], 72),
    "windows": ((2, 1, 128), 16, [70000], [128], 800),
    "followed": ((16, 8, 64), 64, [60000], [400], 8),
}


def some_tokens(q, n, seed):
    ends = [e for s in range(len(q)) for e in (sum(q[:s]), sum(q[:s + 1]) - 1)]
    return set(ends) | set(random.Random(seed).sample(range(sum(q)), n))


@pytest.mark.parametrize("fill", [None, "some"])
@pytest.mark.parametrize("name", MANY)
def test_attend_blocks_of_prompts(name, fill):
    shapes, page, ctx, q, n = MANY[name]
    cache, m, x = filled(shapes, page, ctx, q, seed=4)
    blocks = lists_of(m, q, n, shapes[1], fill=fill)
    before = cache.stats()["launches"]
    out = cache.attend_blocks(1, x, blocks)
    assert cache.stats()["launches"] - before == 4
    check_blocks(cache, m, x, q, blocks, out, 1, tokens=some_tokens(q, 40, 1))
    assert torch.equal(cache.attend_blocks(1, x, blocks), out)
    assert cache.stats()["device_error"] == 0


def test_attend_blocks_of_prompts_values_that_are_not_finite():
    """Infinities and NaN reach the tokens whose lists name them, and no others; entries that do not fit are left out."""
    shapes, page, ctx, q, n = MANY["page64"]
    cache, m, x = filled(shapes, page, ctx, q, seed=6)
    cache.v[0, m.own[0][3], 1, 5, 7] = float("inf")
    cache.v[0, m.own[0][4], 0, 63, 100] = float("nan")
    cache.k[0, m.own[0][9], 0, 1, 1] = float("nan")
    cache.k[0, m.own[1][2], 1, 8, 0] = float("inf")
    cache.v[0, m.own[1][15], 1, 2, 3] = float("-inf")           # a new token's
    blocks = lists_of(m, q, n, 2, fill="some")
    out = cache.attend_blocks(0, x, blocks)
    check_blocks(cache, m, x, q, blocks, out, 0, tokens=some_tokens(q, 60, 2))
    assert cache.stats()["device_error"] == 0
    bad = blocks.clone()
    bad[7, 1, :4] = torch.tensor([5, 1, 3, 4], dtype=torch.int32, device=DEV)
    bad[7, 1, 4:] = -1
    out = cache.attend_blocks(0, x, bad)
    assert cache.stats(reset=True)["device_error"] == 11
    bad[7, 1, :4] = torch.tensor([3, 4, 5, -1], dtype=torch.int32, device=DEV)
    check_blocks(cache, m, x, q, bad, out, 0, tokens={6, 7, 8})


def test_attend_blocks_of_a_fresh_prompt():
    """Nothing comes before the step, so that lists are empty: attend, 128 rows at a time."""
    shapes, page, q = (8, 2, 128), 64, [2000, 1, 130]
    cache, m, x = filled(shapes, page, [0, 700, 63], q, seed=8)
    blocks = lists_of(m, q, 20, 2)
    before = cache.stats()["launches"]
    out = cache.attend_blocks(0, x, blocks)
    assert cache.stats()["launches"] - before == 4
    check_blocks(cache, m, x, q, blocks, out, 0, tokens=some_tokens(q, 30, 7))
    assert torch.equal(cache.attend_blocks(0, x, torch.full((sum(q), 2, 0), -1, dtype=torch.int32, device=DEV))[:2000], out[:2000])


def test_attend_blocks_of_prompts_beside_queries_and_with_groups():
    """Results beside the queries in rows of one buffer; steps with groups of sequences."""
    shapes, page, ctx, q, n = MANY["page64"]
    cache, m, x = filled(shapes, page, ctx, q, seed=4)
    cache.v[1, m.own[0][3], 1, 5, 7] = float("nan")
    blocks = lists_of(m, q, n, 2, fill="some")
    eager = cache.attend_blocks(1, x, blocks)
    check_blocks(cache, m, x, q, blocks, eager, 1, tokens=some_tokens(q, 20, 9))
    both = torch.cat([x, torch.zeros_like(x)], 1)
    before = cache.stats()["launches"]
    cache.attend_blocks(1, both[:, :1024], blocks, out=both[:, 1024:])
    assert cache.stats()["launches"] - before == 4
    assert torch.equal(both[:, 1024:].view(torch.int16), eager.view(torch.int16)) and torch.equal(both[:, :1024], x)
    cache.share([2, 1])
    assert torch.equal(cache.attend_blocks(1, x, blocks).view(torch.int16), eager.view(torch.int16))


def test_attend_blocks_of_many_trees():
    shapes, page, ctx, q = (8, 2, 128), 64, [1700 + 91 * i for i in range(8)], [64] * 6 + [33, 50]
    cache, m, x = filled(shapes, page, ctx, q, seed=3)
    rng = random.Random(8)
    words = [rng.getrandbits(64) for _ in range(sum(q))]
    words[70] = 0
    tree = torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)
    blocks = lists_of(m, q, 28, 2, fill="some")
    blocks[70] = -1
    out = cache.attend_blocks(0, x, blocks, tree=tree)
    check_blocks(cache, m, x, q, blocks, out, 0, tree=words, tokens=some_tokens(q, 30, 3) | {70})
    assert cache.stats()["device_error"] == 0


def test_attend_blocks_of_prompts_in_graphs():
    """Captured before any call of that kind (its workspace is not there then) and after one."""
    shapes, page, ctx, q, n = MANY["page64"]
    cache, m, x = filled(shapes, page, ctx, q, seed=4)
    blocks = lists_of(m, q, n, 2)
    outs, counts = [], []
    for _ in range(2):
        out = torch.zeros_like(x)
        g = torch.cuda.CUDAGraph()
        before = cache.stats()["launches"]
        with torch.cuda.graph(g):
            cache.attend_blocks(1, x, blocks, out=out)
        counts.append(cache.stats()["launches"] - before)
        g.replay()
        g.replay()
        outs.append(out)
        eager = cache.attend_blocks(1, x, blocks)
    assert counts == [1, 4]
    for out in outs:
        check_blocks(cache, m, x, q, blocks, out, 1, tokens=some_tokens(q, 20, 5))
    assert torch.equal(outs[1], eager)


def test_a_single_seen_key_gives_its_value():
    cache, m, x = filled((8, 2, 128), 16, [160], [3], seed=2)
    tree = torch.tensor([1, 2, 4], device=DEV)
    out = cache.attend_blocks(0, x, torch.full((3, 2, 4), -1, dtype=torch.int32, device=DEV), tree=tree)
    v = cache.v[0, m.own[0][10], :, :3]
    assert torch.equal(out.view(3, 2, 4, 128), v.transpose(0, 1)[:, :, None].expand(3, 2, 4, 128))


def test_bad_lists_are_flagged():
    """Entries that do not fit are left out and reported; the others count."""
    shapes, page, ctx, q = (4, 2, 64), 16, [100, 40], [1, 1]
    cache, m, x = filled(shapes, page, ctx, q)
    good = lists_of(m, q, 4, 2)
    for bad, fits in (([0, 6, 7, 8], [0, -1, -1, -1]), ([2, 2, 3, -1], [2, 3, -1, -1]), ([5, 1, 3, 4], [5, 3, 4, -1]),
                      ([-2, 1, 2, 3], [2, 3, -1, -1]), ([1 << 30, -1, -1, -1], [-1] * 4), ([-1, -1, 3, -1], [-1] * 4)):
        blocks = good.clone()
        blocks[0, 1] = torch.tensor(bad, dtype=torch.int32, device=DEV)
        out = cache.attend_blocks(0, x, blocks)
        st = cache.stats(reset=True)
        assert st["status"] == -7 and st["device_error"] == 11, bad
        blocks[0, 1] = torch.tensor(fits, dtype=torch.int32, device=DEV)
        check_blocks(cache, m, x, q, blocks, out, 0)
        assert cache.stats()["status"] == 0


def test_strides_and_outputs():
    """Rows of wider buffers, results into the caller's tensors, what lies beside them untouched."""
    shapes, page, ctx, q = (8, 2, 64), 32, [300, 500], [2, 1]
    c, m, x = with_bounds(shapes, page, ctx, q)
    c.summarize(0, whole=True)
    wide = torch.full((3, 704), 9.0, dtype=torch.bfloat16, device=DEV)
    wide[:, 64:576] = x
    blocks = torch.empty((3, 2, 5), dtype=torch.int32, device=DEV)
    assert c.select(0, wide[:, 64:576], 5, out=blocks) is blocks
    assert torch.equal(blocks.cpu(), select_ref(c, m, 0, x, q, 5))
    out = torch.full((4, 600), 7.0, dtype=torch.bfloat16, device=DEV)
    c.attend_blocks(0, wide[:, 64:576], blocks, out=out[:3, 40:552])
    check_blocks(c, m, x, q, blocks, out[:3, 40:552], 0)
    assert (out[3] == 7).all() and (out[:, :40] == 7).all() and (out[:, 552:] == 7).all()
    with pytest.raises(B.TrimmoeError, match="multiples of 8"):
        c.attend_blocks(0, x, blocks, out=torch.empty((3, 517), dtype=torch.bfloat16, device=DEV)[:, :512])


def test_refusals():
    c, m, x = with_bounds((4, 2, 64), 16, [100], [2])
    good = lists_of(m, [2], 3, 2)
    bare, _, _ = filled((4, 2, 64), 16, [100], [2])
    for call, word in ((lambda: bare.summarize(0), "no bounds"), (lambda: bare.select(0, x, 3), "no bounds"),
                       (lambda: c.summarize(2), "layer"), (lambda: c.select(-1, x, 3), "layer"),
                       (lambda: c.select(0, x, 0), "n must"), (lambda: c.select(0, x, 3, first=2, last=2), "n must"),
                       (lambda: c.select(0, x, 3, first=-1), "n must"), (lambda: c.select(0, x[:1], 3), "shape"),
                       (lambda: c.select(0, x, 3, out=good[:, :, :2].contiguous()), "shape"),
                       (lambda: c.attend_blocks(0, x, good[:1]), "blocks"), (lambda: c.attend_blocks(0, x, good.long()), "int32"),
                       (lambda: c.attend_blocks(0, x, good.transpose(0, 2)), "blocks"),
                       (lambda: c.attend_blocks(0, x, good, scale=-1.0), "scale"),
                       (lambda: c.attend_blocks(5, x, good), "layer"), (lambda: c.set_bounds(c.codes, None), "together"),
                       (lambda: B.PagedCache(c.k, c.v, c.table, c.length, c.ref, 4, 8, bounds=(c.codes[0], c.scales)), "shape"),
                       (lambda: B.PagedCache(c.k, c.v, c.table, c.length, c.ref, 4, 8, bounds=(c.codes, c.scales.half())), "float32")):
        with pytest.raises(B.TrimmoeError, match=word):
            call()
    c.fork([0], [1])
    for call in (lambda: c.summarize(0), lambda: c.select(0, x, 3), lambda: c.attend_blocks(0, x, good)):
        with pytest.raises(B.TrimmoeError, match="no step"):
            call()


def test_a_refused_step_and_a_step_without_tokens():
    """Behind a step without room nothing is written; a step of no tokens has empty results."""
    c, m, x = with_bounds((4, 2, 64), 16, [100], [2])
    c.summarize(0, whole=True)
    codes = c.codes.clone()
    c.step([0], [2])
    full = B.PagedCache.empty(1, 4, 4, 2, 64, 16, 2, 3, T_max=100, bounds=True)
    full.step([0], [40])
    full.step([0], [60])                            # more than max_pages
    y = torch.randn((60, 256), device=DEV).bfloat16()
    blocks, out = torch.full((60, 2, 3), 5, dtype=torch.int32, device=DEV), torch.full((60, 256), 3.0, device=DEV).bfloat16()
    full.codes.fill_(4)
    full.summarize(0)
    full.select(0, y, 3, out=blocks)
    full.attend_blocks(0, y, blocks, out=out)
    assert (blocks == 5).all() and (out == 3).all() and (full.codes == 4).all()
    assert full.stats(reset=True)["device_error"] == 8
    full.step([0, 1], [0, 0])
    e = torch.empty((0, 256), dtype=torch.bfloat16, device=DEV)
    full.summarize(0)
    b = full.select(0, e, 3)
    assert b.shape == (0, 2, 3) and full.attend_blocks(0, e, b).shape == (0, 256)
    full.step([], [])
    full.summarize(0, whole=True)
    assert full.stats()["status"] == 0


def test_graph_and_streams():
    """Step, bounds, selection and attention in one captured graph, replayed on new lengths; a call on another stream."""
    shapes, page = (8, 2, 128), 16
    c = B.PagedCache.empty(1, 80, 8, 2, 128, page, 2, 30, T_max=400, bounds=True)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))
    m = CacheModel(80, 2, 30, page)
    assert m.step([0, 1], [200, 150]) == []
    c.step([0, 1], [200, 150])
    c.summarize(0)
    x = torch.randn((2, 1024), device=DEV).bfloat16()
    blocks, out = torch.empty((2, 2, 5), dtype=torch.int32, device=DEV), torch.empty((2, 1024), dtype=torch.bfloat16, device=DEV)

    def step():
        c.step([0, 1], [1, 1])
        c.summarize(0)
        c.select(0, x, 5, out=blocks)
        c.attend_blocks(0, x, blocks, out=out)

    step()
    m.step([0, 1], [1, 1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(30):
        x.copy_(torch.randn_like(x))
        g.replay()
        m.step([0, 1], [1, 1])
        if i % 7 == 3:
            assert torch.equal(blocks.cpu(), select_ref(c, m, 0, x, [1, 1], 5))
            check_blocks(c, m, x, [1, 1], blocks, out, 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = c.select(0, x, 5, stream=s)
    o = c.attend_blocks(0, x, b, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(b, blocks) and torch.equal(o, out)
    assert c.stats()["status"] == 0


def test_results_do_not_depend_on_timing():
    shapes, page, ctx, q = (8, 2, 128), 64, [3000, 5000, 100], [1, 1, 1]
    c, m, x = with_bounds(shapes, page, ctx, q)
    c.summarize(1, whole=True)
    b = c.select(1, x, 12)
    first = c.attend_blocks(1, x, b)
    for _ in range(20):
        assert torch.equal(c.select(1, x, 12), b) and torch.equal(c.attend_blocks(1, x, b), first)
