"""Attention of sequences that share a prompt (GPU) against plain restatements in float64."""
import random

import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.cache_helpers import CacheModel
from tests.test_gpu_cache import DEV, check_attend

pytestmark = pytest.mark.gpu


def grouped(shapes, page, prefixes, sizes, own, layers=2, seed=0, T_max=4096, slots=0):
    """A cache whose groups of sizes[g] sequences were forked from a prompt of prefixes[g] tokens and then got own[s]
    further tokens each, with random keys and values; places that no position uses hold NaN."""
    hq, hkv, dh = shapes
    n = sum(sizes)
    total = [p + o for p, o in zip([p for p, k in zip(prefixes, sizes) for _ in range(k)], own)]
    width = max(total) // page + 8 + slots
    n_pages = sum(-(-p // page) for p in prefixes) + sum(-(-o // page) + 3 + slots for o in own) + 8
    cache = B.PagedCache.empty(layers, n_pages, hq, hkv, dh, page, n, width, T_max=max(T_max, sum(prefixes), sum(own)))
    m = CacheModel(n_pages, n, width, page)
    heads = [sum(sizes[:g]) for g in range(len(sizes))]

    def step(seq, q):
        cache.step(seq, q)
        assert m.step(seq, q) is not None

    step(heads, prefixes)
    for a, k in zip(heads, sizes):
        if k > 1:
            cache.fork([a] * (k - 1), range(a + 1, a + k))
            m.fork([a] * (k - 1), range(a + 1, a + k))
    if any(own):
        step(range(n), own)
    return cache, m, step, torch.Generator(device=DEV).manual_seed(seed)


def fill(cache, m, g):
    """Random keys and values at every position, NaN elsewhere."""
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    for s in range(len(m.own)):
        for j, p in enumerate(m.own[s]):
            e = min(m.page, m.len[s] - j * m.page)
            for pool in (cache.k, cache.v):
                pool[:, p, :, :e] = torch.randn(pool[:, p, :, :e].shape, generator=g, device=DEV).to(torch.bfloat16)
    assert cache.table.tolist() == m.table().tolist() and cache.length.tolist() == m.len


CASES = {
    # shapes, page, prefixes, sizes, own tokens (modulus), new tokens
    "four": ((8, 2, 128), 64, [700], [4], 50, lambda s: 1),
    "below_a_tile": ((8, 2, 128), 16, [100], [5], 9, lambda s: 1),
    "tile_edges": ((4, 1, 128), 16, [127, 128, 129, 256], [3, 3, 3, 3], 2, lambda s: 1),
    "just_forked": ((8, 2, 64), 64, [500], [6], 1, lambda s: 1),
    "groups": ((8, 2, 128), 32, [1000, 50, 3000, 300], [7, 1, 2, 20], 400, lambda s: 1),
    "one_head_each": ((12, 12, 64), 16, [600, 200], [40, 3], 60, lambda s: 1),
    "many_rows": ((32, 2, 128), 128, [900], [70], 130, lambda s: 1),
    "ragged_new": ((8, 2, 128), 64, [513], [9], 200, lambda s: [0, 1, 5, 33, 70, 2, 0, 129, 300][s]),
    "heads_7": ((7, 1, 64), 16, [300], [11], 33, lambda s: 1 + s % 4),
    "heads_65": ((65, 1, 128), 64, [400], [5], 70, lambda s: 1 + s % 2),
    "heads_128": ((128, 1, 64), 64, [260], [4], 10, lambda s: 1),
    "no_groups": ((8, 2, 128), 64, [300, 5, 128, 1000], [1, 1, 1, 1], 7, lambda s: 1 + s),
    "large_groups": ((4, 4, 128), 64, [2000], [300], 100, lambda s: 1),
    "small_groups": ((8, 2, 128), 16, [1500, 300, 4000, 130], [4, 8, 3, 9], 300, lambda s: 1),
    "small_and_large": ((12, 12, 64), 32, [5000, 2000, 700], [50, 16, 31], 900, lambda s: 1),
    "one_far_longer": ((4, 2, 128), 64, [200, 20000], [5, 1], 30, lambda s: 1),
    "heads_3": ((9, 3, 64), 128, [700, 500], [4, 11], 200, lambda s: 1),
    "heads_16": ((16, 1, 128), 64, [2500, 400], [2, 3], 70, lambda s: 1),
    "many_sequences": ((4, 2, 64), 16, [300, 130] * 30, [5, 12] * 30, 60, lambda s: int(s % 7 != 0)),
    "all_idle_but_one": ((8, 2, 128), 64, [700], [4], 50, lambda s: int(s == 2)),
    "ragged_few": ((8, 2, 128), 64, [513], [40], 200, lambda s: 129 if s == 3 else s % 8),
    "ragged_few_d64": ((12, 12, 64), 32, [900, 300], [12, 5], 100, lambda s: 1 + s * 3 % 11),
    "ragged_few_heads_7": ((14, 2, 128), 16, [2000, 130], [30, 12], 300, lambda s: 1 + s % 4),
    "first_idle": ((8, 2, 128), 64, [700, 400], [4, 3], 50, lambda s: int(s not in (0, 1, 4))),
}


@pytest.mark.parametrize("name", CASES)
def test_attend_shared(name):
    shapes, page, prefixes, sizes, own, new = CASES[name]
    n = sum(sizes)
    cache, m, step, g = grouped(shapes, page, prefixes, sizes, [(s * 37) % own for s in range(n)], slots=8)
    q = [new(s) for s in range(n)]
    step(range(n), q)
    fill(cache, m, g)
    x = (torch.randn((sum(q), shapes[0] * shapes[2]), generator=g, device=DEV) * 1.4).to(torch.bfloat16)
    cache.share(sizes)
    for layer in (0, 1):
        out = cache.attend(layer, x)
        check_attend(cache, m, x, q, out, layer)
        assert torch.equal(out, cache.attend(layer, x))
    assert cache.stats()["device_error"] == 0
    step(range(n), [1] * n)                          # a step without groups is as before
    fill(cache, m, g)
    x = x[:1].expand(n, -1).contiguous()
    check_attend(cache, m, x, [1] * n, cache.attend(0, x), 0)
    assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("large", [False, True])
@pytest.mark.parametrize("shapes,page", [((8, 2, 128), 64), ((6, 6, 64), 16), ((40, 5, 128), 128)])
def test_attend_shared_tree(shapes, page, large):
    """Large trees fill query tiles by themselves (but with one query head each) and are attended as without groups."""
    sizes, q = ([3, 4], [17, 64, 1, 40, 64, 33, 2]) if large else ([6, 9], [5, 12, 1, 9, 3, 12, 8, 2, 11, 4, 12, 1, 6, 7, 3])
    n = sum(sizes)
    cache, m, step, g = grouped(shapes, page, [400, 131], sizes, [(s * 40) % 101 for s in range(n)], slots=8)
    step(range(n), q)
    fill(cache, m, g)
    x = torch.randn((sum(q), shapes[0] * shapes[2]), generator=g, device=DEV).to(torch.bfloat16)
    rng = random.Random(5)
    words = [rng.getrandbits(64) for _ in range(sum(q))]
    words[0] = 0
    tree = torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)
    before = cache.stats()["launches"]
    cache.share(sizes)
    assert cache.stats()["launches"] - before == (0 if large and shapes[0] > shapes[1] else 2)
    check_attend(cache, m, x, q, cache.attend(1, x, tree=tree), 1, tree=words)
    check_attend(cache, m, x, q, cache.attend(1, x, tree=tree, scale=0.05), 1, tree=words, scale=0.05)
    assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,sizes", [((8, 2, 128), [3, 1, 30]), ((12, 12, 64), [20, 2]), ((40, 2, 64), [3, 4])])
def test_single_tokens_by_their_masks(shapes, sizes):
    """A mask without the token's own bit shows it the positions before the step alone."""
    n = sum(sizes)
    cache, m, step, g = grouped(shapes, 16, [300] * len(sizes), sizes, [s % 40 for s in range(n)], slots=8)
    q = [int(s != 1) for s in range(n)]
    step(range(n), q)
    fill(cache, m, g)
    for s in range(n):                               # the new key and value may hold anything when nobody sees them
        if q[s] and s % 3 == 0:
            page, place = m.row(s, m.len[s] - 1)
            cache.k[1, page, :, place] = float("nan")
            cache.v[1, page, :, place] = float("inf")
    words = [int(s % 3 != 0) | (s % 2) << 5 for s in range(n) if q[s]]
    x = torch.randn((sum(q), shapes[0] * shapes[2]), generator=g, device=DEV).to(torch.bfloat16)
    cache.share(sizes)
    check_attend(cache, m, x, q, cache.attend(1, x, tree=torch.tensor(words, device=DEV)), 1, tree=words)
    assert cache.stats()["device_error"] == 0


def test_in_place_of_wider_rows_and_another_stream():
    """Queries and results in rows of wider buffers; share and attend on another stream."""
    cache, m, step, g = grouped((8, 2, 64), 32, [400, 90], [40, 3], [s % 70 for s in range(43)], slots=8)
    step(range(43), [1] * 43)
    fill(cache, m, g)
    wide = torch.randn((43, 1024), generator=g, device=DEV).to(torch.bfloat16)
    out = torch.full((43, 776), 5.0, device=DEV).bfloat16()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    cache.share([40, 3], stream=s)
    cache.attend(0, wide[:, 256:768], out=out[:, 128:640], stream=s)
    torch.cuda.current_stream().wait_stream(s)
    check_attend(cache, m, wide[:, 256:768].contiguous(), [1] * 43, out[:, 128:640], 0)
    assert (out[:, :128] == 5).all() and (out[:, 640:] == 5).all()
    assert cache.stats()["device_error"] == 0


def test_values_that_are_not_finite():
    """In the common part they reach every row that sees them, in masked places none."""
    cache, m, step, g = grouped((8, 2, 128), 32, [400], [5], [3, 40, 7, 0, 70])
    step(range(5), [2] * 5)
    fill(cache, m, g)
    cache.v[0, m.own[0][1], 1, 3, 9] = float("inf")
    cache.k[0, m.row(2, m.len[2] - 1)[0], 0, (m.len[2] - 1) % 32] = float("nan")
    cache.v[0, m.row(1, m.len[1] - 1)[0], :, (m.len[1] - 1) % 32] = float("-inf")
    x = torch.randn((10, 1024), generator=g, device=DEV).to(torch.bfloat16)
    cache.share([5])
    check_attend(cache, m, x, [2] * 5, cache.attend(0, x), 0)
    assert cache.stats()["device_error"] == 0


def test_groups_that_share_nothing():
    """Counts are a hint: sequences without a common prompt, or whose pages part in the middle, are attended as they are."""
    cache, m, step, g = grouped((8, 2, 64), 16, [500, 300, 700], [2, 1, 3], [5, 0, 9, 30, 80, 1])
    cache.truncate([4], [140])                       # shares 8 pages of 16 with its group from here on
    m.truncate([4], [140])
    step([4], [300])
    step(range(6), [1] * 6)
    fill(cache, m, g)
    x = torch.randn((6, 512), generator=g, device=DEV).to(torch.bfloat16)
    for counts in ([6], [2, 1, 3], [1, 2, 3], [1] * 6, [3, 3]):
        cache.share(counts)
        check_attend(cache, m, x, [1] * 6, cache.attend(0, x), 0)
    assert cache.stats()["device_error"] == 0


def test_more_rows_than_groups_are_made_for():
    """65536 query rows and one more token: with groups, then as without."""
    for last in (16, 17):
        q = [16] * 255 + [last]
        cache, m, step, g = grouped((16, 16, 64), 64, [200], [256], [0] * 256, slots=2, layers=1, T_max=4097)
        step(range(256), q)
        fill(cache, m, g)
        x = torch.randn((sum(q), 16 * 64), generator=g, device=DEV).to(torch.bfloat16)
        before = cache.stats()["launches"]
        cache.share([256])
        assert cache.stats()["launches"] - before == (2 if last == 16 else 0)
        check_attend(cache, m, x, q, cache.attend(0, x), 0)
        assert cache.stats()["device_error"] == 0


def test_refusals():
    cache, m, step, g = grouped((8, 2, 64), 16, [50], [3], [0] * 3)
    with pytest.raises(B.TrimmoeError, match="no step|n out of range|add up"):
        cache.share([2])
    step(range(3), [1] * 3)
    for counts, word in (([2], "add up"), ([4], "add up"), ([3, 0], "counts"), ([1, 1, 1, 0], "n out of range"), ([], "add up"),
                         ([4, -1], "counts"), ([1.5], "integers")):
        with pytest.raises(B.TrimmoeError, match=word):
            cache.share(counts)
    cache.share([3])
    cache.truncate([0], [2])
    with pytest.raises(B.TrimmoeError, match="no step"):
        cache.share([3])
    cache.step([], [])
    cache.share([])
    assert cache.stats()["status"] == 0


def test_first_call_in_a_capture_is_refused():
    cache, m, step, g = grouped((8, 2, 64), 16, [300], [3], [0] * 3)
    step(range(3), [1] * 3)
    fill(cache, m, g)
    x = torch.randn((3, 512), generator=g, device=DEV).to(torch.bfloat16)
    before = cache.attend(0, x)
    graph, y = torch.cuda.CUDAGraph(), x * 1
    with torch.cuda.graph(graph):
        y += 1
        with pytest.raises(B.TrimmoeError, match="captured"):
            cache.share([3])
    assert torch.equal(cache.attend(0, x), before)   # the step is what it was
    cache.share([3])
    check_attend(cache, m, x, [1] * 3, cache.attend(0, x), 0)


def test_graph_replays_on_new_lengths():
    """Step, share and attend captured; the replays find the common pages of the lengths that they meet."""
    cache, m, step, g = grouped((8, 2, 128), 16, [150], [4], [0, 3, 7, 1], layers=1, slots=8)
    x = torch.randn((4, 1024), generator=g, device=DEV).to(torch.bfloat16)
    out = torch.empty_like(x)
    cache.step(range(4), [1] * 4)
    m.step(range(4), [1] * 4)
    cache.share([4])
    for pool in (cache.k, cache.v):                  # also where no position is yet
        pool.copy_(torch.randn(pool.shape, generator=g, device=DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.step(range(4), [1] * 4)
        cache.share([4])
        cache.attend(0, x, out=out)
    for i in range(20):
        graph.replay()
        m.step(range(4), [1] * 4)
        if i % 6 == 0:
            check_attend(cache, m, x, [1] * 4, out, 0)
        if i == 8:                                   # the prompt is dropped: nothing in common any more
            cache.truncate(range(4), [0] * 4)
            m.truncate(range(4), [0] * 4)
    assert cache.stats()["device_error"] == 0


def test_a_captured_attend_of_another_step():
    """An attend captured with groups reads the list of its share: replayed behind a step without one it is
    refused and leaves its output; plain attends captured before are as they were."""
    cache, m, step, g = grouped((8, 2, 128), 16, [300], [4], [0, 3, 7, 1], slots=8)
    step(range(4), [1] * 4)
    x = torch.randn((4, 1024), generator=g, device=DEV).to(torch.bfloat16)
    plain, out = torch.empty_like(x), torch.empty_like(x)
    cache.attend(0, x)
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        cache.attend(0, x, out=plain)
    cache.share([4])
    with torch.cuda.graph(two):
        cache.attend(0, x, out=out)
    for again in (True, False):
        fill(cache, m, g)
        out.fill_(3)
        one.replay()
        two.replay()
        check_attend(cache, m, x, [1] * 4, plain, 0)
        if again:
            check_attend(cache, m, x, [1] * 4, out, 0)
            assert cache.stats()["device_error"] == 0
            step(range(4), [1] * 4)                  # and no share
    assert (out == 3).all() and cache.stats(reset=True)["device_error"] == 9
    cache.share([4])
    two.replay()
    check_attend(cache, m, x, [1] * 4, out, 0)
    assert cache.stats()["device_error"] == 0


def test_a_refused_step():
    cache, m, step, g = grouped((8, 2, 64), 16, [300], [3], [0] * 3)
    step(range(3), [1] * 3)
    cache.share([3])
    cache.step(range(3), [1, 1, 4000])
    out = torch.full((4002, 512), 3.0, device=DEV).bfloat16()
    assert cache.stats()["device_error"] == 8
    cache.step(range(3), [1, 1, 1000])
    cache.share([3])
    cache.attend(0, out[:1002] * 2, out=out[:1002])
    assert (out == 3).all() and cache.stats(reset=True)["device_error"] == 8
    step(range(3), [1] * 3)
    fill(cache, m, g)
    x = torch.randn((3, 512), generator=g, device=DEV).to(torch.bfloat16)
    cache.share([3])
    check_attend(cache, m, x, [1] * 3, cache.attend(0, x), 0)
