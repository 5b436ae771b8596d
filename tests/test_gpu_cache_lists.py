"""Lists of blocks as masks and lists that are followed (GPU): which of the two a step takes, and that bad lists mean the
same to both."""
import random

import pytest
import torch

from tests.blocks_helpers import check_blocks
from tests.test_gpu_cache import DEV, filled
from tests.test_gpu_cache_blocks import MANY, lists_of, some_tokens

pytestmark = pytest.mark.gpu


def followed(cache, x, blocks, tree=None):
    """The call as it is captured before any other of its kind: there is no room for masks, and lists are followed."""
    out = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    before = cache.stats()["launches"]
    with torch.cuda.graph(graph):
        cache.attend_blocks(0, x, blocks, out=out, tree=tree)
    assert cache.stats()["launches"] - before == 1
    graph.replay()
    return out


@pytest.mark.parametrize("name", MANY)
def test_which_path_is_taken(name):
    """Masks and lists add in other orders, so that some of the many results differ in their last bit: nearly all cases
    take the masks (whole query tiles do, so differences are not few), and the one that does not is bit for bit the call
    that follows its lists."""
    shapes, page, ctx, q, n = MANY[name]
    cache, m, x = filled(shapes, page, ctx, q, seed=4)
    blocks = lists_of(m, q, n, shapes[1], fill="some")
    a = followed(cache, x, blocks)
    b = cache.attend_blocks(0, x, blocks)
    check_blocks(cache, m, x, q, blocks, a, 0, tokens=some_tokens(q, 10, 1))
    differ = (a != b).any(1).float().mean()
    assert differ == 0 if name == "followed" else differ > 0.5
    assert cache.stats()["device_error"] == 0


def test_items_that_masks_cannot_tell_are_computed_again():
    """What a list leaves out and is not finite: those tokens are bit for bit what following their lists gives, others are not.
    (Every token lists the other page of the key tile: without a listed key a part of a cut item is dropped, NaN and all.)"""
    shapes, page, ctx, q, n = MANY["page64"]
    cache, m, x = filled(shapes, page, ctx, q, seed=6)
    bad = 5
    cache.v[0, m.own[0][bad], 1, 5, 7] = float("nan")
    blocks = lists_of(m, q, n, 2, fill="some")
    for t in range(q[0]):
        mine = {b for b in blocks[t, 1].tolist()[:n - 1] if b >= 0} | {4}
        blocks[t, 1] = torch.tensor(sorted(mine) + [-1] * (n - len(mine)), dtype=torch.int32, device=DEV)
    a = followed(cache, x, blocks)
    b = cache.attend_blocks(0, x, blocks)
    # Key/value head 1 of sequence 0's tokens, all of which the masks multiply with that value.
    again = slice(0, q[0]), slice(512, 1024)
    assert torch.equal(a[again].view(torch.int16), b[again].view(torch.int16))
    named = (blocks[:q[0], 1] == bad).any(1)
    assert torch.equal(torch.isnan(b[:q[0], 512:].view(-1, 4, 128)[..., 7]).all(1), named) and 0 < int(named.sum()) < q[0]
    assert (a[:, :512] != b[:, :512]).any(1).float().mean() > 0.5
    assert cache.stats()["device_error"] == 0


# Lists, and the pages that they mean: entries that are no whole page before the step, not above the one before them or
# behind a -1 are left out, and a page that is named twice counts once.
BAD = [([5, 3, 5], [5]), ([5, 1, 3, 5], [5, 3]), ([2, 7, 2, 7], [2, 7]), ([-1, 3, 4], []), ([4, -1, 5, 6], [4]), ([-1, -1, 3, 4], []),
       ([9, 4, 3, 4], [9, 4]), ([1, 6, 0, 1, 6, 8], [1, 6, 8]), ([-2, 1, 2, 3, 2, 3], [2, 3]), ([3, 3, 3, 4, 4, 9], [3, 4, 9]),
       ([8, 9, 1 << 30, 2, 9], [8, 9]), ([0, 1, 2, -7, 1, 2, 3], [0, 1, 2, 3])]
LONG = list(range(0, 14)) + [3, 5, 7, 9]             # names pages twice far behind


def padded(lists, n):
    return torch.tensor([x + [-1] * (n - len(x)) for x in lists], dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("shapes,page", [((8, 2, 128), 64), ((4, 1, 64), 16), ((4, 2, 64), 128)])
def test_bad_lists_of_single_tokens(shapes, page):
    """By one CTA to an item, and by clusters, whose CTAs begin in the middle of a list."""
    n, hkv = 18, shapes[1]
    for bad, means in BAD + [(LONG, list(range(14)))]:
        for copies in (1, 160):
            q = [1] * copies
            cache, m, x = filled(shapes, page, [20 * page + 3] * copies, q)
            blocks = lists_of(m, q, n, hkv)
            right = blocks.clone()
            blocks[0, -1], right[0, -1] = padded([bad], n)[0], padded([sorted(means)], n)[0]
            out = cache.attend_blocks(0, x, blocks)
            assert cache.stats(reset=True)["device_error"] == 11, bad
            check_blocks(cache, m, x, q, right, out, 0, tokens={0, copies - 1})
            cache.attend_blocks(0, x, right)
            assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,page", [((8, 2, 128), 64), ((6, 6, 64), 16)])
def test_bad_lists_of_prompts(shapes, page):
    """The same lists as masks and followed."""
    ctx, q, n = [25 * page, 22 * page + 5], [300, 200], 20
    cache, m, x = filled(shapes, page, ctx, q, seed=5)
    blocks = lists_of(m, q, n, shapes[1])
    right = blocks.clone()
    rng, at = random.Random(3), set()
    for t in rng.sample(range(500), 60):
        bad, means = rng.choice(BAD + [(LONG, list(range(14)))])
        h = rng.randrange(shapes[1])
        blocks[t, h], right[t, h] = padded([bad], n)[0], padded([sorted(means)], n)[0]
        at.add(t)
    a = followed(cache, x, blocks)
    assert cache.stats(reset=True)["device_error"] == 11
    b = cache.attend_blocks(0, x, blocks)
    assert cache.stats(reset=True)["device_error"] == 11
    assert (a != b).any(1).float().mean() > 0.5      # (that was by masks)
    check_blocks(cache, m, x, q, right, a, 0, tokens=at)
    check_blocks(cache, m, x, q, right, b, 0, tokens=at)
    again = cache.attend_blocks(0, x, right)         # the same pages in another notation
    assert torch.equal(again, b) and cache.stats()["device_error"] == 0


@pytest.mark.parametrize("q", [1, 300])
def test_entries_behind_as_many_as_there_are_pages(q):
    """A list has at most as many columns as there are whole pages before the step; what else it holds is flagged."""
    cache, m, x = filled((8, 2, 128), 64, [64 * 2 + 7], [q])
    blocks = torch.full((q, 2, 40), -1, dtype=torch.int32, device=DEV)
    blocks[:, :, :2] = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    want = cache.attend_blocks(0, x, blocks)
    assert cache.stats()["device_error"] == 0
    for at in (2, 3, 39):
        bad = blocks.clone()
        bad[q // 2, 1, at] = 1
        out = cache.attend_blocks(0, x, bad)
        assert cache.stats(reset=True)["device_error"] == 11 and torch.equal(out, want)
    fresh, _, y = filled((8, 2, 128), 64, [0], [q])
    fresh.attend_blocks(0, y, torch.zeros((q, 2, 1), dtype=torch.int32, device=DEV))
    assert fresh.stats(reset=True)["device_error"] == 11


def test_long_lists_that_begin_again():
    """More entries than are searched for repeats: those behind them are left out once a list is out of order."""
    page, n = 16, 5000
    cache, m, x = filled((2, 1, 64), page, [6000 * page], [1])
    good = torch.arange(n, dtype=torch.int32, device=DEV).view(1, 1, n)
    check_blocks(cache, m, x, [1], good, cache.attend_blocks(0, x, good), 0)
    bad = good.clone()
    bad[0, 0, 100] = 7                               # 7 is no larger than 99; 101 and what follows are larger than 7
    out = cache.attend_blocks(0, x, bad)
    assert cache.stats(reset=True)["device_error"] == 11
    right = torch.full_like(good, -1)
    right[0, 0, :4095] = torch.tensor(list(range(100)) + list(range(101, 4096)), dtype=torch.int32, device=DEV)
    check_blocks(cache, m, x, [1], right, out, 0)
