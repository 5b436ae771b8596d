"""Plans of the paged cache's attention that ordinary cases seldom reach: each test first says, by the step's rules, that
its sizes give the plan that it is about."""
import pytest
import torch

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
