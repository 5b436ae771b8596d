"""Infinities and NaN in attention whose sums are joined from parts (GPU): groups with a common prompt and lists that a
cluster shares give what one sum over all keys gives."""
import pytest
import torch

from tests.blocks_helpers import check_blocks
from tests.test_gpu_cache import DEV, check_attend, filled
from tests.test_gpu_cache_blocks import lists_of
from tests.test_gpu_cache_share import fill, grouped

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def spoil(cache, m, x, kind, s, row, layer=0):
    """Sequence s's last position, or the query of row `row` (one head of it)."""
    page, place = m.row(s, m.len[s] - 1)
    k, v = cache.k[layer, page, :, place], cache.v[layer, page, :, place]
    if kind == "query":
        x[row, cache.head_dim:2 * cache.head_dim] = NAN
    elif kind == "query_element":
        x[row, 3] = NAN
    elif kind == "key":
        k[0, 5] = NAN
    elif kind == "value":
        v[:, 7] = NAN
    elif kind == "infinite_key":                     # scores of either infinity, by the sign of the query's element
        k[:, 5] = INF
    else:                                            # a probability of 0 and a value that is none
        k[:, 5] = INF
        x[row].view(-1, cache.head_dim)[:, 5] = -1
        v[:, 7] = NAN


KINDS = ("query", "query_element", "key", "value", "infinite_key", "nothing_times_nan")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes,q", [([4], 1), ([40], 1), ([3, 1, 30], 1), ([6], 2)])
def test_groups(sizes, q, kind):
    """The new tokens are all that sequences hold behind whole common tiles, or nearly all: small groups' pieces, large
    groups' common tiles beside pieces, items of several tokens."""
    n = sum(sizes)
    cache, m, step, g = grouped((8, 2, 128), 64, [256] * len(sizes), sizes, [0] * n)
    step(range(n), [q] * n)
    fill(cache, m, g)
    x = torch.randn((n * q, 1024), generator=g, device=DEV).to(torch.bfloat16)
    spoil(cache, m, x, kind, 1, 2 * q - 1)
    spoil(cache, m, x, kind, n - 1, n * q - 1)
    alone = cache.attend(0, x)
    cache.share(sizes)
    out = cache.attend(0, x)
    check_attend(cache, m, x, [q] * n, out, 0)
    if kind != "nothing_times_nan":                  # (a part of scores of -inf alone is nothing to the call without groups)
        check_attend(cache, m, x, [q] * n, alone, 0)
        assert torch.equal(torch.isnan(out), torch.isnan(alone))
    assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shapes,page,ctx,n", [((8, 2, 128), 64, [448], 7), ((4, 1, 64), 128, [512], 4), ((20, 1, 128), 16, [96], 6),
                                               ((8, 2, 128), 64, [448] * 160, 7)])
def test_blocks(shapes, page, ctx, n, kind):
    """The new token is the only key that is seen in its stage, and in its CTA of a cluster where there is one."""
    q = [1] * len(ctx)
    cache, m, x = filled(shapes, page, ctx, q)
    spoil(cache, m, x, kind, 0, 0)
    blocks = lists_of(m, q, n, shapes[1])
    out = cache.attend_blocks(0, x, blocks)
    check_blocks(cache, m, x, q, blocks, out, 0, tokens={0, len(q) // 2, len(q) - 1})
    if kind != "nothing_times_nan":
        assert torch.equal(torch.isnan(out), torch.isnan(cache.attend(0, x)))
    assert cache.stats()["device_error"] == 0
