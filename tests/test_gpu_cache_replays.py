"""Attends with groups that were captured, replayed behind steps with other groups (GPU)."""
import pytest
import torch

from tests.test_gpu_cache import DEV, check_attend
from tests.test_gpu_cache_share import fill, grouped

pytestmark = pytest.mark.gpu


def captured(cache, x):
    out = torch.full_like(x, 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(0, x, out=out)
    return graph, out


SMALL, LARGE = [8] * 5 + [3], [40, 3]


def test_small_groups_replayed_behind_a_large_one():
    """The launches of small groups alone leave common tiles out that large groups have: refused, the output and the
    step's own attends are as they were."""
    cache, m, step, g = grouped((8, 2, 128), 64, [2000, 300], LARGE, [s % 60 for s in range(43)], slots=8)
    step(range(43), [1] * 43)
    fill(cache, m, g)
    x = torch.randn((43, 1024), generator=g, device=DEV).to(torch.bfloat16)
    cache.share(SMALL)
    cache.attend(0, x)
    graph, out = captured(cache, x)
    graph.replay()
    check_attend(cache, m, x, [1] * 43, out, 0)
    step(range(43), [1] * 43)
    fill(cache, m, g)
    out.fill_(3)
    cache.share(LARGE)
    graph.replay()
    st = cache.stats(reset=True)
    assert (out == 3).all() and st["device_error"] == 9
    for _ in range(2):                               # the refused one has drawn nothing of the list
        check_attend(cache, m, x, [1] * 43, cache.attend(0, x), 0)
    cache.share(SMALL)
    graph.replay()
    check_attend(cache, m, x, [1] * 43, out, 0)
    assert cache.stats()["device_error"] == 0


def test_large_groups_replayed_behind_small_ones():
    """The launches of large groups compute all that small ones need."""
    cache, m, step, g = grouped((8, 2, 128), 64, [2000, 300], LARGE, [s % 60 for s in range(43)], slots=8)
    step(range(43), [1] * 43)
    fill(cache, m, g)
    x = torch.randn((43, 1024), generator=g, device=DEV).to(torch.bfloat16)
    cache.share(LARGE)
    cache.attend(0, x)
    graph, out = captured(cache, x)
    for counts in (SMALL, [1] * 43, [43], LARGE):
        out.fill_(3)
        cache.share(counts)
        graph.replay()
        check_attend(cache, m, x, [1] * 43, out, 0)
        assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("single_first", [False, True])
def test_other_counts_of_tokens(single_first):
    """Single tokens' launches and those of several tokens do not stand for each other, nor do steps of fewer tokens."""
    cache, m, step, g = grouped((8, 2, 128), 64, [700], [8], [0] * 8, slots=8)
    kinds = [(range(8), [1] * 8, [8]), (range(4), [2] * 4, [4])]
    first, second = kinds if single_first else kinds[::-1]
    step(*first[:2])
    fill(cache, m, g)
    x = torch.randn((8, 1024), generator=g, device=DEV).to(torch.bfloat16)
    cache.share(first[2])
    before = cache.attend(0, x)
    graph, out = captured(cache, x)
    graph.replay()
    assert torch.equal(out, before)
    for seq, q, counts in (second, (range(6), [1] * 6, [6]) if single_first else (range(3), [2] * 3, [3])):
        step(seq, q)
        fill(cache, m, g)
        cache.share(counts)
        out.fill_(3)
        graph.replay()
        assert cache.stats(reset=True)["device_error"] == 9 and (out == 3).all()
        lens = [0] * 8
        for s, k in zip(seq, q):
            lens[s] = k
        rows = x[:sum(q)].contiguous()
        check_attend(cache, m, rows, lens, cache.attend(0, rows), 0)
    assert cache.stats()["device_error"] == 0
