"""Workspaces of steps with groups (GPU): they are as large as the largest step of the cache needs, and that step fits."""
import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.test_gpu_cache import DEV, check_attend
from tests.test_gpu_cache_share import fill, grouped

pytestmark = pytest.mark.gpu


def narrow(cache, T_max):
    """The same cache in a handle whose steps have at most T_max tokens."""
    torch.cuda.synchronize()
    return B.PagedCache(cache.k, cache.v, cache.table, cache.length, cache.ref, q_heads=cache.q_heads, T_max=T_max)


CASES = {
    # shapes, page, prefixes, sizes, own tokens (modulus), new tokens
    "one": ((8, 2, 128), 64, [300], [1], 50, lambda s: 1),
    "four": ((32, 8, 128), 64, [700], [4], 50, lambda s: 1),
    "many_cuts": ((4, 1, 64), 16, [9000], [3], 3000, lambda s: 1),
    "pieces_and_line": ((32, 8, 128), 64, [3000, 2000, 1000], [40, 4, 3], 900, lambda s: 1),
    "several": ((8, 2, 128), 32, [1000, 400], [7, 5], 200, lambda s: 1 + s % 4),
    "heads_3": ((9, 3, 64), 16, [1000], [13], 200, lambda s: 1 + s % 3),
    "heads_65": ((65, 1, 128), 64, [700], [5], 70, lambda s: 1 + s % 2),
    "heads_43": ((43, 1, 64), 64, [700, 300], [5, 9], 70, lambda s: 1),
}


@pytest.mark.parametrize("name", CASES)
def test_the_largest_step(name):
    shapes, page, prefixes, sizes, own, new = CASES[name]
    n = sum(sizes)
    wide, m, _, g = grouped(shapes, page, prefixes, sizes, [(s * 37) % own for s in range(n)], slots=8)
    q = [new(s) for s in range(n)]
    cache = narrow(wide, sum(q))
    cache.step(range(n), q)
    assert m.step(range(n), q) is not None
    fill(cache, m, g)
    x = torch.randn((sum(q), shapes[0] * shapes[2]), generator=g, device=DEV).to(torch.bfloat16)
    for counts in (sizes, [n], [1] * n, sizes[::-1]):
        cache.share(counts)
        check_attend(cache, m, x, q, cache.attend(1, x), 1)
    assert cache.stats()["device_error"] == 0


def test_room_for_small_steps():
    """A cache of few sequences takes tens of MB for its groups, not hundreds."""
    wide, m, _, g = grouped((32, 8, 128), 64, [700], [4], [5] * 4, layers=1)
    cache = narrow(wide, 4)
    cache.step(range(4), [1] * 4)
    m.step(range(4), [1] * 4)
    fill(cache, m, g)
    x = torch.randn((4, 4096), generator=g, device=DEV).to(torch.bfloat16)
    cache.attend(0, x)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    cache.share([4])
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] < 64 << 20
    check_attend(cache, m, x, [1] * 4, cache.attend(0, x), 0)
    assert cache.stats()["device_error"] == 0
