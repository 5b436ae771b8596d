"""Bounds that set_bounds replaces (GPU): their memory is not given away before calls on other streams have used them."""
import pytest
import torch

from tests.test_gpu_cache import DEV
from tests.test_gpu_cache_blocks import with_bounds

pytestmark = pytest.mark.gpu

CALLS = {
    "step": lambda c, x, s: c.step([0, 1], [1, 1], stream=s),
    "summarize": lambda c, x, s: c.summarize(0, whole=True, stream=s),
    "select": lambda c, x, s: c.select(0, x, 3, stream=s),
    "accept": lambda c, x, s: c.accept([0], torch.ones(1, dtype=torch.int32, device=DEV),
                                       torch.zeros((1, 1), dtype=torch.int32, device=DEV), stream=s),
    "compact": lambda c, x, s: c.compact(stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_replaced_bounds_wait_for_other_streams(name):
    c, m, x = with_bounds((4, 2, 64), 16, [200, 90], [1, 1])
    c.summarize(0, whole=True)
    new = c.codes.clone(), c.scales.clone()
    a = torch.randn((4096, 4096), device=DEV)
    CALLS[name](c, x, None)                          # (what a first call sets up is there)
    if name == "accept":
        c.step([0, 1], [1, 1])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(200):                         # some 0.1 s
            b = a @ a
    CALLS[name](c, x, s)
    old = c.codes.data_ptr(), c.scales.data_ptr()
    c.set_bounds(*new)
    held = [torch.empty_like(t) for t in new for _ in range(20)]
    assert not s.query()
    assert not {t.data_ptr() for t in held} & set(old)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert torch.isfinite(b).all() and c.stats()["status"] == 0
