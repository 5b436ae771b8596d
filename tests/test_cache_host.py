"""Paged cache: what can be checked without a GPU."""
import ctypes as C
import os
import random
import re
import subprocess
import tempfile

import pytest

from paper_2608_00573_gb300 import binding as B
from paper_2608_00573_gb300 import build as BUILD
from tests.cache_helpers import CacheModel

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    BUILD.build()
    return B._cache_lib()


def test_struct_sizes_match_the_header():
    names = ("trimmoe_cache_config", "trimmoe_cache_state", "trimmoe_append_args", "trimmoe_attend_args",
             "trimmoe_cache_stats_t")
    src = '#include <stdio.h>\n#include "trimmoe.h"\nint main(){%s}\n' % "".join(
        'printf("%%zu ", sizeof(%s));' % n for n in names)
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "s.c"), "w") as f:
            f.write(src)
        exe = os.path.join(d, "s")
        subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), os.path.join(d, "s.c"), "-o", exe])
        got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [C.sizeof(getattr(B, n)) for n in names]


def test_error_codes_match_the_header():
    with open(os.path.join(ROOT, "include", "trimmoe.h")) as f:
        h = f.read()
    codes = {k: int(v) for k, v in re.findall(r"TRIMMOE_(DEVERR_\w+|ERR_CACHE) = (-?\d+)", h)}
    assert codes["ERR_CACHE"] == -7 and B.STATUS_NAMES[-7] == "ERR_CACHE"
    assert [codes["DEVERR_CACHE_" + n] for n in ("ATTENTION", "FULL", "STATE", "PATH")] == [7, 8, 9, 10]


GOOD = dict(layers=2, q_heads=8, kv_heads=2, head_dim=64, page_size=16, n_pages=8, max_seqs=4, max_pages=4, T_max=64)


def create(lib, st=None, **over):
    cfg = B.trimmoe_cache_config(**{**GOOD, **over})
    p = 0x1000                                     # never read: validation fails first
    st = st or B.trimmoe_cache_state(k=p, v=p, table=p, length=p, ref=p)
    out = C.c_void_p(1)
    rc = lib.trimmoe_cache_create(C.byref(cfg), C.byref(st), C.byref(out))
    assert rc != 0 and not out.value
    return rc, B.trimmoe_last_error(None)


@pytest.mark.parametrize("over,status,word", [
    (dict(layers=0), -1, ">= 1"), (dict(T_max=0), -1, ">= 1"), (dict(max_seqs=-1), -1, ">= 1"),
    (dict(q_heads=9), -1, "multiple"), (dict(head_dim=96), -2, "head_dim"), (dict(page_size=8), -2, "page_size"),
    (dict(page_size=48), -2, "page_size"), (dict(q_heads=258), -2, "<= 128"), (dict(q_heads=8192, kv_heads=8192), -2, "4096"),
    (dict(max_seqs=1025), -2, "max_seqs"), (dict(T_max=(1 << 20) + 1), -2, "T_max"),
    (dict(n_pages=1 << 26), -2, "2^31"), (dict(max_pages=1 << 27), -2, "2^31")])
def test_create_refuses(lib, over, status, word):
    rc, msg = create(lib, **over)
    assert rc == status and word in msg and msg.startswith("cache_create")


def test_create_refuses_missing_and_misaligned_state(lib):
    p = 0x1000
    for field in ("k", "v", "table", "length", "ref"):
        rc, msg = create(lib, B.trimmoe_cache_state(**{**dict(k=p, v=p, table=p, length=p, ref=p), field: None}))
        assert rc == -1 and "NULL" in msg
    rc, msg = create(lib, B.trimmoe_cache_state(k=p + 8, v=p, table=p, length=p, ref=p))
    assert rc == -1 and "aligned" in msg
    assert lib.trimmoe_cache_create(None, None, None) == -1


def test_calls_without_a_handle_are_refused(lib):
    s = B.trimmoe_cache_stats_t()
    assert lib.trimmoe_cache_step(None, 0, None, None, None) == -1
    assert lib.trimmoe_cache_append(None, 0, None, None) == -1
    assert lib.trimmoe_cache_attend(None, 0, None, None) == -1
    assert lib.trimmoe_cache_fork(None, 0, None, None, None) == -1
    assert lib.trimmoe_cache_truncate(None, 0, None, None, None) == -1
    assert lib.trimmoe_cache_accept(None, 0, None, None, None, 0, None) == -1
    assert lib.trimmoe_cache_compact(None, None) == -1
    assert lib.trimmoe_cache_stats(None, C.byref(s), 0) == -1
    assert lib.trimmoe_cache_last_error(None) == b""
    lib.trimmoe_cache_destroy(None)


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(B.TrimmoeError, match="GPU"):
        B.PagedCache.empty(1, 4, 2, 1, 64, 16, 2, 4, 8, device="cpu")
    with pytest.raises(B.TrimmoeError, match="layers"):
        B.PagedCache(torch.zeros(3), torch.zeros(3), torch.zeros(3), torch.zeros(3), torch.zeros(3), 1, 1)


@pytest.mark.parametrize("seed", range(4))
def test_the_model_of_the_tests_keeps_its_invariants(seed):
    """Counts equal holders, pages cover lengths, pages that a step writes have one holder."""
    rng = random.Random(seed)
    m = CacheModel(40, 6, 12, 16)
    for _ in range(300):
        some = rng.sample(range(6), rng.randint(1, 5))
        what = rng.choice(["step", "step", "fork", "cut", "compact"])
        if what == "step":
            q = [rng.choice([0, 1, 5, 20]) for _ in some]
            before = list(m.len)
            if m.step(some, q) is not None:
                for s, n in zip(some, q):
                    for p in range(before[s], before[s] + n):
                        assert m.ref[m.row(s, p)[0]] == 1
        elif what == "fork" and len(some) > 1:
            m.fork([some[0]] * (len(some) - 1), some[1:])
        elif what == "cut":
            m.truncate(some, [m.len[s] // 2 for s in some])
        elif what == "compact":
            m.compact()
        assert m.ref == [sum(r.count(p) for r in m.own) for p in range(40)]
        assert all(len(r) == -(-n // 16) for r, n in zip(m.own, m.len))
