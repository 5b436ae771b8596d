"""Groups with a common prompt, bounds, selection and attention over blocks: what can be checked without a GPU.  The host
side's objects are linked with a CUDA runtime over host memory (fake_cache.cpp) and with launch functions that only keep
their names (fake_cache_blocks.cpp)."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2608_00573_gb300 import binding as B
from paper_2608_00573_gb300 import build as BUILD

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SEQS, PAGES, WIDTH = 4, 8, 4


def test_struct_sizes_match_the_header(tmp_path):
    names = ("trimmoe_select_args", "trimmoe_blocks_args", "trimmoe_append_args", "trimmoe_attend_args")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "trimmoe.h"\nint main(){%s}\n' % "".join(
        'printf("%%zu ", sizeof(%s));' % n for n in names))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "s")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "s")]).split()]
    assert got == [C.sizeof(getattr(B, n)) for n in names]


def test_error_code_matches_the_header():
    with open(os.path.join(ROOT, "include", "trimmoe.h")) as f:
        assert re.search(r"TRIMMOE_DEVERR_CACHE_BLOCKS = 11\b", f.read())


def test_calls_without_a_handle_are_refused():
    BUILD.build()
    lib = B._cache_lib()
    assert lib.trimmoe_cache_share(None, 0, None, None) == -1
    assert lib.trimmoe_cache_set_bounds(None, None, None) == -1
    assert lib.trimmoe_cache_summarize(None, 0, 0, None) == -1
    assert lib.trimmoe_cache_select(None, 0, None, None) == -1
    assert lib.trimmoe_cache_attend_blocks(None, 0, None, None) == -1
    assert all(n in B.EXPORTS and hasattr(lib, n) for n in (
        "trimmoe_cache_share", "trimmoe_cache_set_bounds", "trimmoe_cache_summarize", "trimmoe_cache_select",
        "trimmoe_cache_attend_blocks"))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    BUILD.build()
    out = os.path.join(str(tmp_path_factory.mktemp("fake")), "libcache_fake.so")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(BUILD.nvcc()))), "include")
    subprocess.check_call(["g++", "-shared", "-fPIC", "-std=c++17", "-Wl,-Bsymbolic", "-I", inc,
                           os.path.join(HERE, "fake_cache.cpp"), os.path.join(HERE, "fake_cache_blocks.cpp"),
                           os.path.join(BUILD.BUILD, "cache.o"), os.path.join(BUILD.BUILD, "cache_blocks.o"),
                           "-o", out, "-ldl"])
    L = C.CDLL(out)
    vp, i = C.c_void_p, C.c_int
    L.trimmoe_cache_create.argtypes = [vp, vp, C.POINTER(vp)]
    for name, args in (("step", [vp, i, vp, vp, vp]), ("attend", [vp, i, vp, vp]), ("stats", [vp, vp, i]),
                       ("share", [vp, i, vp, vp]), ("set_bounds", [vp, vp, vp]), ("summarize", [vp, i, i, vp]),
                       ("select", [vp, i, vp, vp]), ("attend_blocks", [vp, i, vp, vp]), ("truncate", [vp, i, vp, vp, vp])):
        getattr(L, "trimmoe_cache_" + name).argtypes = args
    L.trimmoe_cache_last_error.argtypes = [vp]
    L.trimmoe_cache_last_error.restype = L.fake_launched.restype = C.c_char_p
    L.trimmoe_cache_destroy.argtypes = [vp]
    L.trimmoe_cache_destroy.restype = None
    return L


class Cache:
    """A cache of 4 query heads on 2 over host memory."""

    def __init__(self, lib, q_heads=4, T_max=64):
        lib.fake_reset()
        lib.fake_forget()
        lib.fake_capture(0)
        self.lib, self.h = lib, C.c_void_p()
        self.length, self.ref, self.table = (C.c_int * SEQS)(), (C.c_int * PAGES)(), (C.c_int * (SEQS * WIDTH))(*[-1] * 16)
        self.kv = C.create_string_buffer(2 * PAGES * 2 * 16 * 64 * 2 + 64)
        self.p = C.addressof(self.kv) + 63 & ~63
        cfg = B.trimmoe_cache_config(layers=1, q_heads=q_heads, kv_heads=2, head_dim=64, page_size=16, n_pages=PAGES,
                                     max_seqs=SEQS, max_pages=WIDTH, T_max=T_max)
        st = B.trimmoe_cache_state(k=self.p, v=self.p, table=C.addressof(self.table), length=C.addressof(self.length),
                                   ref=C.addressof(self.ref))
        assert lib.trimmoe_cache_create(C.byref(cfg), C.byref(st), C.byref(self.h)) == 0

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.lib.trimmoe_cache_destroy(self.h)

    def call(self, name, *args):
        """Status and reason of a call."""
        rc = getattr(self.lib, "trimmoe_cache_" + name)(self.h, *args)
        return rc, self.lib.trimmoe_cache_last_error(self.h).decode()

    def step(self, *q):
        n = len(q)
        assert self.call("step", n, (C.c_int * max(1, n))(*range(n)), (C.c_int * max(1, n))(*q), None)[0] == 0

    def share(self, *counts):
        return self.call("share", len(counts), (C.c_int * max(1, len(counts)))(*counts), None)

    def launched(self):
        s = self.lib.fake_launched().decode().split()
        self.lib.fake_forget()
        return s

    def attend(self):
        a = B.trimmoe_attend_args(q=self.p, ld_q=512, out=self.p, ld_out=512)
        assert self.call("attend", 0, C.byref(a), None)[0] == 0
        return self.launched()

    def launches(self):
        s = B.trimmoe_cache_stats_t()
        self.lib.trimmoe_cache_stats(self.h, C.byref(s), 0)
        return s.launches


def refused(got, word):
    assert got[0] == -1 and word in got[1], got


def test_share_refuses(lib):
    with Cache(lib) as c:
        refused(c.share(1), "no step")
        c.step(1, 2, 0)
        refused(c.share(2), "add up")
        refused(c.share(4), "add up")
        refused(c.share(2, 1, 0), "counts")
        refused(c.share(4, -1), "counts")
        refused(c.share(1, 1, 1, 1), "n out of range")
        refused(c.call("share", -1, None, None), "n out of range")
        refused(c.call("share", 1, None, None), "NULL")
        refused(c.share(), "add up")
        lib.fake_capture(1)
        refused(c.share(3), "captured")
        lib.fake_capture(0)
        assert c.launched() == [] and c.share(2, 1)[0] == 0 and c.launched() == ["share"]
        lib.fake_capture(1)                           # the workspaces are there
        assert c.share(3)[0] == 0 and c.launched() == ["share"]
        assert c.call("truncate", 1, (C.c_int * 1)(0), (C.c_int * 1)(0), None)[0] == 0
        refused(c.share(3), "no step")


def test_what_attend_launches(lib):
    """Without groups, with groups of more than single tokens, of single tokens, and until when."""
    with Cache(lib) as c:
        c.step(1, 2, 1)
        assert c.attend() == []
        c.share(3)
        c.launched()
        assert c.attend() == ["join"] and c.attend() == ["join"]
        c.step(1, 1, 0, 1)
        assert c.attend() == []                       # a step ends its groups
        c.share(3, 1)
        assert c.launched() == ["share_single"]
        assert c.attend() == ["own", "join"]
        before = c.launches()
        c.attend()
        assert c.launches() - before == 2             # all groups are small: no attention kernel
        c.step(0, 0)
        assert c.share(1, 1)[0] == 0 and c.launched() == []
        c.step()
        assert c.share()[0] == 0 and c.launched() == []
    with Cache(lib, q_heads=32) as c:                 # 16 query heads of a key/value head: a group of three is not small
        c.step(1, 1, 1)
        c.share(3)
        assert c.launched() == ["share_single"]
        before = c.launches()
        a = B.trimmoe_attend_args(q=c.p, ld_q=2048, out=c.p, ld_out=2048)
        assert c.call("attend", 0, C.byref(a), None)[0] == 0
        assert c.launched() == ["own", "join"] and c.launches() - before == 3
    with Cache(lib, q_heads=34) as c:                 # 17 of them
        c.step(1, 1, 1)
        c.share(3)
        assert c.launched() == ["share"]


def test_groups_that_fill_as_many_tiles_as_their_sequences(lib):
    """64 tokens to a tile: groups are taken up when they halve the tiles."""
    with Cache(lib, T_max=400) as c:
        for q, counts, want in (((60, 60, 60), [3], []), ((20, 20, 20), [3], ["share"]), ((32, 32, 1), [3], []),
                                ((31, 32, 1), [3], ["share"]), ((2, 2, 2), [1, 1, 1], []), ((2, 2, 0), [2, 1], ["share"]),
                                ((2, 2, 200), [2, 1], ["share"]), ((2, 0, 250), [2, 1], [])):
            c.step(*q)
            c.launched()
            assert c.share(*counts)[0] == 0 and c.launched() == want, q
            assert c.attend() == ["join"] * len(want)
        c.step(20, 20, 20)
        c.share(3)
        c.share(1, 1, 1)                              # the last one counts
        c.launched()
        assert c.attend() == []


def test_bounds_and_selection_refuse(lib):
    with Cache(lib) as c:
        p = c.p
        sel = lambda **kw: c.call("select", 0, C.byref(B.trimmoe_select_args(  # noqa: E731
            **{**dict(q=p, ld_q=256, n=3, first=1, last=1, blocks=p), **kw})), None)
        refused(c.call("summarize", 0, 0, None), "no step")
        refused(sel(), "no step")
        c.step(3, 1)
        refused(c.call("summarize", 0, 0, None), "no bounds")
        refused(sel(), "no bounds")
        refused(c.call("set_bounds", p, None), "together")
        refused(c.call("set_bounds", None, p), "together")
        refused(c.call("set_bounds", p + 8, p), "aligned")
        refused(c.call("set_bounds", p, p + 2), "aligned")
        assert c.call("set_bounds", p, p)[0] == 0
        for bad in (1, -1):
            refused(c.call("summarize", bad, 0, None), "layer")
            refused(c.call("select", bad, None, None), "layer")
        refused(c.call("select", 0, None, None), "NULL")
        for kw, word in ((dict(n=0), "n must"), (dict(n=-5), "n must"), (dict(first=-1), "n must"), (dict(last=-1), "n must"),
                         (dict(first=2, last=2), "n must"), (dict(first=2147483647, last=2147483647), "n must"),
                         (dict(q=None), "NULL"), (dict(blocks=None), "NULL"), (dict(q=p + 8), "aligned"),
                         (dict(blocks=p + 2), "aligned"), (dict(ld_q=260), "aligned"), (dict(ld_q=248), "shorter"),
                         (dict(ld_q=-256), "shorter")):
            refused(sel(**kw), word)
        assert c.launched() == []
        assert sel()[0] == 0 and c.call("summarize", 0, 0, None)[0] == 0 and c.call("summarize", 0, 7, None)[0] == 0
        assert c.launched() == ["select", "bounds", "bounds_whole"]
        assert c.call("set_bounds", None, None)[0] == 0
        refused(sel(), "no bounds")
        c.call("set_bounds", p, p)
        c.step()
        assert sel()[0] == 0 and c.call("summarize", 0, 0, None)[0] == 0 and c.launched() == []


def test_attend_blocks_refuses(lib):
    with Cache(lib) as c:
        p = c.p
        att = lambda **kw: c.call("attend_blocks", 0, C.byref(B.trimmoe_blocks_args(  # noqa: E731
            **{**dict(q=p, ld_q=256, blocks=p, n=3, out=p, ld_out=256), **kw})), None)
        refused(att(), "no step")
        c.step(3, 1)
        refused(c.call("attend_blocks", 1, None, None), "layer")
        refused(c.call("attend_blocks", 0, None, None), "NULL")
        for kw, word in ((dict(n=-1), "n must"), (dict(q=None), "NULL"), (dict(out=None), "NULL"), (dict(blocks=None), "NULL"),
                         (dict(q=p + 2), "aligned"), (dict(out=p + 8), "aligned"), (dict(blocks=p + 1), "aligned"),
                         (dict(tree=p + 4), "aligned"), (dict(ld_out=252), "aligned"), (dict(ld_out=128), "shorter"),
                         (dict(ld_q=8), "shorter"), (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"),
                         (dict(scale=float("inf")), "scale")):
            refused(att(**kw), word)
        assert c.launched() == []
        assert att()[0] == 0 and att(n=0, blocks=None)[0] == 0 and att(tree=p)[0] == 0
        assert c.launched() == ["blocks"] * 3
    with Cache(lib, T_max=100) as c:
        c.step(65)
        a = B.trimmoe_blocks_args(q=c.p, ld_q=256, blocks=c.p, n=1, out=c.p, ld_out=256, tree=c.p)
        refused(c.call("attend_blocks", 0, C.byref(a), None), "64")
