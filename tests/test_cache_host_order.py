"""What the paged cache's host side orders, on the CPU: its object linked with a CUDA runtime whose streams run only when
the host waits for them (fake_cache.cpp)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2608_00573_gb300 import binding as B
from paper_2608_00573_gb300 import build as BUILD

HERE = os.path.dirname(os.path.abspath(__file__))
SEQS, PAGES = 4, 8


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    BUILD.build()
    d = str(tmp_path_factory.mktemp("fake"))
    out = os.path.join(d, "libcache_fake.so")
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(BUILD.nvcc()))), "include")
    subprocess.check_call(["g++", "-shared", "-fPIC", "-std=c++17", "-Wl,-Bsymbolic", "-I", inc,
                           os.path.join(HERE, "fake_cache.cpp"), os.path.join(BUILD.BUILD, "cache.o"), "-o", out, "-ldl"])
    L = C.CDLL(out)
    vp, i = C.c_void_p, C.c_int
    L.trimmoe_cache_create.argtypes = [vp, vp, C.POINTER(vp)]
    L.trimmoe_cache_step.argtypes = [vp, i, vp, vp, vp]
    L.trimmoe_cache_stats.argtypes = [vp, vp, i]
    L.trimmoe_cache_destroy.argtypes = [vp]
    L.trimmoe_cache_destroy.restype = None
    L.fake_fill.argtypes = [vp, vp, i, i]
    return L


class Cache:
    """A cache over host memory."""

    def __init__(self, lib, before=lambda self: None):
        lib.fake_reset()
        self.lib, self.h = lib, C.c_void_p()
        self.length, self.ref, self.table = (C.c_int * SEQS)(), (C.c_int * PAGES)(), (C.c_int * (SEQS * 4))(*[-1] * 16)
        self.kv = C.create_string_buffer(2 * PAGES * 2 * 16 * 64 * 2 + 64)
        p = C.addressof(self.kv) + 63 & ~63
        before(self)
        cfg = B.trimmoe_cache_config(layers=1, q_heads=4, kv_heads=2, head_dim=64, page_size=16, n_pages=PAGES,
                                     max_seqs=SEQS, max_pages=4, T_max=64)
        st = B.trimmoe_cache_state(k=p, v=p, table=C.addressof(self.table), length=C.addressof(self.length),
                                   ref=C.addressof(self.ref))
        assert lib.trimmoe_cache_create(C.byref(cfg), C.byref(st), C.byref(self.h)) == 0

    def step(self, stream):
        assert self.lib.trimmoe_cache_step(self.h, 1, (C.c_int * 1)(0), (C.c_int * 1)(1), stream) == 0

    def stats(self, reset):
        s = B.trimmoe_cache_stats_t()
        self.lib.trimmoe_cache_stats(self.h, C.byref(s), reset)
        return s.device_error


def test_create_reads_lengths_that_any_stream_wrote(lib):
    """Lengths that another stream is still to write when create is called are those that count."""
    c = Cache(lib, before=lambda c: lib.fake_fill(0x700, C.addressof(c.length), SEQS, 37))
    c.step(0x500)
    assert [lib.fake_base(s) for s in range(SEQS)] == [37] * SEQS
    lib.trimmoe_cache_destroy(c.h)


@pytest.mark.parametrize("stream", [0x500, 0])
def test_an_error_behind_a_reset_stays(lib, stream):
    """stats(reset) returns when the error word is clear: what a kernel flags from then on is reported."""
    c = Cache(lib)
    c.step(stream)
    assert c.stats(0) == 0
    lib.fake_flag_error(8)
    assert c.stats(1) == 8 and c.stats(0) == 0
    lib.fake_flag_error(8)
    assert c.stats(1) == 8
    lib.fake_flag_error(10)
    lib.fake_finish()
    assert c.stats(0) == 10
    lib.trimmoe_cache_destroy(c.h)
