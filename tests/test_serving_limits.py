"""What the serving calls ask for and count at the ends of their ranges, on the host."""
import ctypes
import os
import subprocess

import pytest

import paper_2604_08971_b200 as sentry


@pytest.fixture(scope="module")
def lib():
    sentry.build()
    return sentry.load_library()


def test_cache_workspace_does_not_follow_the_tables(lib):
    """A cache call's workspace holds parts of its rows: how long the page tables could become does not count."""
    def need(max_pages, **kw):
        v = dict(B=64, Tq=200, Hq=8, k_h=8, dtype=sentry.SENTRY_BF16, causal=1)
        v.update(kw)
        c = sentry.KvCache(Hk=2, d=64, page=64, n_pages=100, max_pages=max_pages, format=sentry.SENTRY_I8)
        return lib.sentry_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(sentry.CacheAttendDesc(**v)))
    assert need(1 << 14) == need(64)                        # 2^20 tokens, 2^12 tokens: no axis is split
    assert need(1 << 14) < 1 << 20
    assert need(1 << 14, B=2) == need(1 << 9, B=2) > 2 * 200 * 8 * 64 * 4      # split as often


SOURCE = r"""
#include "linear_tiles.cuh"
extern "C" long long tiles(int extent, int tile) { return linear_tiles(extent, tile); }
"""


def test_linear_tiles_at_the_largest_extents(tmp_path):
    """M and N of any size: the tiles that cover them, and the last index inside the last one."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08971_b200", "csrc")
    (tmp_path / "host.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + csrc, str(tmp_path / "host.cpp"), "-o", str(tmp_path / "host.so")], check=True)
    f = ctypes.CDLL(str(tmp_path / "host.so")).tiles
    f.restype = ctypes.c_longlong
    for tile in (8, 16, 64, 128, 256):
        for extent in (0, 1, tile - 1, tile, tile + 1, 2 ** 31 - 257, 2 ** 31 - 256, 2 ** 31 - 255, 2 ** 31 - tile, 2 ** 31 - tile + 1, 2 ** 31 - 1):
            n = f(extent, tile)
            assert n == -(-extent // tile) and n * tile <= 2 ** 31
