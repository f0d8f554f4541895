"""What the serving calls ask for and count at the ends of their ranges, on the host."""
import ctypes

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
