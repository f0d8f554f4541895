"""Host-side argument checks of the serving calls (8-bit linear layer, cross attention, 8-bit cache): refused before anything is enqueued,
so that no GPU is needed.  The context is a block of zeros that no refused call looks into."""
import ctypes

import pytest

import paper_2604_08971_b200 as sentry

INVALID, SHAPE, UNSUPPORTED = -1, -2, -3
P = 4096            # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    sentry.build()
    return sentry.load_library()


@pytest.fixture()
def ctx():
    return ctypes.create_string_buffer(4096)


def _linear(M=4, K=64, N=32, dtype=sentry.SENTRY_BF16):
    return sentry.LinearDesc(M, K, N, dtype)


def test_linear_refusals(lib, ctx):
    f = lambda d, x=P, xs=P, w=P, ws=P, b=None, y=P: lib.sentry_linear_i8(ctx, ctypes.byref(d), x, xs, w, ws, b, y, None)
    assert lib.sentry_linear_i8(None, ctypes.byref(_linear()), P, P, P, P, None, P, None) == INVALID
    assert lib.sentry_linear_i8(ctx, None, P, P, P, P, None, P, None) == INVALID
    assert f(_linear(dtype=sentry.SENTRY_FP8_E4M3)) == INVALID
    assert f(_linear(M=-1)) == SHAPE and f(_linear(N=-1)) == SHAPE and f(_linear(K=0)) == SHAPE
    assert f(_linear(K=40)) == UNSUPPORTED and f(_linear(K=65552)) == UNSUPPORTED
    for bad in ("x", "xs", "w", "ws", "y"):
        assert f(_linear(), **{bad: None}) == INVALID
    assert f(_linear(), x=P + 8) == INVALID and f(_linear(), w=P + 4) == INVALID and f(_linear(), b=P + 2) == INVALID
    assert f(_linear(M=0)) == 0 and f(_linear(N=0)) == 0          # nothing to do


def test_quantize_refusals(lib, ctx):
    f = lambda M=4, K=64, t=sentry.SENTRY_BF16, x=P, c=P, s=P: lib.sentry_quantize_rows_i8(ctx, M, K, t, x, c, s, None)
    assert f(t=sentry.SENTRY_I8) == INVALID and f(M=-1) == SHAPE and f(K=0) == SHAPE and f(K=24) == UNSUPPORTED
    assert f(x=None) == INVALID and f(c=P + 8) == INVALID and f(s=P + 1) == INVALID
    assert f(M=0) == 0


def _cross(**kw):
    v = dict(B=2, Tq=3, Tk=5, Hq=4, Hk=2, d=32, k_h=4, dtype=sentry.SENTRY_BF16)
    strides = {k: kw.pop(k) for k in ("q_stride", "k_stride", "v_stride") if k in kw}
    v.update(kw)
    d = sentry.CrossDesc(**v)
    for k, s in strides.items():
        setattr(d, k, (ctypes.c_int64 * 3)(*s))
    return d


def test_cross_refusals(lib, ctx):
    def f(d, q=P, k=P, v=P, kept=P, ids=None, masks=None, lengths=None, o=P):
        return lib.sentry_cross_attend_fwd(ctx, ctypes.byref(d), q, k, v, kept, ids, masks, lengths, o, None)
    assert lib.sentry_cross_attend_fwd(ctx, None, P, P, P, P, None, None, None, P, None) == INVALID
    assert f(_cross(dtype=sentry.SENTRY_I8)) == INVALID
    for kw in (dict(B=-1), dict(Tq=-1), dict(Tk=-1), dict(Hq=0), dict(Hk=0), dict(k_h=0), dict(Hq=5), dict(k_h=5)):
        assert f(_cross(**kw)) == SHAPE, kw
    for kw in (dict(d=48), dict(Hq=512, Hk=2), dict(Tq=1 << 24), dict(Tk=1 << 24), dict(B=1 << 23), dict(B=1, Tq=(1 << 24) - 1, Hq=128, Hk=1, k_h=128)):
        assert f(_cross(**kw)) == UNSUPPORTED, kw
    assert f(_cross(q_stride=(96, 4, 32))) == UNSUPPORTED and f(_cross(k_stride=(-8, 8, 8))) == SHAPE
    assert f(_cross(k_stride=(8, 32, 0))) == UNSUPPORTED and f(_cross(v_stride=(8, 32, 0))) == UNSUPPORTED   # one key for all
    assert f(_cross(q_stride=((1 << 38) + 8, 32, 32))) == UNSUPPORTED
    assert f(_cross(k_h=3), kept=None) == SHAPE                        # every head, but fewer outputs
    assert f(_cross(), ids=P) == INVALID and f(_cross(), masks=P) == INVALID
    for bad in ("q", "k", "v", "o"):
        assert f(_cross(), **{bad: None}) == INVALID and f(_cross(), **{bad: P + 8}) == INVALID
    assert f(_cross(), lengths=P + 2) == INVALID
    assert f(_cross(B=0), q=None, k=None, v=None, o=None) == 0 and f(_cross(Tq=0), q=None, o=None) == 0
    for kw in (dict(d=48), dict(B=0), dict(Tq=0), dict(Tk=0), dict(dtype=sentry.SENTRY_F32)):   # refused, or nothing to hold
        assert lib.sentry_cross_workspace_bytes(ctypes.byref(_cross(**kw))) == 0
    assert lib.sentry_cross_workspace_bytes(ctypes.byref(_cross(Tk=9000))) > 0


def _cache(**kw):
    v = dict(Hk=2, d=32, page=16, n_pages=7, max_pages=3, format=sentry.SENTRY_I8, k=P, v=P, k_scales=P, v_scales=P, page_table=P)
    v.update(kw)
    return sentry.KvCache(**v)


BAD_CACHES = [(dict(format=sentry.SENTRY_BF16), INVALID), (dict(Hk=0), SHAPE), (dict(n_pages=-1), SHAPE), (dict(max_pages=-1), SHAPE),
              (dict(d=8), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(max_pages=1 << 28, page=16), UNSUPPORTED), (dict(n_pages=1 << 27), UNSUPPORTED),
              (dict(k=None), INVALID), (dict(v=P + 8), INVALID), (dict(k_scales=None), INVALID), (dict(page_table=P + 1), INVALID)]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_cache_refusals(lib, ctx, kw, want):
    c = _cache(**kw)
    d = sentry.CacheAttendDesc(2, 1, 4, 4, sentry.SENTRY_BF16, 0)
    assert lib.sentry_cache_attend_fwd(ctx, ctypes.byref(c), ctypes.byref(d), P, None, P, P, None) == want
    e = sentry.AppendDesc(2, 1, sentry.SENTRY_BF16)
    assert lib.sentry_cache_append(ctx, ctypes.byref(c), ctypes.byref(e), P, P, None, None, None, P, P + 64, None) == want


def test_cache_attend_refusals(lib, ctx):
    f = lambda d, q=P, kept=None, n=P, o=P: lib.sentry_cache_attend_fwd(ctx, ctypes.byref(_cache()), ctypes.byref(d), q, kept, n, o, None)
    desc = lambda B=2, Tq=1, Hq=4, k_h=4, dtype=sentry.SENTRY_BF16: sentry.CacheAttendDesc(B, Tq, Hq, k_h, dtype, 0)
    assert lib.sentry_cache_attend_fwd(ctx, ctypes.byref(_cache()), None, P, None, P, P, None) == INVALID
    assert f(desc(dtype=sentry.SENTRY_I8)) == INVALID and f(desc(Hq=3, k_h=3)) == SHAPE and f(desc(k_h=2)) == SHAPE
    assert f(desc(), q=None) == INVALID and f(desc(), n=None) == INVALID and f(desc(), o=P + 8) == INVALID
    assert f(desc(B=0), q=None, n=None, o=None) == 0


def test_append_refusals(lib, ctx):
    def f(d, K=P, V=P, ids=None, masks=None, most=None, lengths=P, now=P + 64):
        return lib.sentry_cache_append(ctx, ctypes.byref(_cache()), ctypes.byref(d), K, V, ids, masks, most, lengths, now, None)
    desc = lambda B=2, T=3, dtype=sentry.SENTRY_BF16: sentry.AppendDesc(B, T, dtype)
    assert f(desc(dtype=sentry.SENTRY_FP8_E4M3)) == INVALID and f(desc(B=-1)) == SHAPE and f(desc(T=-1)) == SHAPE
    assert f(desc(T=1 << 24)) == UNSUPPORTED and f(desc(), ids=P) == INVALID and f(desc(), K=None) == INVALID
    assert f(desc(), lengths=None) == INVALID and f(desc(), now=None) == INVALID
    assert f(desc(), now=P) == INVALID and f(desc(), now=P + 4) == INVALID      # the lengths are read while the new ones are written
    d = desc()
    d.k_stride = (ctypes.c_int64 * 3)(96, 32, 20)
    assert f(d) == UNSUPPORTED
    assert f(desc(B=0), K=None, V=None) == 0
