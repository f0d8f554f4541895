"""The serving calls (8-bit linear layer, cross attention, 8-bit cache) against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2604_08971_b200 as sentry
from tests import serving_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def sn():
    s = sentry.Sentry(0)
    yield s
    s.close()


def _np(t):
    return t.detach().cpu().double().numpy()


def _guarded(shape, dtype, fill):
    """A tensor with a margin behind it that nobody may write."""
    n = int(np.prod(shape))
    whole = torch.full((n + 256,), fill, dtype=dtype, device="cuda")
    return whole[:n].view(shape), whole[n:]


# ------------------------------------------------------------------------------------------ 8-bit linear layer

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 48), (5, 1024), (1300, 768), (1200, 4096), (2, 17408)])
def test_quantize_rows(sn, dtype, M, K):
    g = torch.Generator().manual_seed(M * K)
    x = torch.randn((M, K), generator=g)
    if M >= 3:
        x[0] = 0
        x[1] *= 1e-6
        x[2] = (torch.arange(K) % 255 - 127).float() + 0.5 * (torch.arange(K) % 2)   # quotients next to halves
        x[2, 0] = 127
    if M >= 5:
        x[3, K // 2], x[4, K - 1] = float("nan"), float("-inf")
    if M > 100:
        x[5] = 1e-41 * (torch.arange(K) % 5)                # subnormal fp32; zero in the 16-bit types
        x[6] = x[6].sign() * 3e38 if dtype != "f16" else x[6].sign() * 65504
    x = x.to(DT[dtype])
    codes, scales = sn.quantize_rows_i8(x.cuda())
    want_c, want_s = ref.quantize_rows(x)
    np.testing.assert_array_equal(scales.cpu().numpy(), want_s)
    np.testing.assert_array_equal(codes.cpu().numpy(), want_c)


LINEAR = [(1, 16, 1), (4, 1024, 2048), (9, 48, 33), (33, 64, 17), (64, 128, 100), (65, 16, 7), (130, 144, 257), (700, 320, 520), (257, 1040, 768), (70, 65536, 24),
          (3000, 256, 1229)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_linear(sn, dtype, M, K, N):
    g = torch.Generator().manual_seed(M + K + N)
    x = torch.randint(-128, 128, (M, K), generator=g, dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, dtype=torch.int8)
    x[0], w[0] = -128, -128                                       # the largest sum there is
    xs, ws = torch.rand(M, generator=g) * 1e-2, torch.rand(N, generator=g) * 1e-3
    bias = torch.randn(N, generator=g) if N % 2 else None
    if M > 2:
        xs[1] = float("nan")                                      # what a row with a NaN was quantised to
    Y, margin = _guarded((M, N), DT[dtype], 7.0)
    sn.linear_i8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), None if bias is None else bias.cuda(), Y=Y)
    sums = x.double().numpy() @ w.double().numpy().T              # (whole numbers below 2^31: exact)
    y = sums * xs.double().numpy()[:, None] * ws.double().numpy()
    size = np.abs(y)
    if bias is not None:
        y, size = y + bias.double().numpy(), size + np.abs(bias.double().numpy())
    tol = 4 * 2.0 ** -24 * size                                   # the sum as a float, two scales, the bias
    tol = tol + ref.STEP[DT[dtype]] * (np.abs(y) + tol) + ref.TINY[DT[dtype]]
    got = _np(Y)
    if M > 2:
        assert np.isnan(got[1]).all()
        got, y, tol = np.delete(got, 1, 0), np.delete(y, 1, 0), np.delete(tol, 1, 0)
    if dtype == "f16":                                            # beyond fp16's range: infinite
        big = np.abs(y) > 65000
        got, y, tol = got[~big], y[~big], tol[~big]
    ref.check(got, y, tol)
    assert (margin == 7.0).all() and sn.last_status() == 0


def test_linear_layouts_and_refusals(sn):
    x = torch.randn((2, 3, 64), device="cuda").bfloat16()
    codes, scales = sn.quantize_rows_i8(x)
    assert codes.shape == x.shape and scales.shape == (2, 3)
    w, ws = torch.randint(-9, 9, (5, 64), dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda")
    assert sn.linear_i8(codes, scales, w, ws).shape == (2, 3, 5)
    assert sn.linear_i8(codes[:0], scales[:0], w, ws).shape == (0, 3, 5)
    with pytest.raises(ValueError):
        sn.linear_i8(codes, scales, w[:, :32], ws)
    with pytest.raises(ValueError):
        sn.linear_i8(codes, scales[:1], w, ws)
    with pytest.raises(ValueError):
        sn.linear_i8(x, scales, w, ws)
    with pytest.raises(sentry.SentryError):
        sn.quantize_rows_i8(torch.zeros((2, 24), device="cuda"))


# ------------------------------------------------------------------------------------------ attention

def _kept(rng, B, Hq, k_h):
    return np.stack([np.sort(rng.permutation(Hq)[:k_h]) for _ in range(B)]).astype(np.int32)


def _check_attention(O, Q, kept, per, keys_of, dtype, weight_err, q16=False):
    """O [B,k_h,Tq,d] against the reference; keys_of(b, g) -> k, v [N,d], visible [Tq,N]."""
    B, k_h, Tq, d = O.shape
    got, q = _np(O), _np(Q)
    for b in range(B):
        for j in range(k_h):
            h = j if kept is None else int(kept[b, j])
            k, v, visible = keys_of(b, h // per)
            err = 0.0
            if q16:   # bf16 rows as fp16 numbers of [1,2) at most: half of fp16's smallest step, scaled back
                top = np.abs(q[b, h]).max(1, keepdims=True)
                err = np.broadcast_to(2.0 ** -25 * 2.0 ** np.floor(np.log2(np.maximum(top, 1e-300))), q[b, h].shape)
            want, tol = ref.attention(q[b, h], k, v, visible, dtype, weight_err, err)
            ref.check(got[b, j], want, tol, "sample %d head %d" % (b, h))


# B, Tq, Tk, Hq, Hk, d, k_h, keys
CROSS = [(1, 1, 1, 1, 1, 16, 1, "all"), (2, 1, 0, 4, 2, 32, 4, "all"), (3, 1, 33, 4, 4, 64, 3, "lengths"), (2, 5, 31, 6, 2, 64, 4, "modalities"),
         (9, 7, 77, 8, 2, 128, 5, "both"), (2, 1, 1500, 12, 4, 64, 12, "all"), (1, 2, 5000, 8, 1, 128, 8, "lengths"), (4, 17, 129, 4, 1, 16, 4, "modalities"),
         (9, 40, 300, 12, 4, 32, 7, "both"), (2, 130, 257, 4, 2, 64, 4, "lengths"), (3, 300, 640, 6, 2, 128, 5, "both"), (2, 513, 1100, 2, 2, 64, 2, "modalities"),
         (9, 100, 700, 16, 2, 64, 16, "interleaved"), (2, 257, 390, 4, 4, 16, 4, "interleaved"), (2, 600, 200, 8, 8, 32, 3, "lengths"),
         (1, 2000, 4100, 2, 1, 128, 2, "all"), (1, 64, 20000, 4, 1, 64, 4, "lengths")]


def _cross_case(case, dtype, seed=0):
    B, Tq, Tk, Hq, Hk, d, k_h, keys = case
    g, rng = torch.Generator().manual_seed(seed + Tq * Tk), np.random.default_rng(seed + Tk)
    Q, K, V = (torch.randn(s, generator=g).mul_(a).to(DT[dtype]) for s, a in (((B, Hq, Tq, d), 2.0), ((B, Hk, Tk, d), 1.0), ((B, Hk, Tk, d), 1.0)))
    lengths = ids = masks = None
    if keys in ("lengths", "both"):
        lengths = rng.integers(0, Tk + 1, B).astype(np.int32)
        lengths[0], lengths[-1] = Tk, 0 if B > 2 else Tk // 2
    if keys in ("modalities", "both"):
        ids = np.sort(rng.integers(0, 3, Tk)).astype(np.int32)
        masks = np.array([7] + [b % 8 for b in range(1, B)], np.int32)
    if keys == "interleaved":                     # no two neighbours of one modality; one id that is none
        ids = (np.arange(Tk) % 3).astype(np.int32)
        ids[Tk // 2] = 40
        masks = np.array([5] + [b % 8 for b in range(1, B)], np.int32)
    ok = ref.present(B, Tk, lengths, ids, masks)
    kept = _kept(rng, B, Hq, k_h) if k_h < Hq else None
    # what lies at absent keys is nobody's business
    for b in range(B):
        K[b][:, ~ok[b]] = float("nan")
        V[b][:, ~ok[b]] = float("inf")
    return Q, K, V, kept, ids, masks, lengths, ok


def _cuda(*arrays):
    return [None if a is None else (a if torch.is_tensor(a) else torch.from_numpy(a)).cuda() for a in arrays]


WEIGHTS = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 0.0}     # half a step of the type in which weights meet V


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CROSS, ids=lambda c: "x".join(map(str, c)))
def test_cross_attend(sn, case, dtype):
    B, Tq, Tk, Hq, Hk, d, k_h, _ = case
    Q, K, V, kept, ids, masks, lengths, ok = _cross_case(case, dtype)
    O, margin = _guarded((B, k_h, Tq, d), DT[dtype], 5.0)
    gq, gk, gv, gkept, gids, gmasks, glen = _cuda(Q, K, V, kept, ids, masks, lengths)
    sn.cross_attend_fwd(gq, gk, gv, gkept, gids, gmasks, glen, O=O)
    assert sn.last_status() == 0
    k, v = _np(K), _np(V)
    keys_of = lambda b, g: (k[b, g][ok[b]], v[b, g][ok[b]], np.ones((Tq, int(ok[b].sum())), bool))
    _check_attention(O, Q, kept, Hq // Hk, keys_of, DT[dtype], WEIGHTS[dtype])
    assert (margin == 5.0).all()
    again = sn.cross_attend_fwd(gq, gk, gv, gkept, gids, gmasks, glen)
    assert torch.equal(O, again)                 # no order of arrival in it


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [1, 200])
def test_cross_attend_takes_views(sn, dtype, Tq):
    """Q, K and V as they lie in a projection's result, one K for every sample, and a batch out of a larger one."""
    B, Tk, Hq, Hk, d = 3, 150, 4, 2, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    kv = torch.randn((B, Tk, 2, Hk, d), generator=g, device="cuda").to(DT[dtype])
    q = torch.randn((2 * B, Tq, Hq, d), generator=g, device="cuda").to(DT[dtype])
    Q, K, V = q.transpose(1, 2)[::2], kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    one = K[:1].expand(B, -1, -1, -1)
    for k in (K, one):
        assert torch.equal(sn.cross_attend_fwd(Q, k, V), sn.cross_attend_fwd(Q.contiguous(), k.contiguous(), V.contiguous()))
    with pytest.raises(ValueError):
        sn.cross_attend_fwd(Q, K.transpose(2, 3), V.transpose(2, 3))
    with pytest.raises(ValueError):
        sn.cross_attend_fwd(Q, torch.zeros(d, device="cuda", dtype=DT[dtype]).expand(B, Hk, Tk, d), V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [2, 150])
def test_cross_attend_bad_heads(sn, dtype, Tq):
    """An entry that is no head gives zero rows and raises the bit; the same head twice gives the same rows twice."""
    B, Tk, Hq, Hk, d = 2, 90, 4, 2, 32
    g = torch.Generator(device="cuda").manual_seed(4)
    Q, K, V = (torch.randn((B, h, t, d), generator=g, device="cuda").to(DT[dtype]) for h, t in ((Hq, Tq), (Hk, Tk), (Hk, Tk)))
    kept = torch.tensor([[0, 1, 1, 1], [-1, 2, 3, 9]], dtype=torch.int32, device="cuda")
    full = sn.cross_attend_fwd(Q, K, V)
    assert sn.last_status() == 0
    O = sn.cross_attend_fwd(Q, K, V, kept, O=torch.full((B, 4, Tq, d), 3.0, dtype=DT[dtype], device="cuda"))
    assert sn.last_status() == sentry.STATUS_BIT_BAD_INDEX
    assert torch.equal(O[0, 1], O[0, 2]) and torch.equal(O[0, 1], O[0, 3])
    assert (O[1, 0] == 0).all() and (O[1, 3] == 0).all()
    # (rows packed with other neighbours meet the same keys in the same order)
    assert torch.equal(O[0, 0], full[0, 0]) and torch.equal(O[1, 1], full[1, 2])


# ------------------------------------------------------------------------------------------ 8-bit cache

def _pool(rng, n_pages, Hk, page, d, fmt):
    c = rng.integers(-127, 128, (n_pages, Hk, page, d)).astype(np.int8) if fmt == "i8" else \
        (rng.integers(0, 0x7f, (n_pages, Hk, page, d)) | rng.integers(0, 2, (n_pages, Hk, page, d)) * 128).astype(np.uint8)
    s = rng.random((n_pages, Hk)).astype(np.float32) * 0.02 + 0.01 if fmt == "i8" else (2.0 ** rng.integers(-9, -5, (n_pages, Hk))).astype(np.float32)
    return c, s


APPEND = [("i8", "bf16", 3, 1, 2, 16, 32), ("e4m3", "bf16", 5, 7, 2, 32, 64), ("i8", "f16", 4, 40, 1, 16, 16), ("e4m3", "f32", 3, 33, 3, 64, 128),
          ("i8", "f32", 2, 300, 4, 128, 64), ("e4m3", "f16", 9, 130, 2, 128, 128), ("i8", "bf16", 2, 257, 9, 32, 32)]


@pytest.mark.parametrize("fmt,dtype,B,T,Hk,page,d", APPEND)
@pytest.mark.parametrize("keys", ["all", "lengths", "modalities"])
def test_append(sn, fmt, dtype, B, T, Hk, page, d, keys):
    """Three calls behind one another, louder each time: codes, scales and lengths are those of the definition, and nothing else changes."""
    rng = np.random.default_rng(T * d)
    cols = -(-3 * T // page) + 2
    n_pages = B * cols + 2
    pools = [_pool(rng, n_pages, Hk, page, d, fmt) for _ in range(2)]
    table = rng.permutation(n_pages)[:B * cols].reshape(B, cols).astype(np.int32)
    lengths = np.array([(3 * b) % (page + 1) for b in range(B)], np.int32)
    dev = [torch.from_numpy(x).cuda() for p in pools for x in p]
    dt, dlen = torch.from_numpy(table).cuda(), torch.from_numpy(lengths).cuda()
    for call in range(3):
        g = torch.Generator().manual_seed(call)
        K, V = (torch.randn((B, Hk, T, d), generator=g).mul_(3.0 ** call).to(DT[dtype]) for _ in range(2))
        K[0] = 0
        ids = masks = most = None
        if keys == "lengths":
            most = np.array([(5 * b + call) % (T + 2) for b in range(B)], np.int32)
        if keys == "modalities":
            ids, masks = np.sort(rng.integers(0, 3, T)).astype(np.int32), np.array([b % 8 for b in range(B)], np.int32)
        ok = ref.present(B, T, most, ids, masks)
        dlen = sn.cache_append(K.cuda(), V.cuda(), dev[0], dev[2], dev[1], dev[3], dt, dlen, *_cuda(ids, masks, most))
        for X, (c, s) in zip((K, V), pools):
            now = ref.append(X.double().numpy(), c, s, table, lengths, ok, fmt)
        lengths = now
        np.testing.assert_array_equal(dlen.cpu().numpy(), lengths)
        for i, (c, s) in enumerate(pools):
            np.testing.assert_array_equal(dev[2 * i + 1].cpu().numpy(), s)
            np.testing.assert_array_equal(dev[2 * i].cpu().numpy(), c)
    assert sn.last_status() == 0


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
def test_append_edges(sn, fmt):
    """Values that are no numbers, pages and lengths that are none, a full cache, a scale that is no power of two, views."""
    rng = np.random.default_rng(5)
    B, T, Hk, page, d, cols = 7, 20, 2, 16, 16, 3
    n_pages = B * cols
    pools = [_pool(rng, n_pages, Hk, page, d, fmt) for _ in range(2)]
    table = rng.permutation(n_pages).reshape(B, cols).astype(np.int32)
    lengths = np.array([3, 40, -1, 49, 0, 5, 16], np.int32)
    table[4, 0], table[5, 1] = n_pages, -1
    table[1, :2] = 999                                    # behind it: not needed
    for c, s in pools:
        s[table[0, 0], 0] = np.float32(0.0371)            # somebody else's scale
        s[table[6, 0], 0] = np.nan                        # full page: not touched
    g = torch.Generator().manual_seed(1)
    both = torch.randn((B, T, 2, Hk, d), generator=g)
    both[0, 15, 0, 1, 3], both[5, 2, 1, 0, 0] = float("nan"), float("inf")
    both[6] *= 1e-3
    both = both.bfloat16()
    K, V = both[:, :, 0].transpose(1, 2), both[:, :, 1].transpose(1, 2)
    dev = [torch.from_numpy(x).cuda() for p in pools for x in p]
    gb = both.cuda()
    now = sn.cache_append(gb[:, :, 0].transpose(1, 2), gb[:, :, 1].transpose(1, 2), dev[0], dev[2], dev[1], dev[3], *_cuda(table, lengths))
    assert sn.last_status() == sentry.STATUS_BIT_BAD_INDEX
    for X, (c, s) in zip((K, V), pools):
        want = ref.append(X.double().numpy(), c, s, table, lengths, np.ones((B, T), bool), fmt)
    np.testing.assert_array_equal(now.cpu().numpy(), want)
    for i, (c, s) in enumerate(pools):
        np.testing.assert_array_equal(dev[2 * i + 1].cpu().numpy(), s)
        np.testing.assert_array_equal(dev[2 * i].cpu().numpy(), c)
    # nothing to store
    none = sn.cache_append(gb[:, :0, 0].transpose(1, 2), gb[:, :0, 1].transpose(1, 2), dev[0], dev[2], dev[1], dev[3], *_cuda(table, np.full(B, 5, np.int32)))
    assert (none == 5).all() and sn.last_status() == 0
    np.testing.assert_array_equal(dev[0].cpu().numpy(), pools[0][0])


# fmt, dtype, B, Tq, cols, page, Hq, Hk, d, k_h, causal
CACHE = [("i8", "bf16", 3, 1, 2, 16, 2, 2, 16, 2, 0), ("e4m3", "bf16", 5, 1, 3, 32, 4, 2, 32, 3, 0), ("i8", "f16", 4, 3, 5, 16, 8, 2, 64, 5, 1),
         ("e4m3", "f16", 4, 4, 4, 64, 16, 4, 128, 16, 1), ("i8", "bf16", 2, 1, 40, 128, 8, 1, 128, 8, 0), ("e4m3", "bf16", 1, 17, 20, 16, 4, 1, 64, 4, 1),
         ("i8", "f16", 2, 60, 4, 32, 6, 2, 32, 4, 0), ("e4m3", "bf16", 2, 150, 5, 64, 4, 4, 16, 4, 1), ("i8", "bf16", 33, 1, 9, 64, 4, 4, 64, 4, 0),
         ("e4m3", "f32", 3, 5, 3, 16, 4, 2, 32, 3, 1), ("i8", "f32", 2, 1, 4, 128, 4, 2, 128, 4, 0), ("i8", "bf16", 2, 300, 8, 128, 8, 2, 64, 8, 1)]


@pytest.mark.parametrize("case", CACHE, ids=lambda c: "-".join(map(str, c)))
def test_cache_attend(sn, case):
    fmt, dtype, B, Tq, cols, page, Hq, Hk, d, k_h, causal = case
    rng = np.random.default_rng(Tq * cols)
    n_pages, cap = B * cols + 2, cols * page
    (kc, ks), (vc, vs) = (_pool(rng, n_pages, Hk, page, d, fmt) for _ in range(2))
    kc = (kc // 8).astype(np.int8) if fmt == "i8" else np.where(kc & 127 > 0x58, kc & 0xd8, kc).astype(np.uint8)   # scores of ordinary size
    vs *= (10.0 ** rng.integers(-3, 4, vs.shape)).astype(np.float32)                                               # pages of very different sizes
    table = rng.permutation(n_pages)[:B * cols].reshape(B, cols).astype(np.int32)
    lengths = rng.integers(0, cap + 1, B).astype(np.int32)
    lengths[0] = cap - 3
    if B > 1:
        lengths[1] = 1
    if B > 2:
        lengths[2] = 0
    k, v = ref.values(kc, fmt) * ks[..., None, None].astype(np.float64), ref.values(vc, fmt) * vs[..., None, None].astype(np.float64)
    used = np.zeros(n_pages, int)
    for b in range(B):
        for j in range(cols):
            used[table[b, j]] = np.clip(lengths[b] - j * page, 0, page)
    for p in range(n_pages):          # behind the last token: codes and scales that are no numbers
        if fmt == "e4m3":
            kc[p, :, used[p]:], vc[p, :, used[p]:] = 0x7f, 0xff
        if used[p] == 0:
            ks[p], vs[p] = np.nan, np.inf
    kept = _kept(rng, B, Hq, k_h) if k_h < Hq else None
    Q = torch.randn((B, Hq, Tq, d), generator=torch.Generator().manual_seed(7)).to(DT[dtype])
    Q[0, 0, 0] *= 1e-5
    O, margin = _guarded((B, k_h, Tq, d), DT[dtype], 5.0)
    args = _cuda(kc, vc, ks, vs, table, lengths)
    sn.cache_attend_fwd(Q.cuda(), *args, *_cuda(kept), bool(causal), O=O)
    assert sn.last_status() == 0

    def keys_of(b, g):
        n = int(lengths[b])
        kk, vv = (x[table[b]][:, g].reshape(cap, d)[:n] for x in (k, v))
        ok = np.ones((Tq, n), bool)
        if causal:
            ok = np.arange(n)[None] <= np.arange(Tq)[:, None] + n - Tq
        return kk, vv, ok
    weight_err = 2.0 ** -11 if dtype != "f32" else 0.0
    _check_attention(O, Q, kept, Hq // Hk, keys_of, DT[dtype], weight_err, q16=dtype == "bf16")
    assert (margin == 5.0).all()
    assert torch.equal(O, sn.cache_attend_fwd(Q.cuda(), *args, *_cuda(kept), bool(causal)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Tq", [1, 90])
def test_cache_attend_edges(sn, dtype, Tq):
    """Pages shared by samples; entries that are no pages and lengths that are none; a page with a NaN scale is seen by those who see it."""
    rng = np.random.default_rng(9)
    B, page, Hq, Hk, d, cols = 4, 16, 4, 2, 32, 6
    (kc, ks), (vc, vs) = (_pool(rng, 10, Hk, page, d, "i8") for _ in range(2))
    table = np.stack([np.arange(cols)] * B).astype(np.int32)
    table[1, 2] = 10
    table[2, 0] = -5
    lengths = np.array([90, 96, 200, -3], np.int32)
    Q = torch.randn((B, Hq, Tq, d), generator=torch.Generator().manual_seed(2)).to(DT[dtype])
    dev = _cuda(kc, vc, ks, vs)
    O = sn.cache_attend_fwd(Q.cuda(), *dev, *_cuda(table, lengths))
    assert sn.last_status() == sentry.STATUS_BIT_BAD_INDEX
    k, v = (c.astype(np.float64) * s[..., None, None] for c, s in ((kc, ks), (vc, vs)))

    def keys_of(b, g):
        n = int(np.clip(lengths[b], 0, 96))
        ok = np.array([0 <= table[b, i // page] < 10 for i in range(n)], bool)
        kk, vv = (x[np.clip(table[b], 0, 9)][:, g].reshape(-1, d)[:n][ok] for x in (k, v))
        return kk, vv, np.ones((Tq, int(ok.sum())), bool)
    _check_attention(O, Q, None, 2, keys_of, DT[dtype], 2.0 ** -11 if dtype != "f32" else 0.0, q16=dtype == "bf16")
    vs2, ks2 = vs.copy(), ks.copy()
    vs2[5, 0] = ks2[5, 0] = np.nan
    t0 = np.stack([np.arange(cols)] * B).astype(np.int32)
    P = sn.cache_attend_fwd(Q.cuda(), dev[0], dev[1], *_cuda(ks2, vs2, t0, np.array([96, 80, 81, 0], np.int32)), causal=True)
    assert sn.last_status() == 0
    nan = torch.isnan(P).all(-1).cpu().numpy()
    want = np.zeros((B, Hq, Tq), bool)
    for b, n in enumerate((96, 80, 81, 0)):
        want[b, :2] = (np.arange(Tq) + n - Tq >= 80)[None]
    np.testing.assert_array_equal(nan, want)
    assert not torch.isnan(P.cpu()[torch.from_numpy(~want)]).any()


def test_cache_beyond_32_bits(sn):
    """A pool of more than 2^32 bytes, pages at its end."""
    Hk, page, d, n_pages = 4, 128, 128, 66000
    k = torch.zeros((n_pages, Hk, page, d), dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = torch.zeros((n_pages, Hk), device="cuda"), torch.zeros((n_pages, Hk), device="cuda")
    table = torch.tensor([[65999, 0], [65537, 32769]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn((2, Hk, 200, d), generator=g, device="cuda").bfloat16()
    n = sn.cache_append(X, X, k, v, ks, vs, table, torch.zeros(2, dtype=torch.int32, device="cuda"))
    small = torch.arange(4, dtype=torch.int32, device="cuda").reshape(2, 2)
    pick = table.long().reshape(-1)
    Q = torch.randn((2, 8, 3, d), generator=g, device="cuda").bfloat16()
    a = sn.cache_attend_fwd(Q, k, v, ks, vs, table, n)
    b = sn.cache_attend_fwd(Q, k[pick].contiguous(), v[pick].contiguous(), ks[pick].contiguous(), vs[pick].contiguous(), small, n)
    assert torch.equal(a, b) and sn.last_status() == 0 and (a != 0).any() and (ks[table.long()] > 0).all()


# ------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("Tq", [1, 70])
def test_encoder_to_decoder(sn, fmt, Tq):
    """Encoder states -> 8-bit K, V projection -> cache -> a decoder's rows on it, and the 16-bit states beside it; every step against
    its definition on what the step before left."""
    B, Tk, D, Hq, Hk, d, page = 3, 210, 128, 4, 2, 32, 32
    g = torch.Generator().manual_seed(11)
    X, Z = torch.randn((B, Tk, D), generator=g).bfloat16(), torch.randn((B, Tq, D), generator=g).bfloat16()
    wkv, wq = torch.randn((2 * Hk * d, D), generator=g) * 0.1, torch.randn((Hq * d, D), generator=g) * 0.1
    (wkv8, skv), (wq8, sq) = (sn.quantize_rows_i8(w.cuda()) for w in (wkv, wq))
    ids, masks = np.repeat(np.arange(3), 70).astype(np.int32), np.array([7, 5, 2], np.int32)
    gids, gmasks = _cuda(ids, masks)
    KV = sn.linear_i8(*sn.quantize_rows_i8(X.cuda()), wkv8, skv).view(B, Tk, 2, Hk, d)
    Q = sn.linear_i8(*sn.quantize_rows_i8(Z.cuda()), wq8, sq).view(B, Tq, Hq, d).transpose(1, 2)
    for got, x, w in ((KV.reshape(B * Tk, -1), X, wkv), (Q.transpose(1, 2).reshape(B * Tq, -1), Z, wq)):
        (xc, xs), (wc, ws) = ref.quantize_rows(x.reshape(-1, D)), ref.quantize_rows(w)
        y = xc.astype(np.float64) @ wc.astype(np.float64).T * xs.astype(np.float64)[:, None] * ws.astype(np.float64)
        ref.check(_np(got), y, np.abs(y) * (2.0 ** -8 + 2.0 ** -21))
    K, V = KV[:, :, 0].transpose(1, 2), KV[:, :, 1].transpose(1, 2)
    cols = -(-Tk // page)
    code = torch.int8 if fmt == "i8" else torch.float8_e4m3fn
    kc, vc = (torch.zeros((B * cols, Hk, page, d), dtype=torch.uint8, device="cuda").view(code) for _ in range(2))
    ks, vs = torch.zeros((B * cols, Hk), device="cuda"), torch.zeros((B * cols, Hk), device="cuda")
    table = torch.arange(B * cols, dtype=torch.int32, device="cuda").reshape(B, cols)
    n = sn.cache_append(K, V, kc, vc, ks, vs, table, torch.zeros(B, dtype=torch.int32, device="cuda"), gids, gmasks)
    O8, O16 = sn.cache_attend_fwd(Q, kc, vc, ks, vs, table, n), sn.cross_attend_fwd(Q, K, V, key_modality_ids=gids, masks=gmasks)
    assert sn.last_status() == 0
    ok = ref.present(B, Tk, None, ids, masks)
    np.testing.assert_array_equal(n.cpu().numpy(), ok.sum(1))
    k16, v16 = _np(K), _np(V)
    pools = []
    for x in (k16, v16):
        c, s = np.zeros((B * cols, Hk, page, d), np.int8 if fmt == "i8" else np.uint8), np.zeros((B * cols, Hk), np.float32)
        ref.append(x, c, s, table.cpu().numpy(), np.zeros(B, np.int32), ok, fmt)
        pools.append(ref.values(c, fmt) * s[..., None, None])
    everyone = lambda m: np.ones((Tq, m), bool)
    _check_attention(O16, Q, None, 2, lambda b, g: (k16[b, g][ok[b]], v16[b, g][ok[b]], everyone(int(ok[b].sum()))), torch.bfloat16, 2.0 ** -8)
    t = table.cpu().numpy()

    def keys_of(b, g):
        m = int(ok[b].sum())
        return tuple(p[t[b]][:, g].reshape(-1, d)[:m] for p in pools) + (everyone(m),)
    _check_attention(O8, Q, None, 2, keys_of, torch.bfloat16, 2.0 ** -11, q16=True)


def test_decoding_steps_captured(sn):
    """A decoding step (projection, append, attention) captured once on a stream of its own and replayed, with an eager call that needs a larger
    workspace between the replays: what a loop of eager steps gives."""
    B, D, Hq, Hk, d, page, cols = 2, 64, 4, 2, 64, 16, 40
    g = torch.Generator(device="cuda").manual_seed(8)
    w, ws = sn.quantize_rows_i8(torch.randn(((Hq + 2 * Hk) * d, D), generator=g, device="cuda") * 0.2)
    steps = [torch.randn((B, 1, D), generator=g, device="cuda").bfloat16() for _ in range(5)]
    big = [torch.randn((8, h, t, 128), generator=g, device="cuda").bfloat16() for h, t in ((32, 8), (4, 6000), (4, 6000))]

    def new():
        kc, vc = (torch.zeros((B * cols, Hk, page, d), dtype=torch.int8, device="cuda") for _ in range(2))
        ks, vs = (torch.full((B * cols, Hk), 0.01, device="cuda") for _ in range(2))
        table = torch.arange(B * cols, dtype=torch.int32, device="cuda").flip(0).reshape(B, cols).contiguous()
        return kc, vc, ks, vs, table, torch.tensor([600, 3], dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")

    def step(s, x, c):
        kc, vc, ks, vs, table, n, m = c
        y = s.linear_i8(*s.quantize_rows_i8(x), w, ws).view(B, 1, Hq + 2 * Hk, d).transpose(1, 2)
        s.cache_append(y[:, Hq:Hq + Hk], y[:, Hq + Hk:], kc, vc, ks, vs, table, n, new_lengths=m)
        n.copy_(m)
        return s.cache_attend_fwd(y[:, :Hq], kc, vc, ks, vs, table, n)
    one = new()
    want = [step(sn, x, one).clone() for x in steps]
    other = sentry.Sentry(0)
    try:
        two, x = new(), steps[0].clone()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step(other, x, new())
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = step(other, x, two)
        torch.cuda.synchronize()
        for i, xs in enumerate(steps):
            x.copy_(xs)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i]), i
            before = other._ws.numel()
            big_out = other.cross_attend_fwd(*big)
            assert i or other._ws.numel() > before
            assert torch.equal(big_out, sn.cross_attend_fwd(*big))
            junk = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(8)]   # what was freed is somebody else's now
            del junk
        for a, b in zip(one[:6], two[:6]):
            assert torch.equal(a, b)
    finally:
        other.close()


def test_small_batches_equal_large_ones(sn):
    """A sample's result does not depend on what else is in the batch, as long as the axis of keys is not split differently."""
    g = torch.Generator(device="cuda").manual_seed(6)
    Q, K, V = (torch.randn((300, h, t, 64), generator=g, device="cuda").half() for h, t in ((4, 1), (2, 100), (2, 100)))
    whole = sn.cross_attend_fwd(Q, K, V)
    assert torch.equal(whole[17:18], sn.cross_attend_fwd(Q[17:18], K[17:18], V[17:18]))


def test_serving_refusals(sn):
    Q, K = torch.zeros((2, 4, 1, 32), device="cuda").half(), torch.zeros((2, 2, 5, 32), device="cuda").half()
    kc, s = torch.zeros((4, 2, 16, 32), dtype=torch.int8, device="cuda"), torch.zeros((4, 2), device="cuda")
    table, n = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    bad = [lambda: sn.cross_attend_fwd(Q, K, K[:, :, :4]), lambda: sn.cross_attend_fwd(Q, K.float(), K.float()), lambda: sn.cross_attend_fwd(Q, K[:1], K[:1]),
           lambda: sn.cross_attend_fwd(Q, K, K, torch.zeros((1, 4), dtype=torch.int32, device="cuda")),
           lambda: sn.cross_attend_fwd(Q, K, K, key_lengths=n.long()), lambda: sn.cross_attend_fwd(Q, K, K, key_modality_ids=n, masks=n),
           lambda: sn.cross_attend_fwd(Q, K, K, O=torch.zeros((2, 4, 2, 32), device="cuda").half()),
           lambda: sn.cross_attend_fwd(Q.cpu(), K, K), lambda: sn.cache_attend_fwd(Q, kc, kc[:3], s, s, table, n),
           lambda: sn.cache_attend_fwd(Q, kc, kc.view(torch.uint8), s, s, table, n), lambda: sn.cache_attend_fwd(Q, kc.half(), kc.half(), s, s, table, n),
           lambda: sn.cache_attend_fwd(Q, kc, kc, s[:2], s, table, n), lambda: sn.cache_attend_fwd(Q, kc, kc, s, s, table[:1], n),
           lambda: sn.cache_attend_fwd(Q, kc, kc, s, s, table, n[:1]), lambda: sn.cache_append(K, K[:, :, :2], kc, kc, s, s, table, n),
           lambda: sn.cache_append(K, K, kc, kc, s, s, table, n, token_lengths=n[:1])]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(sentry.SentryError):
        sn.cache_append(K, K, kc, kc.clone(), s, s.clone(), table, n, new_lengths=n)
    with pytest.raises(sentry.SentryError):
        sn.cross_attend_fwd(Q, K, K, key_modality_ids=torch.zeros(5, dtype=torch.int32, device="cuda"))
    # empty calls
    assert sn.cross_attend_fwd(Q[:0], K[:0], K[:0]).shape == (0, 4, 1, 32)
    assert sn.cross_attend_fwd(Q[:, :, :0], K, K).shape == (2, 4, 0, 32)
    assert (sn.cache_attend_fwd(Q, kc, kc, s, s, table[:, :0], n) == 0).all() and sn.last_status() == 0


# ------------------------------------------------------------------------------------------ where the paths inside could go wrong

# (keys whose list of present ones is too long for a block's own; single rows, and rows packed into many tiles)
LONG = [(2, 70, 5000, 4, 2, 64, 3, "both"), (3, 33, 4097, 2, 1, 128, 2, "interleaved"), (2, 3, 9000, 4, 2, 64, 4, "both"), (40, 1, 700, 8, 2, 32, 5, "both"),
        (2, 32, 1030, 1, 1, 16, 1, "interleaved"), (2, 33, 1030, 1, 1, 16, 1, "interleaved"), (70, 1, 1000, 32, 1, 64, 32, "lengths"), (1, 1, 65, 64, 1, 128, 64, "all")]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", LONG, ids=lambda c: "x".join(map(str, c)))
def test_cross_attend_long_lists(sn, case, dtype):
    test_cross_attend(sn, case, dtype)


def _ramps(Tq, N, d, top):
    """q [Tq,d] and k [N,d] whose scores rise from -top to top along the keys for every other row, and fall for the rest."""
    sign = np.where(np.arange(Tq) % 2, -1.0, 1.0)[:, None]
    return np.ones((Tq, d)) * sign, np.linspace(-top, top, N)[:, None] / math.sqrt(d) * np.ones((N, d))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Tq,N,d", [(1, 900, 64), (8, 2000, 128), (20, 700, 32), (90, 1500, 64), (300, 1100, 128), (64, 130, 16)])
@pytest.mark.parametrize("top", [15.0, 300.0])
def test_rising_scores(sn, dtype, Tq, N, d, top):
    """The running maximum moves with every step of the keys in one row and never again in the next one."""
    q, k = _ramps(Tq, N, d, top)
    g = torch.Generator().manual_seed(N)
    Q = (torch.from_numpy(q) + 0.01 * torch.randn(q.shape, generator=g, dtype=torch.float64)).to(DT[dtype])[None, None]
    K = torch.from_numpy(k).to(DT[dtype])[None, None]
    V = torch.randn((1, 1, N, d), generator=g).to(DT[dtype])
    O = sn.cross_attend_fwd(Q.cuda(), K.cuda(), V.cuda())
    _check_attention(O, Q, None, 1, lambda b, h: (_np(K[0, 0]), _np(V[0, 0]), np.ones((Tq, N), bool)), DT[dtype], WEIGHTS[dtype])


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Tq,N,d,page", [(1, 900, 64, 64), (8, 2000, 128, 16), (40, 333, 32, 128)])
def test_rising_scores_cache(sn, fmt, dtype, Tq, N, d, page):
    q, k = _ramps(Tq, N, d, 40.0)
    rng = np.random.default_rng(N)
    cols = -(-N // page)
    kc, ks = np.zeros((cols, 1, page, d), np.int8 if fmt == "i8" else np.uint8), np.zeros((cols, 1), np.float32)
    vc, vs = _pool(rng, cols, 1, page, d, fmt)
    table = np.arange(cols, dtype=np.int32)[None]
    ref.append(k[None, None], kc, ks, table, np.zeros(1, np.int32), np.ones((1, N), bool), fmt)
    Q = torch.from_numpy(q).to(DT[dtype])[None, None]
    O = sn.cache_attend_fwd(Q.cuda(), *_cuda(kc, vc, ks, vs, table, np.array([N], np.int32)))
    kk, vv = ((ref.values(c, fmt) * s[..., None, None]).reshape(-1, d)[:N] for c, s in ((kc, ks), (vc, vs)))
    _check_attention(O, Q, None, 1, lambda b, h: (kk, vv, np.ones((Tq, N), bool)), DT[dtype], 2.0 ** -11 if dtype != "f32" else 0.0, q16=dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Tq", [1, 6, 130])
def test_what_is_no_number_stays_where_it_is(sn, dtype, Tq):
    """A NaN in a query makes its own rows NaN, one in a present key or value those of its sample and group, and no other bit changes."""
    B, Tk, Hq, Hk, d = 3, 300, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(12)
    Q, K, V = (torch.randn((B, h, t, d), generator=g, device="cuda").to(DT[dtype]) for h, t in ((Hq, Tq), (Hk, Tk), (Hk, Tk)))
    clean = sn.cross_attend_fwd(Q, K, V)
    want = torch.zeros((B, Hq, Tq), dtype=torch.bool, device="cuda")
    Q[0, 1, Tq // 2, 5] = float("nan")
    want[0, 1, Tq // 2] = True
    K[1, 0, 271, 63] = float("nan")
    want[1, :2] = True
    V[2, 1, 3] = float("nan")
    want[2, 2:] = True
    O = sn.cross_attend_fwd(Q, K, V)
    assert torch.equal(torch.isnan(O).all(-1), want) and torch.equal(torch.isnan(O).any(-1), want)
    assert torch.equal(O[~want], clean[~want]) and sn.last_status() == 0


def _cache_call(B, Tq, cols, page, Hq, Hk, d, seed):
    rng = np.random.default_rng(seed)
    (kc, ks), (vc, vs) = (_pool(rng, 97, Hk, page, d, "i8") for _ in range(2))
    table = rng.integers(0, 97, (B, cols)).astype(np.int32)         # pages that several samples, and several places, share
    lengths = rng.integers(0, cols * page + 1, B).astype(np.int32)
    Q = torch.randn((B, Hq, Tq, d), generator=torch.Generator().manual_seed(seed)).bfloat16()
    return [Q.cuda()] + _cuda((kc // 8).astype(np.int8), vc, ks, vs, table, lengths)


# (samples enough that the last block of a group joins its parts, and so few that a launch of its own does)
SHARED = [(32, 1, 30, 32, 4, 2, 64), (3, 1, 300, 16, 8, 1, 128), (130, 1, 40, 64, 4, 1, 32), (9, 5, 64, 128, 16, 4, 128), (1, 2, 500, 32, 4, 4, 16), (5, 1, 7, 16, 4, 2, 32)]


def test_calls_in_turn_on_streams(sn):
    """Calls of different shapes in turn on one context and a stream of its own, then from two contexts on two streams at once: every result is
    the one that the call gives alone, and that of fp32 rows within both results' tolerance."""
    calls = [_cache_call(*s, seed=i) for i, s in enumerate(SHARED)]
    alone = [sn.cache_attend_fwd(*c) for c in calls]
    for c, o in zip(calls, alone):
        Q, kc, vc, ks, vs, table, lengths = [x.cpu() for x in c]
        Hk, page, d = kc.shape[1:]
        per, cap = Q.shape[1] // Hk, table.shape[1] * page

        def keys_of(b, g):
            n = int(lengths[b])
            k, v = ((x.double() * s.double()[..., None, None])[table[b].long()][:, g].reshape(cap, d)[:n].numpy() for x, s in ((kc, ks), (vc, vs)))
            return k, v, np.ones((Q.shape[2], n), bool)
        _check_attention(o, Q, None, per, keys_of, torch.bfloat16, 2.0 ** -11, q16=True)
    torch.cuda.synchronize()
    other = sentry.Sentry(0)
    try:
        one, two = torch.cuda.Stream(), torch.cuda.Stream()
        got = []
        for i in range(40):
            with torch.cuda.stream(one):
                got.append((i % 6, sn.cache_attend_fwd(*calls[i % 6])))
            with torch.cuda.stream(two):
                got.append((5 - i % 6, other.cache_attend_fwd(*calls[5 - i % 6])))
        torch.cuda.synchronize()
        for i, o in got:
            assert torch.equal(o, alone[i]), i
        assert sn.last_status() == 0 and other.last_status() == 0
    finally:
        other.close()


def test_many_rows_on_two_streams(sn):
    """Kernels that hold tensor memory (projection, many rows of cross attention) from two contexts on two streams at once."""
    g = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn((1500, 256), generator=g, device="cuda").bfloat16()
    w, ws = sn.quantize_rows_i8(torch.randn((768, 256), generator=g, device="cuda"))
    Q, K, V = (torch.randn((4, h, t, 64), generator=g, device="cuda").bfloat16() for h, t in ((8, 300), (2, 900), (2, 900)))
    run = lambda s: (s.linear_i8(*s.quantize_rows_i8(X), w, ws), s.cross_attend_fwd(Q, K, V))
    want = run(sn)
    torch.cuda.synchronize()
    other = sentry.Sentry(0)
    try:
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        got = []
        for _ in range(10):
            for s, st in zip((sn, other), streams):
                with torch.cuda.stream(st):
                    got.append(run(s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o in got for a, b in zip(o, want))
    finally:
        other.close()


def test_sizes_of_one(sn):
    """Views whose dimensions of size one have strides of their own, and one token of a long tensor."""
    g = torch.Generator(device="cuda").manual_seed(1)
    Q, K, V = (torch.randn((5, h, t, 32), generator=g, device="cuda").bfloat16() for h, t in ((2, 9), (1, 40), (1, 40)))
    for i in (0, 8):
        for n in (1, 40):
            q, k, v = Q[3:4, :, i:i + 1], K[3:4, :, :n], V[3:4, :, 40 - n:]
            assert torch.equal(sn.cross_attend_fwd(q, k, v), sn.cross_attend_fwd(q.contiguous(), k.contiguous(), v.contiguous()))
    odd = torch.randn(8 * 32 + 7, generator=g, device="cuda").bfloat16()
    q = torch.as_strided(odd, (1, 8, 1, 32), (3, 32, 5, 1))          # (no index ever multiplies the 3 and the 5)
    assert torch.equal(sn.cross_attend_fwd(q, K[:1], V[:1]), sn.cross_attend_fwd(q.clone(memory_format=torch.contiguous_format), K[:1], V[:1]))


# (prompts of many rows on a cache: fmt, dtype, B, Tq, cols, page, Hq, Hk, d, k_h, causal)
PROMPTS = [("i8", "bf16", 3, 40, 6, 16, 8, 2, 128, 8, 1), ("e4m3", "f16", 2, 200, 4, 128, 4, 2, 128, 3, 0), ("e4m3", "bf16", 5, 70, 9, 64, 2, 1, 128, 2, 1),
           ("i8", "f16", 1, 1000, 10, 128, 2, 2, 64, 2, 1), ("e4m3", "f16", 2, 129, 70, 16, 2, 2, 32, 2, 0), ("i8", "bf16", 9, 65, 3, 32, 4, 4, 16, 4, 1),
           ("i8", "f16", 1, 65, 90, 64, 1, 1, 128, 1, 0), ("e4m3", "bf16", 2, 700, 30, 16, 4, 4, 64, 2, 1)]


@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: "-".join(map(str, c)))
def test_cache_attend_prompts(sn, case):
    test_cache_attend(sn, case)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("Tq,N,d,page", [(200, 900, 64, 64), (300, 2000, 128, 16), (140, 333, 32, 128)])
def test_rising_scores_cache_prompts(sn, fmt, dtype, Tq, N, d, page):
    test_rising_scores_cache(sn, fmt, dtype, Tq, N, d, page)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Tq", [1, 9, 150])
def test_scales_of_any_sign(sn, fmt, dtype, Tq):
    """Pages whose scales are somebody else's: negative, zero, a thousand times the others'."""
    rng = np.random.default_rng(21)
    B, Hq, Hk, d, page, cols = 2, 2, 1, 64, 16, 12
    (kc, ks), (vc, vs) = (_pool(rng, B * cols, Hk, page, d, fmt) for _ in range(2))
    kc = (kc // 8).astype(np.int8) if fmt == "i8" else np.where(kc & 127 > 0x58, kc & 0xd8, kc).astype(np.uint8)
    ks[3::5] *= -1
    ks[4::7] = 0
    vs[1::3] *= -1
    vs[2::5] = 0
    vs[6::7] *= 1000
    table = np.arange(B * cols, dtype=np.int32).reshape(B, cols)
    lengths = np.array([cols * page, 101], np.int32)
    Q = torch.randn((B, Hq, Tq, d), generator=torch.Generator().manual_seed(3)).to(DT[dtype])
    O = sn.cache_attend_fwd(Q.cuda(), *_cuda(kc, vc, ks, vs, table, lengths), causal=True)
    k, v = (ref.values(c, fmt) * s[..., None, None].astype(np.float64) for c, s in ((kc, ks), (vc, vs)))

    def keys_of(b, g):
        n = int(lengths[b])
        kk, vv = (x[table[b]][:, g].reshape(-1, d)[:n] for x in (k, v))
        return kk, vv, np.arange(n)[None] <= np.arange(Tq)[:, None] + n - Tq
    _check_attention(O, Q, None, 2, keys_of, DT[dtype], 2.0 ** -11 if dtype != "f32" else 0.0, q16=dtype == "bf16")
    assert sn.last_status() == 0


def test_prompts_on_two_streams(sn):
    """Blocks of many rows on a cache whose axis is split, from two contexts at once, in turn with single tokens."""
    calls = [_cache_call(*s, seed=30 + i) for i, s in enumerate([(2, 90, 60, 32, 4, 2, 128), (3, 1, 300, 16, 8, 1, 128), (1, 300, 40, 64, 4, 1, 64)])]
    alone = [sn.cache_attend_fwd(*c) for c in calls]
    torch.cuda.synchronize()
    other = sentry.Sentry(0)
    try:
        streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
        for i in range(24):
            for s, st in zip((sn, other), streams):
                with torch.cuda.stream(st):
                    got.append((i % 3, s.cache_attend_fwd(*calls[i % 3])))
        torch.cuda.synchronize()
        assert all(torch.equal(o, alone[i]) for i, o in got)
        assert sn.last_status() == 0 and other.last_status() == 0
    finally:
        other.close()


def test_workspace_outgrown_on_another_stream():
    """A workspace from one stream's memory, used on another stream and replaced there while the call that uses it still waits: whoever
    allocates on the first stream does not get it until then."""
    g = torch.Generator(device="cuda").manual_seed(4)
    Q, K, V = (torch.randn((2, h, t, 64), generator=g, device="cuda").bfloat16() for h, t in ((4, 1), (1, 6000), (1, 6000)))
    big = [torch.randn((8, h, t, 128), generator=g, device="cuda").bfloat16() for h, t in ((32, 8), (4, 6000), (4, 6000))]
    s = sentry.Sentry(0)
    try:
        want = s.cross_attend_fwd(Q, K, V)
        size, side = s._ws.numel(), torch.cuda.Stream()
        torch.cuda.synchronize()
        a = torch.randn((4096, 4096), device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                a = a @ a * 1e-3                          # keeps the stream busy for some ten milliseconds
            O = s.cross_attend_fwd(Q, K, V)
            s.cross_attend_fwd(*big)
        assert s._ws.numel() > size
        junk = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        for _ in range(200):
            for j in junk:
                j.fill_(255)
        torch.cuda.synchronize()
        assert torch.equal(O, want)
    finally:
        s.close()


# (calls large enough for the form of many rows: as above, and views, bad heads, bad pages, odd scales, two streams for it)
MANY = [("i8", "bf16", 3, 140, 10, 128, 8, 2, 128, 8, 1), ("e4m3", "f16", 4, 200, 32, 64, 4, 2, 128, 3, 0), ("e4m3", "bf16", 25, 70, 20, 64, 2, 1, 64, 2, 1),
        ("i8", "f16", 1, 1000, 40, 128, 2, 2, 64, 2, 1), ("e4m3", "f16", 2, 129, 560, 16, 2, 2, 32, 2, 0), ("i8", "bf16", 40, 65, 24, 32, 4, 4, 16, 4, 1),
        ("i8", "f16", 1, 65, 1000, 64, 1, 1, 128, 1, 0), ("e4m3", "bf16", 4, 700, 30, 16, 4, 4, 64, 2, 1)]


@pytest.mark.parametrize("case", MANY, ids=lambda c: "-".join(map(str, c)))
def test_cache_attend_many_rows(sn, case):
    test_cache_attend(sn, case)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 16)])
def test_rising_scores_cache_many_rows(sn, fmt, dtype, d, page):
    test_rising_scores_cache(sn, fmt, dtype, 2100, 2100, d, page)


def test_cache_edges_many_rows(sn):
    test_cache_attend_edges(sn, "bf16", 1200)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales_of_any_sign_many_rows(sn, fmt, dtype):
    test_scales_of_any_sign(sn, fmt, dtype, 5000)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", [(9, 100, 900, 4, 2, 16, 4, "both"), (5, 150, 1030, 4, 2, 64, 3, "interleaved"), (4, 300, 520, 4, 4, 32, 4, "modalities")],
                         ids=lambda c: "x".join(map(str, c)))
def test_cross_attend_many_rows(sn, case, dtype):
    test_cross_attend(sn, case, dtype)


def test_rising_scores_many_rows(sn):
    for d in (16, 64):
        for dtype in ("bf16", "f16"):
            test_rising_scores(sn, dtype, 2000, 1500, d, 300.0)


@pytest.mark.parametrize("d", [32, 128])
def test_views_and_bad_heads_many_rows(sn, d):
    B, Tq, Tk, Hq, Hk = 6, 300, 500, 4, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    kv = torch.randn((B, Tk, 2, Hk, d), generator=g, device="cuda").bfloat16()
    q = torch.randn((2 * B, Tq, Hq, d), generator=g, device="cuda").bfloat16()
    Q, K, V = q.transpose(1, 2)[::2], kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    full = sn.cross_attend_fwd(Q, K, V)
    assert torch.equal(full, sn.cross_attend_fwd(Q.contiguous(), K.contiguous(), V.contiguous()))
    one = K[:1].expand(B, -1, -1, -1)
    assert torch.equal(sn.cross_attend_fwd(Q, one, V), sn.cross_attend_fwd(Q, one.contiguous(), V))
    kept = torch.tensor([[0, 1, 1, 1], [-1, 2, 3, 9], [0, 0, 0, 0], [3, 2, 1, 0], [4, 4, 4, 4], [2, 2, 3, 0]], dtype=torch.int32, device="cuda")
    assert sn.last_status() == 0
    O = sn.cross_attend_fwd(Q, K, V, kept, O=torch.full((B, 4, Tq, d), 3.0, dtype=torch.bfloat16, device="cuda"))
    assert sn.last_status() == sentry.STATUS_BIT_BAD_INDEX
    for b, row in enumerate(kept.tolist()):
        for j, h in enumerate(row):
            assert torch.equal(O[b, j], full[b, h] if 0 <= h < Hq else torch.zeros_like(O[b, j])), (b, j)


def test_many_rows_of_a_cache_on_two_streams(sn):
    """As test_prompts_on_two_streams, with calls that hold tensor memory."""
    calls = [_cache_call(*s, seed=50 + i) for i, s in enumerate([(2, 300, 60, 32, 4, 2, 128), (3, 1, 300, 16, 8, 1, 128), (4, 400, 40, 64, 4, 1, 64)])]
    alone = [sn.cache_attend_fwd(*c) for c in calls]
    torch.cuda.synchronize()
    other = sentry.Sentry(0)
    try:
        streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
        for i in range(24):
            for s, st in zip((sn, other), streams):
                with torch.cuda.stream(st):
                    got.append((i % 3, s.cache_attend_fwd(*calls[i % 3])))
        torch.cuda.synchronize()
        assert all(torch.equal(o, alone[i]) for i, o in got)
        assert sn.last_status() == 0 and other.last_status() == 0
    finally:
        other.close()
