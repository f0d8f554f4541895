"""The serving calls at sizes, weights and callers between those of test_gpu_serving.py, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import paper_2604_08971_b200 as sentry
from tests import serving_reference as ref
from tests.test_gpu_serving import DT, _cuda, _pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sn():
    s = sentry.Sentry(0)
    yield s
    s.close()


# (prompts shorter than a page, whose rows' pieces are no power of two times a warp's share: dtype, Hk, page, d, T)
SHORT = [("bf16", 2, 64, 128, 48), ("f16", 3, 64, 128, 50), ("bf16", 1, 64, 128, 63), ("bf16", 2, 128, 128, 50), ("f16", 2, 128, 128, 80), ("bf16", 5, 128, 128, 100),
         ("bf16", 2, 128, 128, 127), ("f16", 2, 128, 64, 100), ("f32", 2, 32, 128, 25), ("f32", 3, 64, 64, 50), ("f32", 2, 64, 128, 40), ("f32", 1, 64, 128, 63),
         ("f32", 2, 128, 32, 100), ("f32", 2, 128, 64, 70)]


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype,Hk,page,d,T", SHORT)
def test_append_short_prompts(sn, fmt, dtype, Hk, page, d, T):
    """Two calls behind one another, the second louder: from an empty page, from partly filled ones, across the end of one."""
    rng = np.random.default_rng(T + d)
    lengths = np.array([0, 5, page - T, page - 1, 2 * page - 7], np.int32)
    B, cols = len(lengths), 5
    n_pages = B * cols + 1
    pools = [_pool(rng, n_pages, Hk, page, d, fmt) for _ in range(2)]
    table = rng.permutation(n_pages)[:B * cols].reshape(B, cols).astype(np.int32)
    dev = [torch.from_numpy(x).cuda() for p in pools for x in p]
    dt, dlen = torch.from_numpy(table).cuda(), torch.from_numpy(lengths).cuda()
    for call in range(2):
        g = torch.Generator().manual_seed(call)
        K, V = (torch.randn((B, Hk, T, d), generator=g).mul_(0.01 * 30.0 ** call).to(DT[dtype]) for _ in range(2))
        ids = masks = None
        if call:
            ids, masks = (np.arange(T) % 3 // 2).astype(np.int32), np.array([3, 1, 3, 2, 3], np.int32)
        dlen = sn.cache_append(K.cuda(), V.cuda(), dev[0], dev[2], dev[1], dev[3], dt, dlen, *_cuda(ids, masks))
        for X, (c, s) in zip((K, V), pools):
            now = ref.append(X.double().numpy(), c, s, table, lengths, ref.present(B, T, None, ids, masks), fmt)
        lengths = now
        np.testing.assert_array_equal(dlen.cpu().numpy(), lengths)
        for i, (c, s) in enumerate(pools):
            np.testing.assert_array_equal(dev[2 * i + 1].cpu().numpy(), s)
            np.testing.assert_array_equal(dev[2 * i].cpu().numpy(), c)
    assert sn.last_status() == 0


# ------------------------------------------------------------------------------------------ small weights beside a large one

def _strong(rng, N, d, below, at):
    """q [d] and k [N,d] whose weights are 2^-below of the strong ones' at keys `at`, half a power of two up and down."""
    q = np.where(np.arange(d) % 2, 1.0, -1.0)
    k = rng.uniform(-0.5, 0.5, N) * np.log(2)
    k[at] = below * np.log(2)
    return q, (k / np.sqrt(d))[:, None] * q


def _check_alike(O, q, k, v, dtype, weight_err):
    """Every row of O against the same one; a sink's values leave nothing but the small weights'."""
    want, tol = ref.attention(q[None], k, v, np.ones((1, k.shape[0]), bool), dtype, weight_err)
    rows = O.detach().cpu().double().numpy().reshape(-1, q.shape[0])
    ref.check(rows, np.broadcast_to(want, rows.shape), np.broadcast_to(tol, rows.shape))


# Samples enough that no axis of keys is split, so that every small weight meets a strong one: every fourth tile of 32 keys goes to the same warp.
AT = [3, 40, 77, 100]
FEW, MANY = (600, 1), (160, 300)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("sink", [True, False])
@pytest.mark.parametrize("below", [16.3, 20.6, 24.4])
@pytest.mark.parametrize("B,Tq,N,d", [FEW + (8200, 64), MANY + (8200, 64), FEW + (5003, 128), MANY + (5003, 128), FEW + (3001, 32), (1, 1, 3001, 64)])
def test_small_weights_cross(sn, dtype, sink, below, B, Tq, N, d):
    """fp16 weights are good to half a step, 2^-11 of themselves, down to 2^-25 of a row's largest."""
    if dtype == "f32":
        B = 2
    rng = np.random.default_rng(N)
    q, k = _strong(rng, N, d, below, AT)
    v = rng.uniform(0.5, 1.5, (N, d))
    v[AT] = 0.0 if sink else 1.0
    Q = torch.from_numpy(q).to(DT[dtype]).expand(B, 1, Tq, d).contiguous()
    K, V = (torch.from_numpy(x).to(DT[dtype])[None, None] for x in (k, v))
    O = sn.cross_attend_fwd(Q.cuda(), K.cuda().expand(B, 1, N, d), V.cuda().expand(B, 1, N, d))
    assert sn.last_status() == 0
    weight_err = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 0.0}[dtype]
    _check_alike(O, q, K[0, 0].double().numpy(), V[0, 0].double().numpy(), DT[dtype], weight_err)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("sink", [True, False])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("below,times", [(16.3, 1), (24.4, 1), (16.3, 16), (20.4, 16), (20.4, 1.0 / 16), (14.4, 1024)])
@pytest.mark.parametrize("B,Tq,N,d,page", [FEW + (8200, 64, 32), MANY + (8200, 64, 32), FEW + (5003, 128, 16), MANY + (5003, 128, 64), (1, 1, 3001, 64, 16)])
def test_small_weights_cache(sn, dtype, sink, fmt, below, times, B, Tq, N, d, page):
    """The same on a cache, for the product of a weight and its page's value scale: the strong keys' pages have `times` the others' scale."""
    if dtype == "f32":
        B = 2
    rng = np.random.default_rng(N)
    cols = -(-N // page)
    q, k = _strong(rng, N, d, below, AT)
    code = (lambda x: x.astype(np.int8)) if fmt == "i8" else ref.to_e4m3
    strong = np.array(sorted({n // page for n in AT}))
    # (keys that share a strong one's page have coarse codes: the scores are what the codes say)
    ks = np.full((cols, 1), np.abs(k[np.setdiff1d(np.arange(N), AT)]).max() / (100 if fmt == "i8" else 400), np.float32)
    ks[strong] = np.float32(np.abs(k).max() / (127 if fmt == "i8" else 448))
    vs = np.full((cols, 1), 0.01, np.float32)
    vs[strong] *= times
    pad = np.zeros((cols * page, d))
    pad[:N] = k
    kc = code(np.rint(pad / np.repeat(ks, page, 0)) if fmt == "i8" else pad / np.repeat(ks, page, 0)).reshape(cols, 1, page, d)
    v = rng.integers(32, 127, (cols * page, d)).astype(float)
    for p in strong:                                          # values of the strong keys' page: what its scale makes large is the strong key's alone
        v[p * page:(p + 1) * page] = 0.0
    v[AT] = 0.0 if sink else 100.0
    vc = code(v).reshape(cols, 1, page, d)
    table = np.broadcast_to(np.arange(cols, dtype=np.int32), (B, cols)).copy()
    Q = torch.from_numpy(q).to(DT[dtype]).expand(B, 1, Tq, d).contiguous()
    O = sn.cache_attend_fwd(Q.cuda(), *_cuda(kc, vc, ks, vs, table, np.full(B, N, np.int32)))
    assert sn.last_status() == 0
    kk, vv = ((ref.values(c, fmt) * s[..., None, None].astype(np.float64)).reshape(-1, d)[:N] for c, s in ((kc, ks), (vc, vs)))
    _check_alike(O, q, kk, vv, DT[dtype], 2.0 ** -11 if dtype != "f32" else 0.0)


# (all small weights alike, so that they round alike; several sizes, since one may happen to be a number of the type)
EQUAL = [21.23, 22.41, 23.17, 23.77, 24.37]


@pytest.mark.parametrize("below", EQUAL)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,Tq,N,d", [MANY + (8200, 64), MANY + (5003, 128), (2, 300, 5003, 128), FEW + (8200, 64)])
def test_equal_small_weights_cross(sn, dtype, below, B, Tq, N, d):
    q, k = _strong(np.random.default_rng(N), N, d, below, AT)
    k[np.setdiff1d(np.arange(N), AT)] = 0.0
    v = np.ones((N, d))
    v[AT] = 0.0
    Q = torch.from_numpy(q).to(DT[dtype]).expand(B, 1, Tq, d).contiguous()
    K, V = (torch.from_numpy(x).to(DT[dtype])[None, None] for x in (k, v))
    O = sn.cross_attend_fwd(Q.cuda(), K.cuda().expand(B, 1, N, d), V.cuda().expand(B, 1, N, d))
    _check_alike(O, q, K[0, 0].double().numpy(), V[0, 0].double().numpy(), DT[dtype], 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11)


@pytest.mark.parametrize("below", EQUAL)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("B,Tq,N,d,page", [MANY + (8200, 64, 32), MANY + (5003, 128, 64), (2, 600, 5003, 128, 64), FEW + (8200, 64, 32)])
def test_equal_small_weights_cache(sn, dtype, fmt, below, B, Tq, N, d, page):
    q, _ = _strong(np.random.default_rng(N), N, d, below, AT)
    cols, top = -(-N // page), 127 if fmt == "i8" else 448
    k, v = np.zeros((cols * page, d)), np.full((cols * page, d), 96.0)
    k[AT] = top * q
    v[AT] = 0.0
    code = (lambda x: x.astype(np.int8)) if fmt == "i8" else ref.to_e4m3
    kc, vc = (code(x).reshape(cols, 1, page, d) for x in (k, v))
    ks, vs = np.full((cols, 1), below * np.log(2) / np.sqrt(d) / top, np.float32), np.full((cols, 1), 0.01, np.float32)
    table = np.broadcast_to(np.arange(cols, dtype=np.int32), (B, cols)).copy()
    Q = torch.from_numpy(q).to(DT[dtype]).expand(B, 1, Tq, d).contiguous()
    O = sn.cache_attend_fwd(Q.cuda(), *_cuda(kc, vc, ks, vs, table, np.full(B, N, np.int32)))
    kk, vv = ((ref.values(c, fmt) * s[..., None, None].astype(np.float64)).reshape(-1, d)[:N] for c, s in ((kc, ks), (vc, vs)))
    _check_alike(O, q, kk, vv, DT[dtype], 2.0 ** -11)


def test_linear_of_the_most_rows(sn):
    """2^31 - 1 rows: the last tile ends where 32 bits do."""
    M, K = 2 ** 31 - 1, 16
    if torch.cuda.mem_get_info()[0] < 70 << 30:
        pytest.skip("needs 70 GB")
    x, xs = torch.ones((M, K), dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda")
    rows = [0, 255, 256, 2 ** 30, M - 256, M - 2, M - 1]
    for i, r in enumerate(rows):
        x[r] = i + 2
    w, ws = torch.ones((1, K), dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda")
    Y = sn.linear_i8(x, xs, w, ws)
    assert sn.last_status() == 0 and Y.shape == (M, 1)
    assert [Y[r, 0].item() for r in rows] == [16.0 * (i + 2) for i in range(len(rows))]
    assert int((Y == 16).sum()) == M - len(rows)
    del x, xs, Y
    torch.cuda.empty_cache()


class _Allocations(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.shapes = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        if func._schema.name == "aten::empty":
            self.shapes.append(tuple(args[0]))
        return func(*args, **(kwargs or {}))


def test_dispatch_modes_see_outputs(sn):
    """A mode that watches allocations sees the outputs that the calls make, and changes none of them."""
    scores, masks = torch.rand((8, 40), device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    x, w = torch.randn((6, 64), device="cuda").bfloat16(), torch.randn((5, 64), device="cuda")
    Q, K = torch.randn((2, 4, 3, 32), device="cuda").half(), torch.randn((2, 2, 7, 32), device="cuda").half()
    calls = [(lambda: [sn.gate_select(scores, masks, 9)], [(8, 9)]), (lambda: list(sn.quantize_rows_i8(x)), [(6, 64), (6,)]),
             (lambda: [sn.linear_i8(*codes, *weights)], [(6, 5)]), (lambda: [sn.cross_attend_fwd(Q, K, K)], [(2, 4, 3, 32)])]
    codes, weights = sn.quantize_rows_i8(x), sn.quantize_rows_i8(w)
    for call, shapes in calls:
        want = call()
        with _Allocations() as mode:
            got = call()
        assert mode.shapes == shapes
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_sample_of_shared_heads(sn, dtype):
    """One tensor for every head of one sample: what the heads' keys would take if each had its own is no limit."""
    H, T, d, n = 256, (1 << 23) + 8, 128, 100
    q, one = torch.randn((1, H, 1, d), device="cuda").to(DT[dtype]), torch.empty((1, 1, T, d), dtype=DT[dtype], device="cuda")
    one[:, :, :n] = torch.randn((n, d), device="cuda")
    K, lengths = one.expand(1, H, T, d), torch.tensor([n], dtype=torch.int32, device="cuda")
    O = sn.cross_attend_fwd(q, K, K, key_lengths=lengths)
    k = one[0, 0, :n].double().cpu().numpy()
    for h in (0, 100, 255):
        want, tol = ref.attention(q[0, h].double().cpu().numpy(), k, k, np.ones((1, n), bool), DT[dtype], 2.0 ** -8 if dtype == "bf16" else 0.0)
        ref.check(O[0, h].double().cpu().numpy(), want, tol)
    assert sn.last_status() == 0
    del one, K
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------ keys from memory rather than the L2

# B, Tq, N, Hq, Hk, d, k_h, runs of one modality
FAR = [(17, 1, 7961, 21, 3, 128, 21, 900), (64, 1, 3424, 8, 2, 128, 4, 1200), (64, 2, 2979, 14, 2, 128, 7, 20), (64, 2, 7874, 16, 4, 128, 16, 0), (3, 5, 60001, 4, 1, 128, 4, 33),
       (64, 1, 5995, 16, 4, 64, 8, 700), (64, 2, 9001, 14, 2, 32, 7, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", FAR, ids=lambda c: "x".join(map(str, c)))
def test_cross_attend_keys_beyond_the_l2(sn, case, dtype):
    """Copies that land late and out of order: the same bits five times, and the definition's values."""
    B, Tq, N, Hq, Hk, d, k_h, run = case
    g, rng = torch.Generator(device="cuda").manual_seed(N), np.random.default_rng(N)
    kv = torch.randn((B, N, 2, Hk, d), generator=g, device="cuda", dtype=DT[dtype])
    Q = torch.randn((B, Hq, Tq, d), generator=g, device="cuda", dtype=DT[dtype])
    K, V = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    kept = np.stack([np.sort(rng.permutation(Hq)[:k_h]) for _ in range(B)]).astype(np.int32)
    ids = masks = None
    if run:
        ids, masks = (np.arange(N) // run % 5).astype(np.int32), rng.integers(1, 32, B).astype(np.int32)
    args = _cuda(kept, ids, masks)
    sweep = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    out = []
    for i in range(5):
        sweep.fill_(i)
        out.append(sn.cross_attend_fwd(Q, K, V, *args))
    assert sn.last_status() == 0
    assert all(torch.equal(o, out[0]) for o in out)
    ok = ref.present(B, N, None, ids, masks)
    for b in sorted({0, 3, 5, B // 2, B - 1} & set(range(B))):
        q, o, here = Q[b].double().cpu().numpy(), out[0][b].double().cpu().numpy(), torch.from_numpy(ok[b]).cuda()
        for j in range(0, k_h, 3):
            h = int(kept[b, j])
            k, v = (x[b, h * Hk // Hq][here].double().cpu().numpy() for x in (K, V))
            want, tol = ref.attention(q[h], k, v, np.ones((Tq, len(k)), bool), DT[dtype], 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11)
            ref.check(o[j], want, tol, "sample %d head %d" % (b, h))
    del kv, K, V, sweep
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("B,Tq,N,page", [FEW + (2100, 32), MANY + (2100, 32), (2, 3, 9001, 16), (3, 700, 5003, 64), FEW + (400, 16)])
@pytest.mark.parametrize("large", [0, 1, 5])
def test_value_scales_far_apart(sn, dtype, fmt, B, Tq, N, page, large):
    """Every seventh page has values 2^60 times the others' and no weight to speak of: what the others hold is the result."""
    d = 64
    if dtype == "f32":
        B = min(B, 3)
    rng = np.random.default_rng(N)
    cols, top = -(-N // page), 127 if fmt == "i8" else 448
    q = np.where(np.arange(d) % 2, 1.0, -1.0)
    far = np.arange(cols) % 7 == large
    code = (lambda x: np.rint(x).astype(np.int8)) if fmt == "i8" else ref.to_e4m3
    k = rng.uniform(-1, 1, (cols, page, 1)) * q * top
    k[far] = -top * q
    ks = np.full((cols, 1), 1.0 / (8 * top), np.float32)
    ks[far] = 300.0 / (8 * top)                                # scores of -300
    vs = (2.0 ** rng.uniform(-33, -30, (cols, 1))).astype(np.float32)
    vs[far] *= np.float32(2.0 ** 60)
    kc, vc = code(k).reshape(cols, 1, page, d), code(rng.uniform(-1, 1, (cols, 1, page, d)) * top)
    table = np.broadcast_to(np.arange(cols, dtype=np.int32), (B, cols)).copy()
    Q = torch.from_numpy(q).to(DT[dtype]).expand(B, 1, Tq, d).contiguous()
    O = sn.cache_attend_fwd(Q.cuda(), *_cuda(kc, vc, ks, vs, table, np.full(B, N, np.int32)))
    kk, vv = ((ref.values(c, fmt) * s[..., None, None].astype(np.float64)).reshape(-1, d)[:N] for c, s in ((kc, ks), (vc, vs)))
    if dtype == "f16":                                        # (its results are below half's range: in its smallest steps)
        vv = vv * 2.0 ** 22
        O = sn.cache_attend_fwd(Q.cuda(), *_cuda(kc, vc, ks, vs * np.float32(2.0 ** 22), table, np.full(B, N, np.int32)))
    assert sn.last_status() == 0
    _check_alike(O, q, kk, vv, DT[dtype], 2.0 ** -11 if dtype != "f32" else 0.0)
