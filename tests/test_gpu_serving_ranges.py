"""The serving calls at sizes, weights and callers between those of test_gpu_serving.py, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

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
