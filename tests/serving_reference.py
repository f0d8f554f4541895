"""The serving operators in 64 bits, from their definitions (include/sentry.h), and how far a result may be from them."""
import math

import numpy as np
import torch

STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # half a step, relative to the value
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}   # half of the smallest step
RECIP = np.float32(1) / np.float32(127)


def quantize_rows(x):
    """codes int8, scales fp32 of the rows of a tensor."""
    f = x.float().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(f).max(1)
        s = np.where(top > 0, np.maximum(top * RECIP, np.float32(2.0 ** -126)), np.float32(0)).astype(np.float32)
        bad = ~np.isfinite(f).all(1)
        s[bad] = np.nan
        ok = (s > 0)[:, None]
        q = np.where(ok, f.astype(np.float64) / np.where(ok, s.astype(np.float64)[:, None], 1), 0)
    return np.clip(np.rint(q), -127, 127).astype(np.int8), s


def e4m3_values():
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7), m / 8 * 2.0 ** -6) * np.where(c & 128, -1, 1)
    v[0x7f] = v[0xff] = np.nan
    return v


E4M3 = e4m3_values()
_POS = E4M3[:0x7f]


def to_e4m3(q):
    """Codes of the nearest e4m3 values, ties to the even code, at most 448."""
    a = np.minimum(np.abs(q), 448.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, 0x7e)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (pick | np.where(np.signbit(q), 128, 0)).astype(np.uint8)


def values(codes, fmt):
    return codes.astype(np.float64) if fmt == "i8" else E4M3[codes]


def encode(v, s, fmt):
    if not s > 0:
        return np.zeros(v.shape, np.int8 if fmt == "i8" else np.uint8)
    q = v / float(s)
    return np.clip(np.rint(q), -127, 127).astype(np.int8) if fmt == "i8" else to_e4m3(q)


def page_scale(top, fmt):
    top = np.float32(top)
    if not top > 0:
        return np.float32(0)
    if fmt == "i8":
        return max(np.float32(top * RECIP), np.float32(2.0 ** -126))
    m, e = math.frexp(float(top))
    return np.float32(2.0 ** max(e - (8 if m > 0.875 else 9), -126))


def append(X, codes, scales, table, lengths, present, fmt):
    """In place, one of the two pools: X [B,Hk,T,d] float64, codes [pages,Hk,page,d], scales [pages,Hk], present [B,T]."""
    n_pages, Hk, page, _ = codes.shape
    cap = table.shape[1] * page
    out = []
    for b in range(X.shape[0]):
        n = int(np.clip(lengths[b], 0, cap))
        if n != lengths[b]:
            out.append(n)
            continue
        t = np.flatnonzero(present[b])[:cap - n]
        out.append(n + len(t))
        while len(t):
            j, slot = divmod(n, page)
            now, t = t[:page - slot], t[page - slot:]
            n += len(now)
            p = int(table[b, j])
            if not 0 <= p < n_pages:
                continue
            for h in range(Hk):
                x = X[b, h, now]
                s, old = page_scale(np.abs(x).max(), fmt), scales[p, h]
                if slot:
                    s = np.float32(np.nan) if np.isnan(old) else max(s, old)
                if not np.isfinite(x).all():
                    s = np.float32(np.nan)
                if slot and not s == old:
                    codes[p, h, :slot] = encode(values(codes[p, h, :slot], fmt) * float(old), s, fmt)
                codes[p, h, slot:slot + len(now)] = encode(x, s, fmt)
                scales[p, h] = s
    return np.array(out, np.int32)


def present(B, T, lengths=None, ids=None, masks=None):
    ok = np.ones((B, T), bool)
    if lengths is not None:
        ok &= np.arange(T)[None] < np.asarray(lengths)[:, None]
    if ids is not None:
        i = np.asarray(ids)
        ok &= np.array([[0 <= m < 32 and (int(w) >> int(m)) & 1 == 1 for m in i] for w in masks], bool).reshape(B, T)
    return ok


def attention(q, k, v, visible, dtype, weight_err, q_abs_err=0.0):
    """softmax(q k / sqrt d) v and how far a kernel's result in `dtype` may be from it.  q [R,d], k, v [N,d], visible [R,N]; float64.

    A score is a sum of d products in fp32, truncated rather than rounded inside a matrix instruction (2^-22 of the sum of their sizes a
    step, d steps at most), scaled into log2 by two roundings and exponentiated with an error of 2^-22; with q off by q_abs_err per element
    besides.  A relative error e of every weight moves a quotient of sums by 2 e of the weighted sizes; the weights meet v rounded by
    weight_err, and N products are summed in fp32, 2^-22 of the sum of sizes for every 16 of them.  Then one rounding to `dtype`."""
    R, d = q.shape
    if k.shape[0] == 0:
        return np.zeros((R, d)), np.zeros((R, d))
    scale = 1 / math.sqrt(d)
    s = np.where(visible, q @ k.T * scale, -np.inf)
    size = np.where(visible, np.abs(q) @ np.abs(k).T * scale, 0).max(1, keepdims=True)
    drift = d * 2.0 ** -22 * size + 2.0 ** -21 * size + 2.0 ** -21
    if np.ndim(q_abs_err):
        drift = drift + (np.where(visible, q_abs_err @ np.abs(k).T, 0) * scale).max(1, keepdims=True)
    top = s.max(1, keepdims=True)
    p = np.where(visible, np.exp(s - np.where(np.isfinite(top), top, 0)), 0)
    total = p.sum(1, keepdims=True)
    p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
    want = p @ v
    rel = 2 * drift + 2 * weight_err + (k.shape[0] / 16 + 32) * 2.0 ** -22
    return want, rel * (p @ np.abs(v)) + STEP[dtype] * np.abs(want) * (1 + rel) + TINY[dtype]


def check(got, want, tol, what=""):
    off = np.abs(got - want)
    bad = ~(off <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3g times what may be" % (what, bad.sum(), bad.size, (off / np.maximum(tol, 1e-300)).max())
