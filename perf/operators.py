"""The 8-bit serving operators of this library and dense cross attention, as cases that can be timed and compared.

Each case is one call (or the two calls that belong together) of a program that serves a pruned multimodal encoder with a decoder or
a streaming head behind it, through `paper_2604_08971_b200.Sentry`:

  linear   a projection in 8-bit integers: the rows of X are quantised (one scale per token), then multiplied with weights that were
           quantised once (one scale per output channel)
  cross    attention from a decoder's rows to an encoder's states of another length: kept heads, keys of absent modalities left out
  cache    attention over a paged cache of 8-bit keys and values, one scale per page and head, for single tokens and short blocks
  append   new keys and values of the present tokens, quantised into the pages of such a cache

The plain forms below are the operators' definitions in elementary torch operations; `exact` is their definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ESIZE = {"f32": 4, "bf16": 2, "f16": 2}
_CTX = []


def _sentry():
    """The library context, made once and kept as a server keeps it."""
    if not _CTX:
        import paper_2604_08971_b200 as sentry
        _CTX.append(sentry.Sentry(0))
    return _CTX[0]


def listed():
    return [
        # K and V of the few tokens an on-line step brings: the weights' bytes and the calls' latency are all there is
        dict(name="linear_token", kind="linear", dtype="bf16", M=4, K=1024, N=2048, bias=False),
        # a ragged batch in IEEE half on an odd number of kept channels, with a bias
        dict(name="linear_ragged_f16", kind="linear", dtype="f16", M=1531, K=768, N=1229, bias=True),
        # K and V of a whole batch of encoder states (128 windows of 512 tokens)
        dict(name="linear_encoder", kind="linear", dtype="bf16", M=65536, K=1024, N=2048, bias=False),
        # one decoder token per sample looks at its encoder's states
        dict(name="cross_token", kind="cross", dtype="bf16", B=16, Tq=1, Tk=1500, Hq=12, Hk=4, d=64, k_h=12, keys="all"),
        # fusion queries on ragged modalities, every subset of three sensors, none at all among them; pruned heads
        dict(name="cross_fusion_f16", kind="cross", dtype="f16", B=32, Tq=211, Tk=648, Hq=12, Hk=4, d=64, k_h=7, keys="211,97,340"),
        # the largest: long prompts on long encoder states
        dict(name="cross_long", kind="cross", dtype="bf16", B=4, Tq=4096, Tk=8192, Hq=16, Hk=4, d=128, k_h=16, keys="all"),
        # the fp32 call people validate with, padded encoder states of several lengths
        dict(name="cross_f32", kind="cross", dtype="f32", B=2, Tq=129, Tk=333, Hq=4, Hk=2, d=32, k_h=4, keys="lengths"),
        # the ordinary decoding step of a server: one token for each of 32 samples of very different lengths
        dict(name="cache_token_e4m3", kind="cache", fmt="e4m3", dtype="bf16", B=32, Tq=1, cap=4096, page=64, Hq=16, Hk=4, d=128,
             k_h=16, causal=False, lens="ragged"),
        # two recordings of hours: the axis of keys has to be split over the GPU
        dict(name="cache_long_i8", kind="cache", fmt="i8", dtype="bf16", B=2, Tq=1, cap=131072, page=128, Hq=8, Hk=2, d=64, k_h=8,
             causal=False, lens="full"),
        # a block of new tokens that see one another causally; small pages, pruned heads
        dict(name="cache_block_i8", kind="cache", fmt="i8", dtype="f16", B=16, Tq=7, cap=1024, page=16, Hq=12, Hk=4, d=32, k_h=7,
             causal=True, lens="ragged"),
        # the decoding step's one new token per sample, into partly filled pages
        dict(name="append_token_e4m3", kind="append", fmt="e4m3", dtype="bf16", B=32, T=1, cap=512, page=64, Hk=4, d=128, keys="all",
             start="ragged"),
        # a prompt's keys and values with modalities missing, into fresh pages
        dict(name="append_prompt_i8", kind="append", fmt="i8", dtype="bf16", B=32, T=2048, cap=2048, page=32, Hk=4, d=128,
             keys="700,648,700", start="empty"),
    ]


# ------------------------------------------------------------------------------------------ drawing

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    Hk = rng.choice([1, 2, 4, 4, 8])
    Hq = Hk * rng.choice([1, 2, 3, 4, 4, 8])
    return Hq, Hk, rng.choice([Hq, Hq, max(1, int(Hq * rng.uniform(0.3, 1.0)))])


def _keys(rng, T):
    how = rng.choice(["all", "lengths", "modalities"])
    if how != "modalities" or T < 8:
        return "lengths" if how == "lengths" else "all"
    cuts = sorted(rng.sample(range(1, T), rng.choice([1, 2, 2, 3])))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [T]))


def _candidate(rng):
    kind = rng.choice(["linear", "cross", "cache", "append"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16"]))
    if kind == "linear":
        c.update(M=_log_int(rng, 1, 65536), K=16 * _log_int(rng, 4, 256), N=_log_int(rng, 16, 8192), bias=rng.random() < 0.5)
        return c
    d = rng.choice([16, 32, 64, 64, 128, 128])
    Hq, Hk, k_h = _heads(rng)
    B = _log_int(rng, 1, 64)
    if kind == "cross":
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f16", "f16", "f32"])
        top = 512 if c["dtype"] == "f32" else 8192
        Tk = _log_int(rng, 1, top)
        c.update(B=B, Tq=rng.choice([1, _log_int(rng, 1, 4096 if top > 512 else 256), _log_int(rng, 1, 64)]), Tk=Tk, Hq=Hq, Hk=Hk, d=d,
                 k_h=k_h, keys=_keys(rng, Tk))
        return c
    page = rng.choice([16, 32, 64, 64, 128])
    c.update(fmt=rng.choice(["e4m3", "i8"]), B=B, page=page, Hk=Hk, d=d)
    if kind == "cache":
        c.update(Tq=rng.choice([1, 1, 1, rng.randint(2, 16), _log_int(rng, 16, 256)]), cap=page * _log_int(rng, 1, 131072 // page), Hq=Hq,
                 k_h=k_h, causal=rng.random() < 0.5, lens=rng.choice(["ragged", "full"]))
        return c
    T = rng.choice([1, _log_int(rng, 1, 2048)])
    c.update(T=T, keys=_keys(rng, T), start=rng.choice(["empty", "ragged"]))
    c["cap"] = page * -(-(2 * T + rng.randint(1, 300)) // page)
    return c


def draw(rng):
    """One more case of the ranges above; never more work than the largest listed one."""
    top = [work(c) for c in listed()]
    most_bytes, most_flops = max(w["bytes"] for w in top), max(w["flops"] for w in top)
    while True:
        c = _candidate(rng)
        w = work(c)
        if w["bytes"] > most_bytes or w["flops"] > most_flops:
            continue
        if c["kind"] == "cross" and c["B"] * c["k_h"] * c["Tq"] * c["Tk"] > 4 * 16 * 4096 * 8192:   # the plain form's scores
            continue
        if c["kind"] == "cross" and c["dtype"] == "f32" and w["flops"] > 2e9:   # fp32 is for validation
            continue
        if c["kind"] in ("cache", "append") and c["B"] * c["cap"] * c["Hk"] * c["d"] > 1 << 27:
            continue
        if c["kind"] == "cache" and c["B"] * c["k_h"] * c["cap"] * (c["Tq"] + c["d"]) > 1 << 30:
            continue
        return c


# ------------------------------------------------------------------------------------------ shapes

def _modalities(case):
    return [int(x) for x in case["keys"].split(",")]


def _present(case, T):
    """Present tokens of every sample, as the masks or lengths of the batch leave them (the same for every seed)."""
    B = case["B"]
    if case["keys"] == "all":
        return [T] * B
    if case["keys"] == "lengths":
        return [T - (T * ((5 * b + 3) % 8)) // 8 for b in range(B)]
    parts = _modalities(case)
    return [sum(n for j, n in enumerate(parts) if ((b % (1 << len(parts))) >> j) & 1) for b in range(B)]


def _stored(case):
    """Tokens already in the cache, per sample."""
    B, cap = case["B"], case["cap"]
    if case["kind"] == "append":
        room = cap - case["T"]
        return [0 if case["start"] == "empty" else (room * ((7 * b + 3) % 16)) // 16 for b in range(B)]
    return [cap if case["lens"] == "full" else max(1, cap - (3 * cap * ((5 * b + 3) % 16)) // 64) for b in range(B)]


def _groups(case):
    """Expected KV groups that kept heads reference."""
    r = case["Hq"] // case["Hk"]
    rest = case["Hq"] - r
    return case["Hk"] * (1 - (math.comb(rest, case["k_h"]) if rest >= case["k_h"] else 0) / math.comb(case["Hq"], case["k_h"]))


def work(case):
    """Bytes and operations one pass cannot do without: present tokens, kept heads, referenced groups."""
    kind, e = case["kind"], _ESIZE[case["dtype"]]
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": float(M * K * (e + 1) + 4 * M + N * K + 4 * N * (2 if case["bias"] else 1) + M * N * e), "flops": 2.0 * M * N * K}
    if kind == "append":
        new = sum(_present(case, case["T"]))
        return {"bytes": 2.0 * new * case["Hk"] * case["d"] * (e + 1) + 8.0 * -(-new // case["page"]) * case["Hk"], "flops": 0.0}
    B, Tq, d, k_h, g = case["B"], case["Tq"], case["d"], case["k_h"], _groups(case)
    rows = 2.0 * B * k_h * Tq * d * e
    if kind == "cross":
        keys = sum(_present(case, case["Tk"]))
        return {"bytes": rows + 2.0 * keys * g * d * e, "flops": 4.0 * keys * Tq * k_h * d}
    lens = _stored(case)
    pairs = sum(sum(max(0, n - Tq + i + 1) for i in range(Tq)) if case["causal"] else n * Tq for n in lens)
    return {"bytes": rows + 2.0 * sum(lens) * g * d + 8.0 * sum(-(-n // case["page"]) for n in lens) * g, "flops": 4.0 * pairs * k_h * d}


# ------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype=torch.float32, std=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std).to(dtype)


def _kept(g, B, n, k):
    return torch.rand((B, n), generator=g, device="cuda").topk(k, dim=1).indices.sort(dim=1).values.to(torch.int32).contiguous()


def _which(case, s, T):
    """Which tokens of a batch count: modality ids and masks, lengths, or neither."""
    s["ids"] = s["masks"] = s["lengths"] = None
    if case["keys"] == "lengths":
        s["lengths"] = torch.tensor(_present(case, T), dtype=torch.int32, device="cuda")
    elif case["keys"] != "all":
        parts = _modalities(case)
        s["ids"] = torch.from_numpy(np.repeat(np.arange(len(parts)), parts).astype(np.int32)).cuda()
        s["masks"] = torch.tensor([b % (1 << len(parts)) for b in range(case["B"])], dtype=torch.int32, device="cuda")


def _cache(case, g, s):
    """A pool of pages whose order says nothing, and each sample's pages; what the stored tokens hold is random."""
    B, page, Hk, d, cols = case["B"], case["page"], case["Hk"], case["d"], case["cap"] // case["page"]
    pages = B * cols + 3
    s["table"] = torch.randperm(pages, generator=g, device="cuda")[: B * cols].reshape(B, cols).to(torch.int32).contiguous()
    s["stored"] = torch.tensor(_stored(case), dtype=torch.int32, device="cuda")
    for name in ("k", "v"):
        x = _normal(g, (pages, Hk, page, d))
        if case["fmt"] == "i8":
            s[name] = (x * 40).round().clamp_(-127, 127).to(torch.int8)
            s[name + "_scales"] = torch.rand((pages, Hk), generator=g, device="cuda") * 0.02 + 0.015
        else:
            s[name] = (x * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            s[name + "_scales"] = torch.exp2(-torch.randint(5, 8, (pages, Hk), generator=g, device="cuda").float())


def prepare(case, seed):
    g, kind, dt = _generator(seed), case["kind"], _DTYPES[case["dtype"]]
    s = {"case": case}
    if kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        # activations with a few loud channels, as transformers have them
        loud = 1 + 7 * (torch.rand((K,), generator=g, device="cuda") < 0.02).float()
        s["X"] = (torch.randn((M, K), generator=g, device="cuda") * loud).to(dt)
        W = _normal(g, (N, K), std=0.03)
        s["w_scales"] = (W.abs().amax(1) / 127).contiguous()
        s["W"] = (W / s["w_scales"][:, None]).round().clamp_(-127, 127).to(torch.int8).contiguous()
        s["bias"] = _normal(g, (N,), std=0.1) if case["bias"] else None
        return s
    if kind == "cross":
        B, Tq, Tk, Hq, Hk, d = (case[k] for k in ("B", "Tq", "Tk", "Hq", "Hk", "d"))
        s["Q"] = _normal(g, (B, Hq, Tq, d), dt, 1.5)
        s["K"], s["V"] = _normal(g, (B, Hk, Tk, d), dt), _normal(g, (B, Hk, Tk, d), dt)
        s["kept"] = _kept(g, B, Hq, case["k_h"]) if case["k_h"] < Hq else None
        _which(case, s, Tk)
        return s
    _cache(case, g, s)
    if kind == "cache":
        B, Hq = case["B"], case["Hq"]
        s["Q"] = _normal(g, (B, Hq, case["Tq"], case["d"]), dt, 1.5)
        s["kept"] = _kept(g, B, Hq, case["k_h"]) if case["k_h"] < Hq else None
        return s
    B, T, Hk, d = case["B"], case["T"], case["Hk"], case["d"]
    # new values of the stored ones' range, louder for some samples, so that some pages' scales grow
    loud = torch.exp2(torch.randint(-1, 2, (B, 1, 1, 1), generator=g, device="cuda").float())
    s["K"], s["V"] = (_normal(g, (B, Hk, T, d)) * loud).to(dt), (_normal(g, (B, Hk, T, d)) * loud).to(dt)
    _which(case, s, T)
    return s


# ------------------------------------------------------------------------------------------ plain forms

def _tokens_in(s, B, T):
    """[B, T]: which tokens are present."""
    ok = torch.ones((B, T), dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        ok = ok & (torch.arange(T, device="cuda")[None] < s["lengths"][:, None])
    if s["ids"] is not None:
        ok = ok & ((s["masks"][:, None] >> s["ids"][None]) & 1).bool()
    return ok


def _attend(Q, K, V, kept, group, visible):
    """softmax(q k / sqrt d) v in 32 bits over the visible keys, zero where there is none; heads in kept order."""
    B, Hq, Tq, d = Q.shape
    if kept is None:
        kept = torch.arange(Hq, device="cuda")[None].expand(B, Hq)
    rows, kept = torch.arange(B, device="cuda")[:, None], kept.long()
    q, g = Q[rows, kept].float(), kept // group
    s = torch.matmul(q, K[rows, g].transpose(2, 3)) * d ** -0.5
    s = torch.where(visible[:, None], s, -math.inf)
    top = s.amax(3, keepdim=True) if s.shape[3] else s.new_zeros(s.shape[:3] + (1,))
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)
    return torch.where(total > 0, torch.matmul(p, V[rows, g]) / total, 0.0).to(Q.dtype)


def _pages(s, name, fmt):
    """The cache of every sample as [B, Hk, tokens, d] in 32 bits."""
    codes = s[name] if fmt == "i8" else s[name].view(torch.float8_e4m3fn)
    at = s["table"].long()
    x = codes[at].float() * s[name + "_scales"][at][..., None, None]
    B, cols, Hk, page, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, Hk, cols * page, d)


def _page_scale(top, fmt):
    """The scale under which `top` is the largest code: an eight-bit integer's 127, or a power of two and e4m3's 448."""
    if fmt == "i8":
        scale = (top / 127).clamp_min(2.0 ** -126)
    else:
        m, e = torch.frexp(top)
        scale = torch.ldexp(torch.ones_like(top), (e - torch.where(m > 0.875, 8, 9)).clamp_min(-126))
    return torch.where(top > 0, scale, 0.0)


def _codes(x, scale, fmt):
    """x / scale rounded to the nearest code; the quotient in 64 bits, since it decides between neighbours."""
    y = x.double() / torch.where(scale > 0, scale, 1.0).double()
    if fmt == "i8":
        return y.round().clamp(-127, 127).to(torch.int8)
    return y.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)   # (a power of two: the quotient is exact)


def _append(s, name, X, fmt, page, present, pos):
    """New tokens into one of the two pools. A page's scale grows to what the new tokens need, its older codes with it."""
    B, Hk, T, d = X.shape
    cols = s["table"].shape[1]
    stored, table = s["stored"].long(), s["table"].long()
    codes, scales = s[name], s[name + "_scales"]
    block = (pos // page).clamp(0, cols - 1)                                               # [B, T]
    top = torch.where(present[:, None], X.float().abs().amax(3), 0.0)                      # [B, Hk, T]
    need = torch.zeros((B, Hk, cols), device="cuda").scatter_reduce(2, block[:, None].expand(B, Hk, T), top, "amax")
    need = _page_scale(need, fmt)
    touched = torch.zeros((B, cols), dtype=torch.int32, device="cuda").scatter_reduce(1, block, present.int(), "amax").bool()
    rows, first = torch.arange(B, device="cuda"), (stored // page).clamp_max(cols - 1)
    part = (stored % page > 0) & touched[rows, first]                                      # a partly filled page gets more
    at = table[rows, first]
    old = torch.where(part[:, None], scales[at], 0.0)                                      # [B, Hk]
    new = need.clone()
    new[rows, :, first] = torch.maximum(need[rows, :, first], old)
    # older codes of the page under its new scale
    held = codes[at]
    values = (held if fmt == "i8" else held.view(torch.float8_e4m3fn)).double() * old[..., None, None].double()
    again = _codes(values, new[rows, :, first][..., None, None], fmt)
    older = (torch.arange(page, device="cuda")[None] < (stored % page)[:, None]) & part[:, None]
    codes[at] = torch.where(older[:, None, :, None], again, held)
    # the new tokens'
    b, t = present.nonzero(as_tuple=True)
    j, slot = block[b, t], pos[b, t] % page
    codes[table[b, j], :, slot] = _codes(X[b, :, t].float(), new[b, :, j][..., None], fmt)
    b, j = touched.nonzero(as_tuple=True)
    scales[table[b, j]] = new[b, :, j]


def _view(codes, fmt):
    return codes if fmt == "i8" else codes.view(torch.float8_e4m3fn)


def _pool(s, fmt):
    return {"k": _view(s["k"], fmt), "v": _view(s["v"], fmt), "k_scales": s["k_scales"], "v_scales": s["v_scales"]}


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "linear":
        if own:
            sn = _sentry()
            codes, scales = sn.quantize_rows_i8(s["X"])
            return {"Y": sn.linear_i8(codes, scales, s["W"], s["w_scales"], s["bias"], dtype=s["X"].dtype), "codes": codes, "scales": scales}
        x = s["X"].float()
        scales = x.abs().amax(1) / 127
        codes = (x.double() / torch.where(scales > 0, scales, 1.0).double()[:, None]).round().clamp(-127, 127)
        y = torch.matmul(codes.float(), s["W"].float().t()) * scales[:, None] * s["w_scales"][None]
        if s["bias"] is not None:
            y = y + s["bias"]
        return {"Y": y.to(s["X"].dtype), "codes": codes.to(torch.int8), "scales": scales}
    if kind == "cross":
        if own:
            return _sentry().cross_attend_fwd(s["Q"], s["K"], s["V"], kept_heads=s["kept"], key_modality_ids=s["ids"], masks=s["masks"],
                                              key_lengths=s["lengths"])
        B, Hk, Tk, _ = s["K"].shape
        visible = _tokens_in(s, B, Tk)[:, None]
        return _attend(s["Q"], s["K"].float(), s["V"].float(), s["kept"], case["Hq"] // Hk, visible)
    fmt = case["fmt"]
    if kind == "cache":
        if own:
            return _sentry().cache_attend_fwd(s["Q"], s["k"], s["v"], s["k_scales"], s["v_scales"], s["table"], s["stored"],
                                              kept_heads=s["kept"], causal=case["causal"])
        K, V = _pages(s, "k", fmt), _pages(s, "v", fmt)
        Tq, key = case["Tq"], torch.arange(K.shape[2], device="cuda")[None, None]
        last = s["stored"].long()[:, None, None].expand(-1, Tq, 1)
        if case["causal"]:
            last = last - Tq + 1 + torch.arange(Tq, device="cuda")[None, :, None]
        return _attend(s["Q"], K, V, s["kept"], case["Hq"] // case["Hk"], key < last)
    if own:
        lengths = _sentry().cache_append(s["K"], s["V"], s["k"], s["v"], s["k_scales"], s["v_scales"], s["table"], s["stored"],
                                         token_modality_ids=s["ids"], masks=s["masks"], token_lengths=s["lengths"])
        return {"lengths": lengths, **_pool(s, fmt)}
    B, _, T, _ = s["K"].shape
    present = _tokens_in(s, B, T)
    pos = s["stored"].long()[:, None] + present.long().cumsum(1) - 1
    _append(s, "k", s["K"], fmt, case["page"], present, pos)
    _append(s, "v", s["V"], fmt, case["page"], present, pos)
    return {"lengths": (s["stored"] + present.sum(1)).to(torch.int32), **_pool(s, fmt)}


# ------------------------------------------------------------------------------------------ 64 bits

def _exact_softmax(q, k, v, ok):
    """Rows of q on the keys that ok lets each see, in 64 bits."""
    s = torch.einsum("hqd,hkd->hqk", q, k) / math.sqrt(q.shape[-1])
    s = s.masked_fill(~ok, -math.inf)
    p = torch.softmax(s, -1)
    return torch.einsum("hqk,hkd->hqd", torch.nan_to_num(p, nan=0.0), v)


def _heads_of(s, case, b):
    return (torch.arange(case["Hq"], device="cuda") if s["kept"] is None else s["kept"][b]).long()


def _to_e4m3(x):
    """Nearest value of 3 fraction bits, exponents from -6 on, at most 448; ties to the even fraction."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), e.clamp_min(-5) - 4)
    return (torch.round(x / step) * step).clamp(-448, 448)


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "linear":
        x = s["X"].double()
        scales = (s["X"].float().abs().amax(1) / 127).double()     # (a 32-bit number: it is stored as one)
        codes = torch.round(x / scales.clamp_min(1e-300)[:, None])
        y = torch.einsum("mk,nk->mn", codes, s["W"].double())
        y = y * scales[:, None] * s["w_scales"].double()
        return {"Y": y if s["bias"] is None else y + s["bias"].double(), "codes": None, "scales": x.abs().amax(1) / 127}
    if kind in ("cross", "cache"):
        if work(case)["flops"] > 2e12:
            return None
        r, out = case["Hq"] // case["Hk"], []
        for b in range(case["B"]):
            h = _heads_of(s, case, b)
            q = s["Q"][b, h].double()
            if kind == "cross":
                ok = torch.ones(case["Tk"], dtype=torch.bool, device="cuda")
                if s["lengths"] is not None:
                    ok[int(s["lengths"][b]):] = False
                if s["ids"] is not None:
                    ok &= torch.tensor([(int(s["masks"][b]) >> int(i)) & 1 == 1 for i in s["ids"].tolist()], device="cuda")
                k, v = s["K"][b].double()[h // r], s["V"][b].double()[h // r]
                parts = [_exact_softmax(q[i:i + 1], k[i:i + 1], v[i:i + 1], ok[None, None]) for i in range(len(h))]
                out.append(torch.cat(parts))
                continue
            n, Tq = int(s["stored"][b]), case["Tq"]
            side = []
            for name in ("k", "v"):
                pages = s["table"][b].long()
                c = (s[name] if case["fmt"] == "i8" else s[name].view(torch.float8_e4m3fn))[pages].double()
                c = c * s[name + "_scales"][pages].double()[..., None, None]
                side.append(c.transpose(0, 1).flatten(1, 2)[:, :n][h // r])
            ok = torch.ones((Tq, n), dtype=torch.bool, device="cuda")
            if case["causal"]:
                ok = torch.arange(n, device="cuda")[None] <= torch.arange(Tq, device="cuda")[:, None] + n - Tq
            out.append(_exact_softmax(q, side[0], side[1], ok[None]))
        return torch.stack(out)
    if case["fmt"] == "i8":   # whole numbers and the scales that go with them: equal or not
        return None
    page, B, T = case["page"], case["B"], case["T"]
    where = _tokens_in(s, B, T).cpu().numpy()
    res = {"lengths": None}
    for name, X in (("k", s["K"]), ("v", s["V"])):
        c, sc = s[name].view(torch.float8_e4m3fn).double(), s[name + "_scales"].double()
        for b in range(B):
            t = torch.from_numpy(np.flatnonzero(where[b])).cuda()
            at, n = int(s["stored"][b]), len(t)
            x = X[b][:, t].double()
            done = 0
            while done < n:   # page by page
                j, slot = divmod(at + done, page)
                m, p = min(page - slot, n - done), int(s["table"][b, j])
                part = x[:, done:done + m]
                need = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 2)).clamp_min(1e-300) / 448)))
                if slot:
                    need = torch.maximum(need, sc[p])
                    c[p, :, :slot] = _to_e4m3(c[p, :, :slot] * (sc[p] / need)[:, None, None])
                c[p, :, slot:slot + m] = _to_e4m3(part / need[:, None, None])
                sc[p] = need
                done += m
        res[name], res[name + "_scales"] = c, sc
    return res
