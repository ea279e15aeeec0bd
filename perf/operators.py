"""The timed cases of the cache operators: decoding from a paged cache whose
keys and values are held in 8 bits with one scale per page and head.

kinds: append  elsaa_cache_append: rows of new tokens into the cache
       attend  elsaa_cache_attention: the newest tokens against the cache,
               with the weight that every cached token received where
               `weights` is set
       sparse  elsaa_cache_select, then elsaa_cache_attention over the pages
               it chose
       evict   elsaa_cache_evict: the tokens of least accumulated weight go

Sizes are those of the repository's workloads (12 heads of 64 at N = 4096 and
8192, 16 heads of 128 at 16384, 32 at 65536) and generic ones of grouped heads.
`run` computes the operators in their plain form, in elementary torch
operations, unless `own` is set: then it makes a user's calls.

The cache: codes are e4m3 numbers [page, head, row, d], value = code * scale,
scales powers of two; `bounds` holds each page's channel-wise extremes of its
key codes over 4, rounded outwards to int8 [page, head, (high, low), d].
"""
from __future__ import annotations

import math

import torch

own = False

_DEFAULTS = dict(kind="attend", dtype="bf16", B=1, Hkv=1, G=1, d=128, ps=64,
                 len=1024, T=1, ragged=False, weights=False, n_sel=0, keep=0,
                 recent=0)


def _case(**kw):
    return dict(_DEFAULTS, **kw)


def listed():
    return [
        # a prompt of the headline prefill goes into the cache
        _case(name="append_prompt_16k", kind="append", B=2, Hkv=16, ps=128,
              len=0, T=16384),
        # one decoding step of a busy server: 64 sequences, a token each,
        # somewhere inside their open pages
        _case(name="append_step", kind="append", B=64, Hkv=8, len=2000, T=1,
              ragged=True),
        # the smallest call: one sequence of a 12-head model; latency
        _case(name="attend_short", B=1, Hkv=12, d=64, len=700, T=1),
        # a small fp32 model, ragged batch
        _case(name="attend_fp32", dtype="fp32", B=4, Hkv=12, d=64, len=4096,
              ragged=True),
        # ungrouped heads at the headline length
        _case(name="attend_16k", B=2, Hkv=16, ps=128, len=16384),
        # a serving batch of grouped heads with the weights that eviction
        # wants; lengths from none to 8192
        _case(name="attend_batch_weights", B=32, Hkv=8, G=4, ps=32, len=8192,
              ragged=True, weights=True),
        # several drafted tokens a sequence are verified in one call; odd
        # lengths, fewer drafts in some sequences
        _case(name="attend_verify", B=8, Hkv=8, G=4, len=4099, T=5,
              ragged=True),
        # long contexts: N = 64K; the largest call
        _case(name="attend_64k", B=16, Hkv=8, G=4, len=65536),
        # sparse decoding: 32 of 1024 pages for every sequence and head
        _case(name="sparse_64k", kind="sparse", B=8, Hkv=8, G=4, len=65536,
              n_sel=32),
        # sparse decoding of a 12-head model, few pages: latency
        _case(name="sparse_4k", kind="sparse", B=4, Hkv=12, d=64, ps=32,
              len=4096, n_sel=24, ragged=True),
        # a long prompt is cut to a quarter
        _case(name="evict_16k", kind="evict", B=2, Hkv=16, ps=128, len=16384,
              keep=4096, recent=128),
        # a ragged batch is cut to 2000 tokens each
        _case(name="evict_batch", kind="evict", B=16, Hkv=8, d=64, ps=32,
              len=8192, keep=2000, recent=64, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: kinds, types, head sizes and page sizes as
    in the listed ones; batch, heads and lengths spread over their
    logarithms, any length."""
    kind = rng.choice(["append", "attend", "attend", "attend", "sparse",
                       "evict"])
    d, ps = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    kw = dict(kind=kind, d=d, ps=ps, ragged=rng.random() < 0.5)
    kw["Hkv"] = rng.choice([1, 2, 4, 8, 12, 16, 32])
    if kind in ("attend", "sparse"):
        kw["G"] = rng.choice([1, 1, 2, 4, 5, 8, 16])
        kw["T"] = rng.choice([1, 1, 1, 2, 3, 4])
    # token-heads x d of one call, below the largest of its kind
    cap = dict(append=2 * 16 * 16384 * 128, attend=16 * 8 * 65536 * 128,
               sparse=8 * 8 * 65536 * 128, evict=2 * 16 * 16384 * 128)[kind]
    if kind == "attend" and rng.random() < 0.2:
        kw.update(dtype="fp32")
        cap = 4 * 12 * 8192 * 64
    elif kind == "attend":
        kw["weights"] = rng.random() < 0.3
        cap //= 4 if kw["weights"] else 1
    top = 65536 if kind in ("attend", "sparse") else 16384
    kw["B"] = max(1, min(_log_int(rng, 1, 64), cap // (kw["Hkv"] * d * 256)))
    n = _log_int(rng, 64, max(64, min(top, cap // (kw["B"] * kw["Hkv"] * d))))
    if kind == "append":
        if rng.random() < 0.5:
            kw.update(len=n, T=rng.choice([1, 1, 2, 5]))
        else:
            kw.update(len=rng.choice([0, 0, 37]), T=n)
    elif kind == "sparse":
        n = max(n, 4 * ps)
        pages = -(-n // ps)
        kw.update(len=n, n_sel=rng.randrange(3, max(4, pages // 4) + 1))
    elif kind == "evict":
        keep = max(32, int(n * rng.uniform(0.1, 0.6)))
        kw.update(len=n, keep=keep, recent=rng.randrange(0, keep // 4 + 1))
    else:
        kw.update(len=n)
    return _case(**kw)


def _lengths(case):
    """(tokens held with the new ones, new ones) of every sequence. Ragged:
    the first sequence is the longest, one holds nothing, one a single
    token."""
    held, new = [], []
    for b in range(case["B"]):
        f = (b * 0.6180339887) % 1.0 if b and case["ragged"] else 1.0
        n = case["T"]
        if case["ragged"] and case["T"] > 1:
            n = max(1, round(case["T"] * ((b * 0.7548776662) % 1.0 or 1.0)))
        old = int(case["len"] * f)
        if case["kind"] != "append":
            old = max(0, old - n)
        if case["ragged"] and b in (3, 4) and case["kind"] != "append":
            old, n = 0, b - 3
        held.append(old + n)
        new.append(n)
    return held, new


def _exponent(amax, top, low, high):
    """Least e in [low, high] with amax <= top 2^e."""
    m, x = torch.frexp(amax)  # amax = m 2^x, m in [0.5, 1)
    tm, tx = math.frexp(top)
    e = x - tx + (m > tm).to(x.dtype)
    e = torch.where(amax > 0, e, torch.full_like(e, low))
    return e.clamp(low, high)


def _e4m3(x):
    return x.to(torch.float8_e4m3fn)


def _pow2(e):
    return torch.exp2(e.float())


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    rnd = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    B, Hkv, G, d, ps, T = (case[x] for x in ("B", "Hkv", "G", "d", "ps", "T"))
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    held, new = _lengths(case)
    P = -(-max(max(held), 1) // ps) + 1  # a spare entry behind the longest
    used = [-(-n // ps) for n in held]
    kept = [-(-min(n, case["keep"]) // ps) for n in held]
    num = sum(used) + (sum(kept) if case["kind"] == "evict" else 0) + 3
    place = torch.randperm(num, generator=g, device=dev).to(torch.int32)
    at = 0

    def table(counts, width):
        nonlocal at
        t = torch.full((B, width), -1, dtype=torch.int32, device=dev)
        for b, n in enumerate(counts):
            t[b, :n] = place[at:at + n]
            at += n
        return t

    s = dict(case=case, held=held, new=new, P=P, dt=dt)
    s["table"] = table(used, P)
    s["lengths"] = torch.tensor(held, dtype=torch.int32, device=dev)
    s["new_len"] = torch.tensor(new, dtype=torch.int32, device=dev)
    # keys with channels of different size and offset, as projected ones have
    size, off = torch.exp(0.5 * rnd(Hkv, 1, d)), 0.7 * rnd(Hkv, 1, d)
    for x in "kv":
        pool = torch.empty((num, Hkv, ps, d), dtype=torch.float8_e4m3fn,
                           device=dev)
        scale = torch.empty((num, Hkv), device=dev)
        step = max(1, (1 << 28) // (Hkv * ps * d))
        for i in range(0, num, step):
            val = rnd(min(step, num - i), Hkv, ps, d)
            if x == "k":
                val = val * size + off
            e = _exponent(val.abs().amax((2, 3)), 448.0, -64, 120)
            pool[i:i + step] = _e4m3(val * _pow2(-e)[..., None, None])
            scale[i:i + step] = _pow2(e)
        s[x], s[x + "_scale"] = pool, scale
    s["bounds"] = torch.empty((num, Hkv, 2, d), dtype=torch.int8, device=dev)
    step = max(1, (1 << 28) // (Hkv * ps * d))
    for i in range(0, num, step):
        val = s["k"][i:i + step].float()
        s["bounds"][i:i + step, :, 0] = torch.ceil(val.amax(2) / 4).to(torch.int8)
        s["bounds"][i:i + step, :, 1] = torch.floor(val.amin(2) / 4).to(torch.int8)
    if case["kind"] == "append":
        s["k_new"] = (rnd(B, Hkv, T, d) * size + off).to(dt)
        s["v_new"] = rnd(B, Hkv, T, d).to(dt)
    elif case["kind"] == "evict":
        # what attention leaves behind: a few heavy tokens, many light ones,
        # and untouched ones that tie
        w = torch.exp(2.0 * rnd(B, Hkv, P * ps) - 4.0)
        s["weight"] = torch.where(rnd(B, Hkv, P * ps) < -1.2,
                                  torch.zeros_like(w), w)
        s["dst"] = table(kept, -(-case["keep"] // ps))
        s["weight_out"] = torch.zeros(B, Hkv, -(-case["keep"] // ps) * ps,
                                      device=dev)
        s["lengths_out"] = torch.zeros(B, dtype=torch.int32, device=dev)
        s["kept"] = torch.full((B, Hkv, case["keep"]), -1, dtype=torch.int32,
                               device=dev)
    else:
        # scores of standard deviation around 2
        q = rnd(B, Hkv * G, T, d) * (2.0 / 1.6)
        s["q"] = q.to(dt)
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, Hkv * G, T), device=dev)
        if case["weights"]:
            s["weight_in"] = torch.exp(2.0 * rnd(B, Hkv, P * ps) - 4.0)
            s["weight_out"] = s["weight_in"].clone()
        if case["kind"] == "sparse":
            s["pages"] = torch.full((B, Hkv, case["n_sel"]), -1,
                                    dtype=torch.int32, device=dev)
    if own:
        from paper_2607_20214_gb300 import elsaa as E
        s["E"] = E
        s["cache"] = E.make_cache(
            s["k"], s["v"], s["k_scale"], s["v_scale"], s["bounds"],
            s["table"], s["lengths"], H=Hkv * G, dtype=case["dtype"])
        s["ws"] = None if case["kind"] == "append" else \
            E.new_cache_workspace(s["cache"], T=T, weights=case["weights"],
                                  keep=case["keep"])
    return s


# ------------------------------------------------------------ plain forms

def _append(s):
    c, ps = s["case"], s["case"]["ps"]
    T, dev = c["T"], s["k"].device
    n, end = s["new_len"].long(), s["lengths"].long()
    start = end - n
    first = start // ps                              # first page written
    W = -(-T // ps) + 1                              # pages of the window
    page = first[:, None] + torch.arange(W, device=dev)
    live = (page * ps < end[:, None]) & (n[:, None] > 0)
    ids = s["table"].gather(1, page.clamp(max=s["P"] - 1)).long().clamp(min=0)
    pos = first[:, None] * ps + torch.arange(W * ps, device=dev)
    t = pos - start[:, None]
    old = (t < 0).view(-1, W, 1, ps, 1)
    fresh = ((t >= 0) & (t < n[:, None])).view(-1, W, 1, ps, 1)
    had = old.any(3)[..., 0]                         # [B, W, 1]
    zero = torch.zeros((), device=dev)
    for x in "kv":
        rows = s[x + "_new"].float().gather(
            2, t.clamp(0, T - 1)[:, None, :, None].expand(
                -1, c["Hkv"], -1, c["d"]))
        rows = rows.view(c["B"], c["Hkv"], W, ps, c["d"]).transpose(1, 2)
        codes, scale = s[x][ids].float(), s[x + "_scale"][ids]
        e_old = torch.log2(scale).round().int()
        e = _exponent(torch.where(fresh, rows.abs(), zero).amax((3, 4)),
                      448.0, -64, 120)
        e = torch.where(had, torch.maximum(e, e_old), e)
        drop = _pow2(e_old - e)
        put = torch.where(fresh, rows * _pow2(-e)[..., None, None],
                          torch.where(old, codes * drop[..., None, None],
                                      codes))
        put = _e4m3(put)
        s[x][ids[live]] = put[live]
        s[x + "_scale"][ids[live]] = _pow2(e)[live]
        if x == "k":
            b = s["bounds"][ids].float() * drop[..., None, None]
            low = torch.full_like(b[..., 0, :], -1e9)
            put = put.float()
            hi = torch.maximum(
                torch.where(had[..., None], b[..., 0, :], low).ceil(),
                torch.where(fresh, put, -1e9 + zero).amax(3).div(4).ceil())
            lo = torch.minimum(
                torch.where(had[..., None], b[..., 1, :], -low).floor(),
                torch.where(fresh, put, 1e9 + zero).amin(3).div(4).floor())
            s["bounds"][ids[live]] = torch.stack([hi, lo], 3)[live].to(
                torch.int8)
    return {x: s[x] for x in ("k", "v", "k_scale", "v_scale", "bounds")}


def _attend(s, pages=None):
    """pages None: every page of the table, one list for all heads."""
    c, ps, dev = s["case"], s["case"]["ps"], s["k"].device
    B, Hkv, G, T, d = (c[x] for x in ("B", "Hkv", "G", "T", "d"))
    n, end = s["new_len"].long(), s["lengths"].long()
    if pages is None:
        P = s["P"] - 1
        ids = s["table"][:, :P].long().clamp(min=0)
        k = s["k"][ids].float() * s["k_scale"][ids][..., None, None]
        v = s["v"][ids].float() * s["v_scale"][ids][..., None, None]
        k, v = k.transpose(1, 2), v.transpose(1, 2)  # [B, Hkv, P, ps, d]
        pos = torch.arange(P * ps, device=dev).view(1, 1, P * ps)
    else:
        P = pages.shape[2]
        lp = pages.long().clamp(min=0)
        ids = s["table"].long()[:, None].expand(-1, Hkv, -1).gather(2, lp)
        ids = ids.clamp(min=0)
        h = torch.arange(Hkv, device=dev)[None, :, None]
        k = s["k"].view(torch.uint8)[ids, h].view(torch.float8_e4m3fn).float()
        v = s["v"].view(torch.uint8)[ids, h].view(torch.float8_e4m3fn).float()
        k = k * s["k_scale"][ids, h][..., None, None]
        v = v * s["v_scale"][ids, h][..., None, None]
        pos = (lp[..., None] * ps + torch.arange(ps, device=dev)).flatten(2)
        pos = pos + (pages < 0).repeat_interleave(ps, 2) * (1 << 40)
    q = s["q"].float().view(B, Hkv, G * T, d)
    z = torch.matmul(q, k.reshape(B, Hkv, P * ps, d).transpose(2, 3))
    z = z.view(B, Hkv, G, T, P * ps) * (1.0 / math.sqrt(d))
    t = torch.arange(T, device=dev)
    last = (end - n)[:, None] + t                    # [B, T]
    sees = pos[:, :, None] <= last[:, None, :, None]
    z = z.masked_fill(~sees[:, :, None], -math.inf)
    top = z.amax(4, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(z - top)
    den = p.sum(4, keepdim=True)
    lse = torch.where(den > 0, top + torch.log(den), -math.inf)[..., 0]
    p = p / torch.where(den > 0, den, torch.ones_like(den))
    o = torch.matmul(p.view(B, Hkv, G * T, P * ps),
                     v.reshape(B, Hkv, P * ps, d))
    valid = (t < n[:, None])[:, None]                # [B, 1, T]
    o = torch.where(valid[..., None], o.view(B, Hkv * G, T, d).to(s["dt"]),
                    s["o"])
    lse = torch.where(valid, lse.view(B, Hkv * G, T), s["lse"])
    out = dict(o=o, lse=lse)
    if c["weights"]:
        m = (p * valid[:, :, None, :, None]).sum((2, 3))
        w = s["weight_in"].clone()
        held = torch.arange(P * ps, device=dev) < end[:, None, None]
        w[..., :P * ps] += torch.where(held, m, torch.zeros_like(m))
        out["weight"] = w
    return out


def _select(s, first=1, last=1):
    c, ps, dev = s["case"], s["case"]["ps"], s["k"].device
    B, Hkv, G, T, d = (c[x] for x in ("B", "Hkv", "G", "T", "d"))
    n, end = s["new_len"].long(), s["lengths"].long()
    P = s["P"] - 1
    q = s["q"].float()
    e = _exponent(q.abs().amax(3), 127.0, -60, 120)
    qi = torch.round(q * _pow2(-e)[..., None]).view(B, Hkv, G * T, d)
    ids = s["table"][:, :P].long().clamp(min=0)
    bound = s["bounds"][ids].float().transpose(1, 2)  # [B, Hkv, P, 2, d]
    # sum_i max(q_i hi_i, q_i lo_i): whole numbers below 2^24, exact
    u = torch.matmul(qi.clamp(min=0), bound[..., 0, :].transpose(2, 3)) + \
        torch.matmul(qi.clamp(max=0), bound[..., 1, :].transpose(2, 3))
    u = u.view(B, Hkv, G, T, P) * _pow2(e).view(B, Hkv, G, T, 1)
    u = u * (4.0 * s["k_scale"][ids]).transpose(1, 2)[:, :, None, None]
    valid = torch.arange(T, device=dev) < n[:, None]
    u = u.masked_fill(~valid[:, None, None, :, None], -math.inf).amax((2, 3))
    page, held = torch.arange(P, device=dev), -(-end // ps)[:, None]
    must = (page < first) | (page >= held - last)
    u = u.masked_fill(must[:, None], math.inf)
    u = u.masked_fill((page >= held)[:, None], -math.inf)
    order = torch.sort(u, dim=2, descending=True, stable=True).indices
    order = order[..., :c["n_sel"]]
    pad = c["n_sel"] - order.shape[2]
    order = torch.nn.functional.pad(order, (0, pad), value=P)
    drop = (order >= held[:, None]) | (n == 0)[:, None, None]
    order = torch.where(drop, P, order).sort(2).values
    return torch.where(order >= P, -1, order).to(torch.int32)


def _evict(s):
    c, ps, dev = s["case"], s["case"]["ps"], s["k"].device
    B, Hkv, d, keep = c["B"], c["Hkv"], c["d"], c["keep"]
    end = s["lengths"].long()[:, None, None]
    L = s["weight"].shape[2]
    pos = torch.arange(L, device=dev)
    w = s["weight"].masked_fill(pos >= end - c["recent"], math.inf)
    w = w.masked_fill(pos >= end, -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True).indices
    order = order[..., :keep]
    order = torch.nn.functional.pad(order, (0, keep - order.shape[2]), value=L)
    rows = torch.where(order < end, order, L).sort(2).values
    none = rows >= L
    PK = s["dst"].shape[1]
    at = torch.nn.functional.pad(rows, (0, PK * ps - keep), value=L)
    live = (at < L).view(B, Hkv, PK, ps, 1).transpose(1, 2)
    at = at.clamp(max=L - 1)
    ids = s["table"].long()[:, None].expand(-1, Hkv, -1).gather(2, at // ps)
    ids, h = ids.clamp(min=0), torch.arange(Hkv, device=dev)[None, :, None]
    pages = torch.arange(PK, device=dev) * ps < end.view(B, 1).clamp(max=keep)
    dst = s["dst"].long()[pages]
    zero = torch.zeros((), device=dev)
    for x in "kv":
        val = s[x].view(torch.uint8)[ids, h, at % ps].view(
            torch.float8_e4m3fn).float() * s[x + "_scale"][ids, h][..., None]
        val = val.view(B, Hkv, PK, ps, d).transpose(1, 2)
        e = _exponent(torch.where(live, val.abs(), zero).amax((3, 4)), 448.0,
                      -64, 120)
        code = _e4m3(val * _pow2(-e)[..., None, None])
        was = s[x].view(torch.uint8)[s["dst"].long().clamp(min=0)]
        put = torch.where(live, code.view(torch.uint8), was)
        s[x].view(torch.uint8)[dst] = put[pages]
        s[x + "_scale"][dst] = _pow2(e)[pages]
        if x == "k":
            code = code.float()
            hi = torch.where(live, code, -1e9 + zero).amax(3).div(4).ceil()
            lo = torch.where(live, code, 1e9 + zero).amin(3).div(4).floor()
            s["bounds"][dst] = torch.stack([hi, lo], 3)[pages].to(torch.int8)
    got = s["weight"].gather(2, at)
    s["weight_out"].copy_(torch.where(live.transpose(1, 2).reshape(
        B, Hkv, PK * ps), got, s["weight_out"]))
    s["lengths_out"].copy_(s["lengths"].clamp(max=keep))
    s["kept"].copy_(torch.where(none, -1, rows))
    return _evicted(s)


def _evicted(s):
    return {x: s[x] for x in ("k", "v", "k_scale", "v_scale", "bounds",
                              "weight_out", "lengths_out", "kept")}


def run(s):
    c = s["case"]
    if own:
        E, cache, ws = s["E"], s["cache"], s["ws"]
        if c["kind"] == "append":
            E.elsaa_cache_append(cache, s["k_new"], s["v_new"],
                                 new_len=s["new_len"])
            return {x: s[x] for x in ("k", "v", "k_scale", "v_scale",
                                      "bounds")}
        if c["kind"] == "evict":
            E.elsaa_cache_evict(cache, s["weight"], c["keep"], c["recent"],
                                s["dst"], lengths_out=s["lengths_out"],
                                weight_out=s["weight_out"], kept=s["kept"],
                                workspace=ws)
            return _evicted(s)
        pages = None
        if c["kind"] == "sparse":
            pages = E.elsaa_cache_select(cache, s["q"], c["n_sel"], first=1,
                                         last=1, new_len=s["new_len"],
                                         pages=s["pages"], workspace=ws)
        E.elsaa_cache_attention(cache, s["q"], pages=pages,
                                new_len=s["new_len"],
                                weight_in=s.get("weight_in"),
                                weight_out=s.get("weight_out"), o=s["o"],
                                lse=s["lse"], workspace=ws)
        out = dict(o=s["o"], lse=s["lse"])
        if c["weights"]:
            out["weight"] = s["weight_out"]
        if pages is not None:
            out["pages"] = pages
        return out
    if c["kind"] == "append":
        return _append(s)
    if c["kind"] == "evict":
        return _evict(s)
    if c["kind"] == "sparse":
        pages = _select(s)
        return dict(_attend(s, pages), pages=pages)
    return _attend(s)


# -------------------------------------------- the definition, in 64 bits

def _least(amax, top, low, high):
    """Least e in [low, high] with amax <= top 2^e, for one number."""
    if not amax > 0:
        return low
    e = math.ceil(math.log2(amax / top)) - 1
    while amax > top * 2.0 ** e:
        e += 1
    return min(max(e, low), high)


def _round8(x):
    """float64 to the nearest e4m3 value (ties to even), as float64."""
    _, e = torch.frexp(x)
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    B, Hkv, G, d, ps, T = (case[x] for x in ("B", "Hkv", "G", "d", "ps", "T"))
    held, new, table = s["held"], s["new"], s["table"].tolist()
    if case["kind"] == "append":
        if sum(-(-x // ps) + 1 for x in new) * Hkv > 20000:
            return None
        out = {x: s[x].double() for x in ("k", "v", "k_scale", "v_scale")}
        for b in range(B):
            start = held[b] - new[b]
            for page in range(start // ps, -(-held[b] // ps)):
                i = table[b][page]
                r0 = max(0, start - page * ps)
                r1 = min(ps, held[b] - page * ps)
                t0 = page * ps + r0 - start
                for x in "kv":
                    rows = s[x + "_new"][b, :, t0:t0 + r1 - r0].double()
                    amax = rows.abs().amax((1, 2)).tolist()
                    was = s[x + "_scale"][i].tolist()
                    for h in range(Hkv):
                        e = _least(amax[h], 448.0, -64, 120)
                        if r0:
                            e = max(e, round(math.log2(was[h])))
                            out[x][i, h, :r0] = _round8(
                                out[x][i, h, :r0] * (was[h] / 2.0 ** e))
                        out[x][i, h, r0:r1] = _round8(rows[h] / 2.0 ** e)
                        out[x + "_scale"][i, h] = 2.0 ** e
        return dict(out, bounds=None)
    if case["kind"] == "evict":
        k = {x: s[x].double() for x in ("k", "v", "k_scale", "v_scale")}
        wout = s["weight_out"].double()
        w = s["weight"].double().cpu()
        dst = s["dst"].tolist()
        if B * Hkv * (case["keep"] // ps + 1) > 20000:
            return None
        src = {x: s[x].double() * s[x + "_scale"].double()[..., None, None]
               for x in "kv"}
        for b in range(B):
            n, m = held[b], min(held[b], case["keep"])
            ids = torch.tensor(table[b], device=s["k"].device)
            for h in range(Hkv):
                v = w[b, h, :n].tolist()
                safe = max(0, n - case["recent"])
                best = sorted(range(safe), key=lambda j: (-v[j], j))
                best = sorted(best[:max(0, m - (n - safe))] +
                              list(range(safe, n)))[-m:] if m else []
                at = torch.tensor(best, device=s["k"].device,
                                  dtype=torch.long)
                wout[b, h, :m] = s["weight"][b, h, at].double()
                for x in "kv":
                    rows = src[x][ids[at // ps], h, at % ps]
                    for p in range(-(-m // ps)):
                        r = rows[p * ps:(p + 1) * ps]
                        e = _least(float(r.abs().max()), 448.0, -64, 120)
                        k[x][dst[b][p], h, :len(r)] = _round8(r / 2.0 ** e)
                        k[x + "_scale"][dst[b][p], h] = 2.0 ** e
        return dict(k, bounds=None, weight_out=wout, lengths_out=None,
                    kept=None)
    if B * Hkv > 4096:
        return None
    pages = None
    if case["kind"] == "sparse":
        pages = _select_exact(s).tolist()
    o = s["o"].double()
    lse = s["lse"].double()
    wt = s["weight_in"].double() if case["weights"] else None
    for b in range(B):
        if not new[b]:
            continue
        for h in range(Hkv):
            lp = list(range(-(-held[b] // ps))) if pages is None else [
                p for p in pages[b][h] if p >= 0]
            ids = torch.tensor([table[b][p] for p in lp],
                               device=s["k"].device)
            k, v = (s[x].view(torch.uint8)[ids, h].view(
                torch.float8_e4m3fn).double().flatten(0, 1) *
                s[x + "_scale"][ids, h].double().repeat_interleave(ps)[:, None]
                for x in "kv")
            pos = torch.tensor(lp, device=ids.device)[:, None] * ps + \
                torch.arange(ps, device=ids.device)
            pos = pos.flatten()
            q = s["q"][b, h * G:(h + 1) * G, :new[b]].double()
            z = (q.reshape(-1, d) @ k.T).view(G, new[b], -1) / math.sqrt(d)
            at = held[b] - new[b] + torch.arange(new[b], device=ids.device)
            z = z.masked_fill(pos > at[:, None], -math.inf)
            L = torch.logsumexp(z, 2)
            p = torch.exp(z - L[..., None])
            o[b, h * G:(h + 1) * G, :new[b]] = p @ v
            lse[b, h * G:(h + 1) * G, :new[b]] = L
            if wt is not None:
                wt[b, h, :held[b]] += p.sum((0, 1))[:held[b]]
    out = dict(o=o, lse=lse)
    if wt is not None:
        out["weight"] = wt
    if pages is not None:
        out["pages"] = None
    return out


def _select_exact(s):
    """The pages of select(), one sequence and head at a time."""
    case = s["case"]
    ps, G, keep = case["ps"], case["G"], case["n_sel"]
    got = torch.full((case["B"], case["Hkv"], keep), -1)
    for b, (n, m) in enumerate(zip(s["held"], s["new"])):
        held = -(-n // ps)
        if not m:
            continue
        ids = s["table"][b, :held].long()
        q = s["q"][b, :, :m].double()
        for h in range(case["Hkv"]):
            best = torch.full((held,), -math.inf, dtype=torch.float64,
                              device=q.device)
            box = s["bounds"][ids, h].double()
            scale = 4.0 * s["k_scale"][ids, h].double()
            for x in q[h * G:(h + 1) * G].flatten(0, 1):
                e = _least(float(x.abs().max()), 127.0, -60, 120)
                x = torch.round(x / 2.0 ** e)
                u = torch.maximum(x * box[:, 0], x * box[:, 1]).sum(1)
                best = torch.maximum(best, u * 2.0 ** e * scale)
            best[:1], best[max(0, held - 1):] = math.inf, math.inf
            v = best.tolist()
            order = sorted(range(held), key=lambda p: (-v[p], p))[:keep]
            got[b, h, :len(order)] = torch.tensor(sorted(order))
    return got


def work(case):
    """Bytes and operations of one pass: every cached byte that the result
    depends on once, every input once, every output once."""
    B, Hkv, G, d, ps, T = (case[x] for x in ("B", "Hkv", "G", "d", "ps", "T"))
    el = 4 if case["dtype"] == "fp32" else 2
    held, new = _lengths(case)
    pages = [-(-n // ps) for n in held]
    if case["kind"] == "append":
        rows = sum(new) * Hkv
        return dict(bytes=rows * 2 * d * (el + 1), flops=rows * 2 * d * 4)
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in held) * Hkv
        return dict(bytes=sum(held) * Hkv * 4 + kept * (4 * d + 8),
                    flops=kept * 2 * d * 2)
    seen = held
    b = sum(new) * Hkv * G * (2 * d * el + 4)
    f = 0
    if case["kind"] == "sparse":
        b += sum(pages) * Hkv * (2 * d + 4) + B * Hkv * case["n_sel"] * 4
        f += sum(p * m for p, m in zip(pages, new)) * Hkv * G * 2 * d
        seen = [min(n, case["n_sel"] * ps) for n in held]
    b += sum(seen) * Hkv * 2 * d + sum(min(p, case["n_sel"] or p)
                                       for p in pages) * Hkv * 8
    if case["weights"]:
        b += sum(seen) * Hkv * 8
    f += sum(n * m for n, m in zip(seen, new)) * Hkv * G * 4 * d
    return dict(bytes=b, flops=f)
