"""The timed cases of the operators around the attention core: from the
projection's rows to heads (norm and position rotation in one pass, one or
several position axes), exact attention, and the backward pass of both.

kinds: heads       elsaa_heads_forward: rows [B, N, heads, d] as the Q/K/V
                   projection writes them, to normed and rotated heads
                   [B, heads, N, d]
       heads_grad  elsaa_heads_backward: gradients of the heads, to those of
                   the rows and of the norm's weights
       exact       elsaa_exact_forward: softmax attention over all keys
       exact_grad  elsaa_exact_backward: dQ, dK, dV from the saved O and lse

Sizes are those of the repository's workloads (16 heads of 128 at N = 16384, 12
of 64 at 4096 and 8192) and generic ones: grouped heads, odd lengths, padded
batches. `run` computes the operators in their plain form, in elementary torch
operations, unless `own` is set: then it makes a user's calls.

What lies behind a sequence's last row holds NaN in the inputs and is left as
it was (zeros here) in the outputs.
"""
from __future__ import annotations

import math

import torch

own = False

_DEFAULTS = dict(kind="heads", dtype="bf16", B=1, Hkv=1, G=1, d=128, N=1024,
                 Nk=0, ragged=False,
                 # heads: norm with weights, rotated channels, their pairing
                 # (neighbours or halves), axes (in turn or in blocks), K and
                 # V copied to every query head, type of the gradients
                 norm=True, rot=128, neighbours=False, axes=1, turn=False,
                 expand=False, grad="fp32", cached=0,
                 # exact
                 causal=True)


def _case(**kw):
    return dict(_DEFAULTS, **kw)


def listed():
    return [
        # a decoding step of a busy server: a token of 64 sequences, each at
        # its own position; latency
        _case(name="heads_step", B=64, Hkv=8, G=4, N=1, cached=2000,
              ragged=True),
        # the headline prompt, 2 x 16 heads of 128 at 16384 tokens
        _case(name="heads_prompt_16k", B=2, Hkv=16, N=16384),
        # image and video tokens: three axes in turn, a padded batch of odd
        # length, grouped heads copied for an operator without groups
        _case(name="heads_axes", B=4, Hkv=4, G=3, d=64, N=4099, rot=64,
              axes=3, turn=True, expand=True, ragged=True),
        # a small fp32 model without norm, half of the channels rotated
        _case(name="heads_fp32", dtype="fp32", Hkv=2, G=2, d=32, N=333,
              norm=False, rot=16, neighbours=True),
        # the training step's backward pass, from elsaa_backward's fp32
        # gradients; 8 x 12 heads of 64 at 8192 tokens
        _case(name="heads_grad_8k", kind="heads_grad", B=8, Hkv=12, d=64,
              N=8192, rot=64),
        # 16-bit gradients of copied heads, two axes in blocks, a padded batch
        _case(name="heads_grad_axes", kind="heads_grad", B=2, Hkv=4, G=4,
              N=2047, rot=64, axes=2, expand=True, grad="bf16", ragged=True),
        # the smallest call: an encoder's short text; latency
        _case(name="exact_short", kind="exact", Hkv=12, d=64, N=200,
              causal=False),
        # one long prompt of grouped heads; the largest call
        _case(name="exact_16k", kind="exact", Hkv=4, G=4, N=16384),
        # a chunk of a prompt against what was read before, padded batch
        _case(name="exact_chunk", kind="exact", B=8, Hkv=4, G=4, N=500,
              Nk=4096, ragged=True),
        # a small fp32 model, forward of a training step
        _case(name="exact_fp32", kind="exact", dtype="fp32", B=2, Hkv=4, d=64,
              N=1000),
        # a training step's exact layer: 4 x 12 heads of 64 at 4096
        _case(name="exact_grad_4k", kind="exact_grad", B=4, Hkv=12, d=64,
              N=4096),
        # the same of grouped heads of 128, a padded batch of odd length
        _case(name="exact_grad_groups", kind="exact_grad", B=2, Hkv=4, G=4,
              N=4099, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: kinds, types, head sizes and options as in
    the listed ones; batch, heads and lengths spread over their logarithms,
    any length."""
    kind = rng.choice(["heads", "heads", "heads_grad", "exact", "exact",
                       "exact_grad"])
    kw = dict(kind=kind, d=rng.choice([64, 64, 128, 128, 32]),
              Hkv=rng.choice([1, 2, 4, 8, 12, 16]),
              G=rng.choice([1, 1, 2, 3, 4, 8]), ragged=rng.random() < 0.4)
    if rng.random() < 0.2:
        kw["dtype"] = "fp32"
    d, H = kw["d"], kw["Hkv"] * kw["G"]
    B = _log_int(rng, 1, 64)
    if kind in ("heads", "heads_grad"):
        kw.update(norm=rng.random() < 0.7, neighbours=rng.random() < 0.3,
                  rot=rng.choice([d, d, d // 2]), axes=rng.choice([1, 1, 2, 3]),
                  turn=rng.random() < 0.5, expand=rng.random() < 0.3,
                  grad=rng.choice(["fp32", "bf16"]))
        if kw.get("dtype") == "fp32":
            kw["grad"] = "fp32"
        # channels of one call: those of heads_prompt_16k, half of them for
        # the gradients or in fp32
        cap = 2 * 16 * 3 * 16384 * 128
        cap //= 2 if kind == "heads_grad" or kw.get("dtype") == "fp32" else 1
        row = (H + 2 * (H if kw["expand"] else kw["Hkv"])) * d
        if kind == "heads" and rng.random() < 0.4:
            kw.update(B=B, N=rng.choice([1, 1, 2, 4]), axes=1,
                      cached=_log_int(rng, 1, 100000))
        else:
            B = max(1, min(B, cap // (row * 64)))
            kw.update(B=B, N=_log_int(rng, 64, max(64, min(16384,
                                                           cap // (row * B)))))
        return _case(**kw)
    kw["causal"] = rng.random() < 0.6
    # visible pairs times channels of one call, at most those of exact_16k;
    # two products forward, five backward; fp32 runs on CUDA cores
    cap = 16 * 16384 * 16384 * 128 // 2
    cap //= 10 if kind == "exact_grad" else 4
    cap //= 16 if kw.get("dtype") == "fp32" or d == 32 else 1
    B = max(1, min(B, cap // (H * d * 128 * 128)))
    top = math.isqrt(cap // (B * H * d))
    N = _log_int(rng, 64, max(64, min(16384, top)))
    kw.update(B=B, N=N)
    if kind == "exact" and rng.random() < 0.4:
        kw["Nk"] = max(N, min(4 * N, _log_int(rng, 64, 16384), top * top // N))
    return _case(**kw)


# ------------------------------------------------------------------ inputs

def _spread(B, N, ragged, step):
    """Rows of every sequence: N, or for a padded batch from 1 to N, the first
    N and the third none."""
    out = [max(1, int(N * ((b * step) % 1.0 or 1.0))) for b in range(B)]
    if not ragged:
        out = [N] * B
    elif B > 2:
        out[2] = 0
    return out


def _frequencies(case):
    """Radians per position of every pair: base 10000 over the rotated
    channels."""
    n = case["rot"] // 2
    return [10000.0 ** (-i / n) for i in range(n)]


def _sections(case):
    """Pairs of every axis, as even as they come."""
    n, a = case["rot"] // 2, case["axes"]
    return [n // a + (i < n % a) for i in range(a)]


def _axis_of_pair(case):
    """In blocks: the first axis' pairs, then the next's; in turn: pair p of
    axis p mod axes, while that has any left."""
    left = _sections(case)
    if not case["turn"]:
        return [i for i, n in enumerate(left) for _ in range(n)]
    out, i = [], 0
    while sum(left):
        if left[i]:
            left[i] -= 1
            out.append(i)
        i = (i + 1) % len(left)
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    rnd = lambda *s: torch.randn(*s, generator=g, device=dev)  # noqa: E731
    B, Hkv, G, d, N = (case[x] for x in ("B", "Hkv", "G", "d", "N"))
    H = Hkv * G
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    i32 = dict(dtype=torch.int32, device=dev)
    s = dict(case=case, dt=dt, H=H)
    if case["kind"].startswith("heads"):
        new = _spread(B, N, case["ragged"] and N > 1, 0.7548776662)
        s["new"] = new
        s["new_len"] = torch.tensor(new, **i32) if case["ragged"] else None
        s["lengths"] = s["positions"] = None
        if case["cached"]:
            f = [(b * 0.6180339887) % 1.0 if b and case["ragged"] else 1.0
                 for b in range(B)]
            s["held"] = [int(case["cached"] * x) + n for x, n in zip(f, new)]
            s["lengths"] = torch.tensor(s["held"], **i32)
        elif case["axes"] > 1:
            # text, then an image's rows and columns, then text
            n = torch.arange(N, device=dev).repeat(B, 1)
            side = max(1, math.isqrt(N))
            s["positions"] = torch.stack(
                [n // (side * side)] +
                [n // side % side, n % side][:case["axes"] - 1]).to(
                    torch.int32).contiguous()
        behind = torch.arange(N, device=dev)[None] >= torch.tensor(
            new, device=dev)[:, None]
        # projected rows: channels of different size and offset
        x = rnd(B, N, H + 2 * Hkv, d) * torch.exp(
            0.5 * rnd(H + 2 * Hkv, d)) + 0.5 * rnd(H + 2 * Hkv, d)
        x = x.masked_fill_(behind[:, :, None, None], math.nan).to(dt)
        s["rows"] = x
        s["q"], s["k"], s["v"] = (x[:, :, :H], x[:, :, H:H + Hkv],
                                  x[:, :, H + Hkv:])
        s["wq"] = 1 + 0.2 * rnd(d) if case["norm"] else None
        s["wk"] = 1 + 0.2 * rnd(d) if case["norm"] else None
        Ho = H if case["expand"] else Hkv
        if case["kind"] == "heads":
            for x, h in (("qo", H), ("ko", Ho), ("vo", Ho)):
                s[x] = torch.zeros((B, h, N, d), dtype=dt, device=dev)
        else:
            gt = torch.float32 if case["grad"] == "fp32" else dt
            for x, h in (("dq", H), ("dk", Ho), ("dv", Ho)):
                s[x] = rnd(B, h, N, d).masked_fill_(
                    behind[:, None, :, None], math.nan).to(gt)
            s["drows"] = torch.zeros_like(s["rows"])
            s["dwq"] = s["dwk"] = None
            if case["norm"]:
                s["dwq"], s["dwk"] = (torch.zeros(d, device=dev)
                                      for _ in "qk")
        if own:
            from paper_2607_20214_gb300 import elsaa as E
            s["E"] = E
            s["heads"] = E.make_heads(
                B, H, Hkv, N, d, dtype=case["dtype"], norm=case["norm"],
                rotary=E.make_rotary(case["rot"], base=10000.0,
                                     interleaved=case["neighbours"],
                                     sections=_sections(case),
                                     in_turn=case["turn"]),
                expand=case["expand"], grad_fp32=case["grad"] == "fp32")
            if case["kind"] == "heads_grad":
                s["ws"] = E.new_heads_workspace(s["heads"], dev)
        return s
    M = case["Nk"] or N
    s["M"] = M
    s["ql"] = _spread(B, N, case["ragged"], 0.7548776662)
    s["kl"] = _spread(B, M, case["ragged"], 0.7548776662)
    if case["ragged"] and case["Nk"]:
        # chunks: a sequence with fewer keys than queries, one without any
        s["kl"] = [max(1, int(M * ((b * 0.6180339887) % 1.0 or 1.0)))
                   for b in range(B)]
        s["kl"][3 % B] = 0 if B > 3 else s["kl"][3 % B]
    s["q_len"] = s["k_len"] = None
    if case["ragged"]:
        s["q_len"], s["k_len"] = (torch.tensor(x, **i32)
                                  for x in (s["ql"], s["kl"]))
    qb, kb = (torch.arange(n, device=dev)[None] >= torch.tensor(
        x, device=dev)[:, None] for n, x in ((N, s["ql"]), (M, s["kl"])))
    s["qb"], s["kb"] = qb[:, None, :, None], kb[:, None, :, None]
    scale = 1.0 / math.sqrt(d)
    # scores of standard deviation 2
    s["q"] = (rnd(B, H, N, d) * 1.25).masked_fill_(s["qb"], math.nan).to(dt)
    s["k"], s["v"] = ((rnd(B, Hkv, M, d) * f).masked_fill_(
        s["kb"], math.nan).to(dt) for f in (1.6, 1.0))
    s["scale"] = scale
    if case["kind"] == "exact":
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, H, N), device=dev)
    else:
        # what the forward pass left, and the gradient of its O
        s["do"] = rnd(B, H, N, d).masked_fill_(s["qb"], math.nan).to(dt)
        f = _attend(s)
        s["o"] = f["o"].masked_fill(s["qb"], math.nan)
        s["lse"] = f["lse"].masked_fill(s["qb"][..., 0], math.nan)
        s["dq"], s["dk"], s["dv"] = (torch.zeros_like(s[x]) for x in "qkv")
    if own:
        from paper_2607_20214_gb300 import elsaa as E
        s["E"] = E
        s["exact"] = E.make_exact(B, H, Hkv, N, M, d, dtype=case["dtype"],
                                  causal=case["causal"])
        s["ws"] = E.new_exact_workspace(
            s["exact"], dev, backward=case["kind"] == "exact_grad")
    return s


# ------------------------------------------------------------- plain forms

def _turns(s):
    """cos and sin [B, N, 1, pairs] of every row's angles."""
    c = s["case"]
    n = torch.arange(c["N"], device=s["rows"].device).expand(c["B"], -1)
    if s["lengths"] is not None:
        new = c["N"] if s["new_len"] is None else s["new_len"][:, None]
        n = n + s["lengths"][:, None] - new
    pos = n[None] if s["positions"] is None else s["positions"]
    axis = torch.tensor(_axis_of_pair(c), device=n.device)
    if s["positions"] is None:
        axis = torch.zeros_like(axis)
    a = pos.double()[axis] * torch.tensor(
        _frequencies(c), dtype=torch.float64, device=n.device)[:, None, None]
    a = a.permute(1, 2, 0)[:, :, None]
    return torch.cos(a).float(), torch.sin(a).float()


def _rotate(c, x, cos, sin):
    r = c["rot"]
    if c["neighbours"]:
        lo, hi = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1)
        y = y.flatten(-2)
    else:
        lo, hi = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _valid(s):
    """Rows that a sequence has, [B, N, 1, 1], or None for all."""
    if s["new_len"] is None:
        return None
    n = torch.arange(s["case"]["N"], device=s["rows"].device)
    return (n[None] < s["new_len"][:, None])[:, :, None, None]


def _heads(s):
    c, valid = s["case"], _valid(s)
    cos, sin = _turns(s)

    def done(x, copies=1):
        if valid is not None:
            x = torch.where(valid, x, 0.0)
        if copies > 1:
            x = x.repeat_interleave(copies, 2)
        return x.to(s["dt"]).transpose(1, 2).contiguous()

    def normed(x, w):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        return _rotate(c, x, cos, sin)

    copies = c["G"] if c["expand"] else 1
    return dict(q=done(normed(s["q"], s["wq"])),
                k=done(normed(s["k"], s["wk"]), copies),
                v=done(s["v"].float(), copies))


def _heads_grad(s):
    c, valid = s["case"], _valid(s)
    cos, sin = _turns(s)
    H, Hkv, out = s["H"], c["Hkv"], {}

    def grad(g, heads):
        g = g.float().transpose(1, 2)
        if valid is not None:
            g = torch.where(valid, g, 0.0)
        if g.shape[2] > heads:
            g = g.unflatten(2, (heads, -1)).sum(3)
        return g

    def back(g, x, w):
        u = _rotate(c, g, cos, -sin)
        if not c["norm"]:
            return u, None
        x = x.float() if valid is None else torch.where(valid, x.float(), 0.0)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        xh = x * r
        t = u * w
        dx = r * (t - xh * (t * xh).mean(-1, keepdim=True))
        return dx, (u * xh).sum((0, 1, 2), dtype=torch.float64).float()

    dq, wq = back(grad(s["dq"], H), s["q"], s["wq"])
    dk, wk = back(grad(s["dk"], Hkv), s["k"], s["wk"])
    rows = torch.cat([dq, dk, grad(s["dv"], Hkv)], 2).to(s["dt"])
    out = dict(rows=rows)
    if c["norm"]:
        out.update(wq=wq, wk=wk)
    return out


def _scores(s):
    """Scores of what a query sees, -inf elsewhere [B, Hkv, G, N, M], and
    inputs with zeros behind the sequences, heads in groups."""
    c = s["case"]
    q, k, v = (s[x].float() for x in "qkv")
    if c["ragged"]:
        q = q.masked_fill(s["qb"], 0.0)
        k, v = k.masked_fill(s["kb"], 0.0), v.masked_fill(s["kb"], 0.0)
    q, k, v = q.unflatten(1, (c["Hkv"], c["G"])), k[:, :, None], v[:, :, None]
    x = (q.flatten(2, 3) @ k[:, :, 0].transpose(2, 3)) * s["scale"]
    x = x.unflatten(2, (c["G"], c["N"]))
    i = torch.arange(c["N"], device=x.device)[:, None]
    j = torch.arange(s["M"], device=x.device)
    if c["ragged"]:
        ql, kl = (s[n][:, None, None, None, None] for n in ("q_len", "k_len"))
        hidden = (i >= ql) | (j >= kl)
        if c["causal"]:
            hidden = hidden | (j > i + (kl - ql))
        x.masked_fill_(hidden, -math.inf)
    elif c["causal"]:
        x.masked_fill_(j > i + (s["M"] - c["N"]), -math.inf)
    return x, q, k, v


def _attend(s):
    c = s["case"]
    x, q, k, v = _scores(s)
    m = x.amax(-1, keepdim=True).clamp(min=-1e30)
    p = x.sub_(m).exp_()
    n = p.sum(-1, keepdim=True)
    o = (p.flatten(2, 3) @ v[:, :, 0]).unflatten(2, (c["G"], c["N"]))
    o = torch.where(n > 0, o / n, 0.0)
    lse = (m + torch.log(n))[..., 0].flatten(1, 2)
    if c["ragged"]:
        lse = lse.masked_fill(s["qb"][..., 0], 0.0)
    return dict(o=o.flatten(1, 2).to(s["dt"]), lse=lse)


def _attend_grad(s):
    c = s["case"]
    x, q, k, v = _scores(s)
    do, o, lse = s["do"].float(), s["o"].float(), s["lse"]
    if c["ragged"]:
        do, o = do.masked_fill(s["qb"], 0.0), o.masked_fill(s["qb"], 0.0)
        lse = lse.masked_fill(s["qb"][..., 0], 0.0)
    groups = lambda t: t.unflatten(1, (c["Hkv"], c["G"]))  # noqa: E731
    # a row without a key has lse = -inf and scores of -inf: weights of 0
    lse = groups(lse.clamp(min=-1e30))[..., None]
    p = x.sub_(lse).exp_().flatten(2, 3)
    delta = groups((do * o).sum(-1))[..., None].flatten(2, 3)
    do = groups(do).flatten(2, 3)
    dv = p.transpose(2, 3) @ do
    ds = (do @ v[:, :, 0].transpose(2, 3)).sub_(delta).mul_(p)
    dq = (ds @ k[:, :, 0]) * s["scale"]
    dk = (ds.transpose(2, 3) @ q.flatten(2, 3)) * s["scale"]
    dq = dq.unflatten(2, (c["G"], c["N"])).flatten(1, 2)
    return dict(dq=dq.to(s["dt"]), dk=dk.to(s["dt"]), dv=dv.to(s["dt"]))


def run(s):
    c = s["case"]
    if own:
        E = s["E"]
        if c["kind"] == "heads":
            E.elsaa_heads_forward(
                s["heads"], s["q"], s["k"], s["v"], w_q=s["wq"], w_k=s["wk"],
                positions=s["positions"], lengths=s["lengths"],
                new_len=s["new_len"], q_out=s["qo"], k_out=s["ko"],
                v_out=s["vo"])
            return dict(q=s["qo"], k=s["ko"], v=s["vo"])
        if c["kind"] == "heads_grad":
            x, H, Hkv = s["drows"], s["H"], c["Hkv"]
            E.elsaa_heads_backward(
                s["heads"], s["dq"], s["dk"], s["dv"], q=s["q"], k=s["k"],
                w_q=s["wq"], w_k=s["wk"], positions=s["positions"],
                lengths=s["lengths"], new_len=s["new_len"], dq_rows=x[:, :, :H],
                dk_rows=x[:, :, H:H + Hkv], dv_rows=x[:, :, H + Hkv:],
                dw_q=s["dwq"], dw_k=s["dwk"], workspace=s["ws"])
            out = dict(rows=x)
            if c["norm"]:
                out.update(wq=s["dwq"], wk=s["dwk"])
            return out
        if c["kind"] == "exact":
            E.elsaa_exact_forward(s["exact"], s["q"], s["k"], s["v"],
                                  q_len=s["q_len"], k_len=s["k_len"],
                                  o=s["o"], lse=s["lse"], workspace=s["ws"])
            return dict(o=s["o"], lse=s["lse"])
        E.elsaa_exact_backward(s["exact"], s["q"], s["k"], s["v"], s["o"],
                               s["lse"], s["do"], q_len=s["q_len"],
                               k_len=s["k_len"], dq=s["dq"], dk=s["dk"],
                               dv=s["dv"], workspace=s["ws"])
        return dict(dq=s["dq"], dk=s["dk"], dv=s["dv"])
    if c["kind"] == "heads":
        return _heads(s)
    if c["kind"] == "heads_grad":
        return _heads_grad(s)
    if c["kind"] == "exact":
        return _attend(s)
    return _attend_grad(s)


# -------------------------------------------- the definition, in 64 bits

def _turn_matrix(s, b):
    """Sequence b's rotations as one complex number a row and pair."""
    c, N = s["case"], s["case"]["N"]
    dev = s["rows"].device
    start = s["held"][b] - s["new"][b] if s["lengths"] is not None else 0
    z = []
    for axis, f in zip(_axis_of_pair(c), _frequencies(c)):
        if s["positions"] is not None:
            p = s["positions"][axis, b].to(torch.float64)
        else:
            p = start + torch.arange(N, dtype=torch.float64, device=dev)
        z.append(torch.polar(torch.ones_like(p), p * f))
    return torch.stack(z, -1)


def _paired(c, x):
    """The rotated channels as complex pairs, and the others."""
    r, rest = c["rot"], x[..., c["rot"]:]
    if c["neighbours"]:
        return torch.view_as_complex(
            x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()), rest
    return torch.complex(x[..., :r // 2].contiguous(),
                         x[..., r // 2:r].contiguous()), rest


def _unpaired(c, z, rest):
    if c["neighbours"]:
        y = torch.view_as_real(z).reshape(*z.shape[:-1], c["rot"])
    else:
        y = torch.cat((z.real, z.imag), -1)
    return torch.cat((y, rest), -1)


def _exact_heads(s):
    c = s["case"]
    B, N, H, Hkv, G = c["B"], c["N"], s["H"], c["Hkv"], c["G"]
    out = {x: torch.zeros(s[x + "o"].shape, dtype=torch.float64,
                          device=s["rows"].device) for x in "qkv"}
    for b in range(B):
        n = s["new"][b]
        turn = _turn_matrix(s, b)[:n]
        for x, w, heads in (("q", s["wq"], H), ("k", s["wk"], Hkv),
                            ("v", None, Hkv)):
            for h in range(heads):
                y = s[x][b, :n, h].double()
                if x != "v":
                    if c["norm"]:
                        y = y / torch.sqrt((y * y).mean(1, True) + 1e-6)
                        y = y * w.double()
                    z, rest = _paired(c, y)
                    y = _unpaired(c, z * turn, rest)
                copies = G if c["expand"] and x != "q" else 1
                for i in range(copies):
                    out[x][b, h * copies + i, :n] = y
    return out


def _exact_heads_grad(s):
    c = s["case"]
    B, H, Hkv, G, d = c["B"], s["H"], c["Hkv"], c["G"], c["d"]
    rows = torch.zeros(s["rows"].shape, dtype=torch.float64,
                       device=s["rows"].device)
    dw = {x: torch.zeros(d, dtype=torch.float64, device=rows.device)
          for x in "qk"}
    for b in range(B):
        n = s["new"][b]
        if n == 0:
            continue
        turn = _turn_matrix(s, b)[:n].conj()
        for x, w, heads, at in (("q", s["wq"], H, 0), ("k", s["wk"], Hkv, H),
                                ("v", None, Hkv, H + Hkv)):
            copies = G if c["expand"] and x != "q" else 1
            for h in range(heads):
                g = s["d" + x][b, h * copies:(h + 1) * copies, :n]
                g = g.double().sum(0)
                if x != "v":
                    z, rest = _paired(c, g)
                    g = _unpaired(c, z * turn, rest)
                    if c["norm"]:
                        # the Jacobian of y = w x / sqrt(mean x^2 + eps)
                        y = s[x][b, :n, h].double()
                        m = (y * y).mean(1, True) + 1e-6
                        dw[x] += (g * y / torch.sqrt(m)).sum(0)
                        g = g * w.double()
                        g = (g - y * (g * y).sum(1, True) / (d * m)) \
                            / torch.sqrt(m)
                rows[b, :n, at + h] = g
    out = dict(rows=rows)
    if c["norm"]:
        out.update(wq=dw["q"], wk=dw["k"])
    return out


def _exact_softmax(s, b, h):
    """Weights, lse and inputs of one query head, over what it holds."""
    c = s["case"]
    nq, nk = s["ql"][b], s["kl"][b]
    q = s["q"][b, h, :nq].double()
    k, v = (s[x][b, h // c["G"], :nk].double() for x in "kv")
    if nk == 0:
        return None, torch.full((nq,), -math.inf, dtype=torch.float64,
                                device=q.device), q, k, v
    x = torch.mm(q, k.t()).mul_(s["scale"])
    if c["causal"]:
        x = x.masked_fill_(torch.ones_like(x, dtype=torch.bool).triu_(
            1 + nk - nq), -math.inf)
    lse = torch.logsumexp(x, 1)
    seen = torch.isfinite(lse)
    p = x.sub_(torch.where(seen, lse, 0.0)[:, None]).exp_()
    return p, lse, q, k, v


def _exact_attend(s):
    c = s["case"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(s["q"].shape[:3], dtype=torch.float64,
                      device=o.device)
    for b in range(c["B"]):
        for h in range(s["H"]):
            p, z, _, _, v = _exact_softmax(s, b, h)
            lse[b, h, :len(z)] = z
            if p is not None:
                o[b, h, :len(z)] = p @ v
    return dict(o=o, lse=lse)


def _exact_attend_grad(s):
    c = s["case"]
    out = {x: torch.zeros(s[x[1]].shape, dtype=torch.float64,
                          device=s["q"].device) for x in ("dq", "dk", "dv")}
    for b in range(c["B"]):
        for h in range(s["H"]):
            p, z, q, k, v = _exact_softmax(s, b, h)
            if p is None or not len(z):
                continue
            nq, nk, j = len(q), len(k), h // c["G"]
            g = s["do"][b, h, :nq].double()
            out["dv"][b, j, :nk] += p.t() @ g
            t = g @ v.t()
            t = p * (t - (p * t).sum(1, True))
            out["dq"][b, h, :nq] = s["scale"] * (t @ k)
            out["dk"][b, j, :nk] += s["scale"] * (t.t() @ q)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "heads":
        return _exact_heads(s)
    if case["kind"] == "heads_grad":
        return _exact_heads_grad(s)
    # 64-bit products at about 1 TFLOP/s
    if work(case)["flops"] * (2 if case["causal"] else 1) > 8e12:
        return None
    return _exact_attend(s) if case["kind"] == "exact" else \
        _exact_attend_grad(s)


# -------------------------------------------------------------------- work

def _pairs(nq, nk, causal):
    """Pairs of a query and a key that it sees."""
    if not causal:
        return nq * nk
    # query i sees i + 1 + nk - nq keys, or none
    first = max(0, nq - nk)
    n = nq - first
    return n * (1 + first + nk - nq) + n * (n - 1) // 2


def work(case):
    """Bytes and operations of one pass: every input and output that a
    sequence has once; attention's products over the pairs that are seen."""
    B, Hkv, G, d, N = (case[x] for x in ("B", "Hkv", "G", "d", "N"))
    el = 4 if case["dtype"] == "fp32" else 2
    H = Hkv * G
    if case["kind"].startswith("heads"):
        n = sum(_spread(B, N, case["ragged"] and N > 1, 0.7548776662))
        rows, out = H + 2 * Hkv, H + 2 * (H if case["expand"] else Hkv)
        if case["kind"] == "heads":
            return dict(bytes=n * d * el * (rows + out),
                        flops=n * d * 8 * rows)
        ge = 4 if case["grad"] == "fp32" else 2
        b = n * d * (out * ge + rows * el)
        if case["norm"]:
            b += n * d * el * (H + Hkv)
        return dict(bytes=b, flops=n * d * 14 * rows)
    M = case["Nk"] or N
    ql = _spread(B, N, case["ragged"], 0.7548776662)
    kl = _spread(B, M, case["ragged"], 0.7548776662)
    if case["ragged"] and case["Nk"]:
        kl = [max(1, int(M * ((b * 0.6180339887) % 1.0 or 1.0)))
              for b in range(B)]
        kl[3 % B] = 0 if B > 3 else kl[3 % B]
    pairs = H * sum(_pairs(q, k, case["causal"]) for q, k in zip(ql, kl))
    q, k = sum(ql) * H, sum(kl) * Hkv
    if case["kind"] == "exact":
        return dict(bytes=(2 * q + 2 * k) * d * el + 4 * q,
                    flops=4 * d * pairs)
    return dict(bytes=(4 * q + 4 * k) * d * el + 4 * q, flops=10 * d * pairs)
