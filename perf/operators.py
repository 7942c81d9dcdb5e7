"""The operators a training step of a transformer block needs between its quantized linears, as cases that can be timed: the norm of
queries and keys with the position rotation, and attention that keeps its row statistic, each with its gradient.

A case is a dict of plain values.  ``listed()`` gives the fixed ones, ``draw(rng)`` one more of the same ranges, ``prepare``
what a program holds before the call, ``run`` one pass (the plain form in elementary torch operations, or the calls of
``paper_2512_05746_b200.binding`` where ``own`` is true), ``work`` the bytes and operations a pass cannot do without, ``exact``
the same outputs in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # queries and keys of one image of 16 latent tokens: latency
        dict(name="qk_rope_16", kind="rope", rows=16, tokens=16, heads=8, kv_heads=8, dh=64, rot=64, interleaved=False, dtype="bf16",
             gamma=True, positions=False),
        # the 32x32 level at a full batch of 64 images, in the fused qkv tensor
        dict(name="qk_rope_64k", kind="rope", rows=65536, tokens=1024, heads=8, kv_heads=8, dh=64, rot=64, interleaved=False,
             dtype="bf16", gamma=True, positions=False),
        # gradient of the same
        dict(name="qk_rope_grad_64k", kind="rope_grad", rows=65536, tokens=1024, heads=8, kv_heads=8, dh=64, rot=64,
             interleaved=False, dtype="bf16", gamma=True, positions=False),
        # gradient in a diffusion-transformer block of width 1152 (32 images of 256 tokens, 16 heads of 72) in fp32, with
        # token positions of a packed batch and a part of the head left unrotated
        dict(name="qk_rope_grad_dit", kind="rope_grad", rows=8192, tokens=256, heads=16, kv_heads=16, dh=72, rot=64, interleaved=True,
             dtype="f32", gamma=True, positions=True),
        # attention of two images of 8x8 latent tokens: latency
        dict(name="attn_64", kind="attn", Nb=2, Lq=64, Lk=64, heads=8, kv_heads=8, dh=64, causal=False, lens=False),
        # the diffusion-transformer block: 32 images of 256 tokens, 16 heads of 72
        dict(name="attn_dit_256", kind="attn", Nb=32, Lq=256, Lk=256, heads=16, kv_heads=16, dh=72, causal=False, lens=False),
        # the 32x32 level at a full batch
        dict(name="attn_1024", kind="attn", Nb=64, Lq=1024, Lk=1024, heads=8, kv_heads=8, dh=64, causal=False, lens=False),
        # long token sequences in raster order, two key heads for sixteen query heads
        dict(name="attn_causal_4096", kind="attn", Nb=2, Lq=4096, Lk=4096, heads=16, kv_heads=2, dh=128, causal=True, lens=False),
        # gradients of the above
        dict(name="attn_grad_64", kind="attn_grad", Nb=2, Lq=64, Lk=64, heads=8, kv_heads=8, dh=64, causal=False, lens=False),
        dict(name="attn_grad_1024", kind="attn_grad", Nb=64, Lq=1024, Lk=1024, heads=8, kv_heads=8, dh=64, causal=False, lens=False),
        dict(name="attn_grad_causal_4096", kind="attn_grad", Nb=2, Lq=4096, Lk=4096, heads=16, kv_heads=2, dh=128, causal=True,
             lens=False),
        # 64x64 latent tokens that look at up to 77 text tokens, the first caption dropped altogether
        dict(name="attn_grad_text_77", kind="attn_grad", Nb=8, Lq=4096, Lk=77, heads=8, kv_heads=8, dh=40, causal=False, lens=True),
    ]


# ------------------------------------------------------------------------------------------------------ drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope_grad", "attn", "attn", "attn_grad", "attn_grad", "attn_grad"])
    heads, kv_heads = rng.choice([(4, 4), (8, 8), (8, 2), (12, 12), (16, 16), (16, 1), (16, 4), (6, 3)])
    dh = rng.choice([32, 40, 48, 64, 64, 72, 80, 96, 128])
    if kind in ("rope", "rope_grad"):
        tokens = _log_int(rng, 1, 4096)
        rows = _log_int(rng, 1, 33_000_000 // (heads * dh) // 2)
        return dict(kind=kind, rows=rows, tokens=tokens, heads=heads, kv_heads=kv_heads, dh=dh, rot=rng.choice([dh, dh, dh // 2]),
                    interleaved=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]), gamma=rng.random() < 0.8,
                    positions=rng.random() < 0.5)
    Lq = _log_int(rng, 1, 4096)
    Lk = rng.choice([Lq, Lq, _log_int(rng, 1, 4096)])
    most = 3.4e11 / (10 * dh * heads * Lq * Lk)
    Nb = _log_int(rng, 1, max(1, min(64, int(most))))
    return dict(kind=kind, Nb=Nb, Lq=Lq, Lk=Lk, heads=heads, kv_heads=kv_heads, dh=dh, causal=rng.random() < 0.3,
                lens=rng.random() < 0.4)


# --------------------------------------------------------------------------------------- what a program has in hand

def _lengths(L, Nb):
    """Lengths of a padded batch, from an empty sample (a dropped caption) to a full one; one sample is full."""
    return [L] if Nb == 1 else [L * n // (Nb - 1) for n in range(Nb)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    H, G, dh = case["heads"], case["kv_heads"], case["dh"]
    state = dict(case)
    if case["kind"] in ("rope", "rope_grad"):
        dt, rows, tokens, half = DTYPES[case["dtype"]], case["rows"], case["tokens"], case["rot"] // 2
        # rows of the fused projection: queries, keys and values; a few channels are larger than the rest
        width = (H + 2 * G) * dh
        qkv = randn(rows, width)
        qkv[:, torch.randperm(width, generator=gen, device="cuda")[: max(1, width // 100)]] *= 8.0
        qkv = qkv.to(dt)
        angle = torch.arange(tokens, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (
            -torch.arange(half, dtype=torch.float64, device="cuda") / max(1, half))
        state.update(q=qkv[:, : H * dh], k=qkv[:, H * dh: (H + G) * dh], cos=angle.cos().float(), sin=angle.sin().float(),
                     gamma_q=1.0 + 0.2 * randn(dh) if case["gamma"] else None, gamma_k=1.0 + 0.2 * randn(dh) if case["gamma"] else None,
                     pos=torch.randint(0, tokens, (rows,), generator=gen, device="cuda").to(torch.int32) if case["positions"] else None)
        if case["kind"] == "rope":
            state.update(q_out=torch.empty((rows, H * dh), dtype=dt, device="cuda"), k_out=torch.empty((rows, G * dh), dtype=dt, device="cuda"))
        else:
            dqkv = torch.empty((rows, width), dtype=dt, device="cuda")
            state.update(dq_out=randn(rows, H * dh).to(dt), dk_out=randn(rows, G * dh).to(dt), dq=dqkv[:, : H * dh],
                         dk=dqkv[:, H * dh: (H + G) * dh], dgamma_q=torch.empty(dh, device="cuda"), dgamma_k=torch.empty(dh, device="cuda"))
        return state
    Nb, Lq, Lk = case["Nb"], case["Lq"], case["Lk"]
    bf = torch.bfloat16
    if Lq == Lk:                                   # self-attention: slices of the fused projection
        qkv = randn(Nb * Lq, (H + 2 * G) * dh).to(bf)
        q, k, v = qkv[:, : H * dh], qkv[:, H * dh: (H + G) * dh], qkv[:, (H + G) * dh:]
    else:                                          # queries of the image, keys and values of the text
        q, kv = randn(Nb * Lq, H * dh).to(bf), randn(Nb * Lk, 2 * G * dh).to(bf)
        k, v = kv[:, : G * dh], kv[:, G * dh:]
    order = torch.randperm(Nb, generator=gen, device="cuda")
    k_lens = torch.tensor(_lengths(Lk, Nb), dtype=torch.int32, device="cuda")[order].contiguous() if case["lens"] else None
    state.update(q=q, k=k, v=v, k_lens=k_lens, q_lens=k_lens if Lq == Lk else None, scale=1.0 / math.sqrt(dh))
    if case["kind"] == "attn":
        state.update(out=torch.empty((Nb * Lq, H * dh), dtype=bf, device="cuda"), lse=torch.empty((Nb, H, Lq), device="cuda"))
        return state
    out, lse = _attention(state)
    dqkv = torch.empty((Nb * Lq, (H + 2 * G) * dh), dtype=bf, device="cuda") if Lq == Lk else None
    dkv = torch.empty((Nb * Lk, 2 * G * dh), dtype=bf, device="cuda") if Lq != Lk else None
    state.update(out=out, lse=lse, dout=randn(Nb * Lq, H * dh).to(bf))
    if Lq == Lk:
        state.update(dq=dqkv[:, : H * dh], dk=dqkv[:, H * dh: (H + G) * dh], dv=dqkv[:, (H + G) * dh:])
    else:
        state.update(dq=torch.empty((Nb * Lq, H * dh), dtype=bf, device="cuda"), dk=dkv[:, : G * dh], dv=dkv[:, G * dh:])
    return state


# ----------------------------------------------------------------------------------------------------- plain forms

def _table(s, dtype):
    """cos and sin of every row, [rows, 1, rot / 2]."""
    at = s["pos"].long() if s["pos"] is not None else torch.arange(s["rows"], device="cuda") % s["tokens"]
    return s["cos"].to(dtype)[at][:, None], s["sin"].to(dtype)[at][:, None]


def _halves(x, rot, interleaved):
    """The first and second members of the rotated pairs, and what is not rotated."""
    r = x[..., :rot]
    return (r[..., 0::2], r[..., 1::2], x[..., rot:]) if interleaved else (r[..., : rot // 2], r[..., rot // 2:], x[..., rot:])


def _join(a, b, rest, interleaved):
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1)


def _rope(s, x, heads, gamma):
    y = x.float().reshape(x.shape[0], heads, -1)
    y = y * (y.square().mean(-1, keepdim=True) + EPS).rsqrt()
    if gamma is not None:
        y = y * gamma
    c, sn = _table(s, torch.float32)
    a, b, rest = _halves(y, s["rot"], s["interleaved"])
    return _join(a * c - b * sn, b * c + a * sn, rest, s["interleaved"]).flatten(1).to(x.dtype)


def _rope_grad(s, x, dout, heads, gamma):
    y, u = x.float().reshape(x.shape[0], heads, -1), dout.float().reshape(x.shape[0], heads, -1)
    inv = (y.square().mean(-1, keepdim=True) + EPS).rsqrt()
    c, sn = _table(s, torch.float32)
    a, b, rest = _halves(u, s["rot"], s["interleaved"])
    u, y = _join(a * c + b * sn, b * c - a * sn, rest, s["interleaved"]), y * inv
    dgamma = (u * y).sum((0, 1))
    if gamma is not None:
        u = u * gamma
    return (inv * (u - y * (u * y).mean(-1, keepdim=True))).flatten(1).to(x.dtype), dgamma


def _heads(x, Nb, heads, dtype):
    return x.to(dtype).reshape(Nb, -1, heads, x.shape[1] // heads).transpose(1, 2)


def _visible(s):
    """[Nb, 1, 1, Lq, Lk]: which keys a query looks at."""
    Nb, Lq, Lk = s["Nb"], s["Lq"], s["Lk"]
    ql = (s["q_lens"] if s["q_lens"] is not None else torch.full((Nb,), Lq, device="cuda")).long().view(Nb, 1, 1)
    kl = (s["k_lens"] if s["k_lens"] is not None else torch.full((Nb,), Lk, device="cuda")).long().view(Nb, 1, 1)
    i, j = torch.arange(Lq, device="cuda").view(1, Lq, 1), torch.arange(Lk, device="cuda").view(1, 1, Lk)
    seen = (i < ql) & (j < kl)
    if s["causal"]:
        seen = seen & (j <= i + (kl - ql))
    return seen[:, None, None]


def _scores(s, dtype):
    Nb, H, G = s["Nb"], s["heads"], s["kv_heads"]
    q, k, v = _heads(s["q"], Nb, H, dtype).unflatten(1, (G, H // G)), _heads(s["k"], Nb, G, dtype)[:, :, None], _heads(s["v"], Nb, G, dtype)[:, :, None]
    S = (q @ k.transpose(-1, -2)) * s["scale"]
    if s["causal"] or s["k_lens"] is not None:
        S = S.masked_fill(~_visible(s), -math.inf)
    return q, k, v, S


def _attention(s):
    q, k, v, S = _scores(s, torch.float32)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = (S - m).exp_()
    l = P.sum(-1, keepdim=True)
    out = (P @ v) / torch.where(l == 0, torch.ones_like(l), l)
    return out.flatten(1, 2).transpose(1, 2).flatten(0, 1).flatten(1).to(torch.bfloat16), (m + l.log()).flatten(1, 2)[..., 0]


def _rows(x):
    """[Nb, G, heads a group, L, dh] -> [Nb * L, heads * dh]"""
    return x.flatten(1, 2).transpose(1, 2).flatten(0, 1).flatten(1)


def _attention_grad(s, dtype):
    q, k, v, S = _scores(s, dtype)
    Nb, H, G = s["Nb"], s["heads"], s["kv_heads"]
    group = lambda x: _heads(x, Nb, H, dtype).unflatten(1, (G, H // G))  # noqa: E731
    lse = s["lse"].to(dtype).unflatten(1, (G, H // G))[..., None]
    P = (S - torch.where(lse == -math.inf, torch.full_like(lse, math.inf), lse)).exp_()
    dout, out = group(s["dout"]), group(s["out"])
    dS = (dout @ v.transpose(-1, -2) - (dout * out).sum(-1, keepdim=True)).mul_(P)
    dq, dk = (dS @ k) * s["scale"], (dS.transpose(-1, -2) @ q).sum(2, keepdim=True) * s["scale"]
    dv = (P.transpose(-1, -2) @ dout).sum(2, keepdim=True)
    return _rows(dq), _rows(dk), _rows(dv)


def _plain(s):
    H, G = s["heads"], s["kv_heads"]
    if s["kind"] == "rope":
        return {"q": _rope(s, s["q"], H, s["gamma_q"]), "k": _rope(s, s["k"], G, s["gamma_k"])}
    if s["kind"] == "rope_grad":
        dq, dgq = _rope_grad(s, s["q"], s["dq_out"], H, s["gamma_q"])
        dk, dgk = _rope_grad(s, s["k"], s["dk_out"], G, s["gamma_k"])
        return {"dq": dq, "dk": dk, "dgamma_q": dgq, "dgamma_k": dgk} if s["gamma"] else {"dq": dq, "dk": dk}
    if s["kind"] == "attn":
        out, lse = _attention(s)
        return {"out": out, "lse": lse}
    dq, dk, dv = _attention_grad(s, torch.float32)
    return {"dq": dq.to(torch.bfloat16), "dk": dk.to(torch.bfloat16), "dv": dv.to(torch.bfloat16)}


# ----------------------------------------------------------------------------------------------- the framework's calls

def _workspace(s, size, *args):
    """The workspace of these sizes, which a program allocates once."""
    if "workspace" not in s:
        s["workspace"] = torch.empty((max(16, size(*args)),), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own(s):
    from paper_2512_05746_b200 import binding as hq
    H, G = s["heads"], s["kv_heads"]
    if s["kind"] == "rope":
        hq.hq_qk_norm_rope(s["q"], s["k"], H, G, s["gamma_q"], s["gamma_k"], EPS, s["cos"], s["sin"], s["q_out"], s["k_out"],
                           positions=s["pos"], interleaved=s["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if s["kind"] == "rope_grad":
        ws = _workspace(s, hq.hq_qk_norm_rope_bwd_workspace_size, s["rows"], H, G, s["dh"])
        dgq, dgk = (s["dgamma_q"], s["dgamma_k"]) if s["gamma"] else (None, None)
        hq.hq_qk_norm_rope_bwd(s["q"], s["k"], H, G, s["gamma_q"], s["gamma_k"], EPS, s["cos"], s["sin"], s["dq_out"], s["dk_out"],
                               s["dq"], s["dk"], dgq, dgk, ws, positions=s["pos"], interleaved=s["interleaved"])
        return {"dq": s["dq"], "dk": s["dk"], "dgamma_q": dgq, "dgamma_k": dgk} if s["gamma"] else {"dq": s["dq"], "dk": s["dk"]}
    if s["kind"] == "attn":
        ws = _workspace(s, hq.hq_attention_fwd_workspace_size, s["Nb"], s["Lq"], s["Lk"], H, G, s["dh"])
        hq.hq_attention_fwd(s["q"], s["k"], s["v"], s["Nb"], H, G, s["out"], s["lse"], ws, q_lens=s["q_lens"], k_lens=s["k_lens"],
                            causal=s["causal"], scale=s["scale"])
        return {"out": s["out"], "lse": s["lse"]}
    ws = _workspace(s, hq.hq_attention_bwd_workspace_size, s["Nb"], s["Lq"], s["Lk"], H, G, s["dh"])
    hq.hq_attention_bwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["Nb"], H, G, s["dq"], s["dk"], s["dv"], ws,
                        q_lens=s["q_lens"], k_lens=s["k_lens"], causal=s["causal"], scale=s["scale"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work and exactness

def _pairs(case):
    """Visible (query, key) pairs of one head over the batch, and the query and key rows inside their lengths."""
    Nb, Lq, Lk = case["Nb"], case["Lq"], case["Lk"]
    kl = _lengths(Lk, Nb) if case["lens"] else [Lk] * Nb
    ql = kl if case["lens"] and Lq == Lk else [Lq] * Nb
    pairs = 0
    for a, b in zip(ql, kl):
        if case["causal"]:                         # query i sees keys 0 .. i + b - a
            first = max(0, a - b)                  # the first query that sees a key
            n = a - first
            pairs += n * (first + 1 + b - a) + n * (n - 1) // 2 if n > 0 and b > 0 else 0
        else:
            pairs += a * b
    return pairs, sum(ql), sum(kl)


def work(case):
    H, G, dh = case["heads"], case["kv_heads"], case["dh"]
    if case["kind"] in ("rope", "rope_grad"):
        size, elements = (2 if case["dtype"] == "bf16" else 4), case["rows"] * (H + G) * dh
        tables = 4 * min(case["tokens"], case["rows"]) * case["rot"] + (4 * case["rows"] if case["positions"] else 0)
        if case["kind"] == "rope":
            return {"bytes": 2 * size * elements + tables, "flops": 10 * elements}
        return {"bytes": 3 * size * elements + tables + (8 * dh if case["gamma"] else 0), "flops": 20 * elements}
    pairs, rows_q, rows_k = _pairs(case)
    Nb, Lq, Lk = case["Nb"], case["Lq"], case["Lk"]
    if case["kind"] == "attn":
        return {"bytes": 2 * dh * (H * (rows_q + Nb * Lq) + 2 * G * rows_k) + 4 * Nb * H * Lq, "flops": 4 * dh * H * pairs}
    return {"bytes": 2 * dh * (H * (3 * rows_q + Nb * Lq) + 2 * G * (rows_k + Nb * Lk)) + 4 * H * rows_q, "flops": 10 * dh * H * pairs}


def exact(case, seed):
    """From the definitions, in 64 bits: the rotation as a product of complex numbers, the softmax by torch's logsumexp, and
    the gradients by torch's differentiation of the norm and, for attention, of the scores."""
    s = prepare(case, seed)
    H, G, dh = case["heads"], case["kv_heads"], case["dh"]
    f64 = torch.float64
    if case["kind"] in ("rope", "rope_grad"):
        at = s["pos"].long() if s["pos"] is not None else torch.arange(case["rows"], device="cuda") % case["tokens"]
        turn = torch.complex(s["cos"].to(f64), s["sin"].to(f64))[at][:, None]
        rot = case["rot"]

        def forward(x, heads, gamma):
            x = x.reshape(x.shape[0], heads, dh)
            y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / dh + EPS)
            y = y * gamma if gamma is not None else y
            if case["interleaved"]:
                z = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:-1], rot // 2, 2).contiguous()) * turn
                z = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(y[..., : rot // 2].contiguous(), y[..., rot // 2: rot].contiguous()) * turn
                z = torch.cat((z.real, z.imag), -1)
            return torch.cat((z, y[..., rot:]), -1).flatten(1)

        wide = lambda t: None if t is None else t.to(f64).clone()  # noqa: E731
        if case["kind"] == "rope":
            return {"q": forward(wide(s["q"]), H, wide(s["gamma_q"])), "k": forward(wide(s["k"]), G, wide(s["gamma_k"]))}
        found = {}
        for n, heads in (("q", H), ("k", G)):
            x, g = wide(s[n]).requires_grad_(), wide(s["gamma_" + n])
            leaves = [x] if g is None else [x, g.requires_grad_()]
            grads = torch.autograd.grad(forward(x, heads, g), leaves, s["d%s_out" % n].to(f64))
            found["d" + n] = grads[0]
            if g is not None:
                found["dgamma_" + n] = grads[1]
        return {n: found[n] for n in (("dq", "dk", "dgamma_q", "dgamma_k") if case["gamma"] else ("dq", "dk"))}
    Nb, Lq, Lk = case["Nb"], case["Lq"], case["Lk"]
    q = s["q"].to(f64).view(Nb, Lq, H, dh).permute(0, 2, 1, 3)
    k, v = (t.to(f64).view(Nb, Lk, G, dh).permute(0, 2, 1, 3).repeat_interleave(H // G, 1) for t in (s["k"], s["v"]))
    ql = s["q_lens"].tolist() if s["q_lens"] is not None else [Lq] * Nb
    kl = s["k_lens"].tolist() if s["k_lens"] is not None else [Lk] * Nb
    S = torch.einsum("nhid,nhjd->nhij", q, k) / math.sqrt(dh)
    hidden = torch.zeros((Nb, 1, Lq, Lk), dtype=torch.bool, device="cuda")
    for n in range(Nb):
        hidden[n, :, ql[n]:], hidden[n, :, :, kl[n]:] = True, True
        if case["causal"]:
            hidden[n] |= torch.ones((Lq, Lk), dtype=torch.bool, device="cuda").triu(kl[n] - ql[n] + 1)
    S.masked_fill_(hidden, -math.inf)
    if case["kind"] == "attn":
        lse = torch.logsumexp(S, -1)
        P = S.sub_(lse[..., None]).exp_().nan_to_num_(nan=0.0)
        return {"out": torch.einsum("nhij,nhjd->nihd", P, v).reshape(Nb * Lq, H * dh), "lse": lse}
    P = S.sub_(s["lse"].to(f64)[..., None]).exp_().nan_to_num_(nan=0.0)
    dout, out = (s[t].to(f64).view(Nb, Lq, H, dh).permute(0, 2, 1, 3) for t in ("dout", "out"))
    dv = torch.einsum("nhij,nhid->njhd", P, dout).reshape(Nb, Lk, G, H // G, dh).sum(3)
    dS = torch.einsum("nhid,nhjd->nhij", dout, v).sub_((dout * out).sum(-1)[..., None]).mul_(P)
    dq = torch.einsum("nhij,nhjd->nihd", dS, k) / math.sqrt(dh)
    dk = torch.einsum("nhij,nhid->njhd", dS, q).reshape(Nb, Lk, G, H // G, dh).sum(3) / math.sqrt(dh)
    return {"dq": dq.reshape(Nb * Lq, H * dh), "dk": dk.reshape(Nb * Lk, G * dh), "dv": dv.reshape(Nb * Lk, G * dh)}
