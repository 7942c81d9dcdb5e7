"""The operators a training step of a conditional diffusion transformer needs around its linears and its attention, as cases that can be
timed: the gated residual with the norms before and after a block and its gradient, the embedding lookup with scaling and its gradient,
and the norm of all gradients with clipping.

A case is a dict of plain values.  ``listed()`` gives the fixed ones, ``draw(rng)`` one more of the same ranges, ``prepare``
what a program holds before the call, ``run`` one pass (the plain form in elementary torch operations, or the calls of
``paper_2512_05746_b200.binding`` where ``own`` is true), ``work`` the bytes and operations a pass cannot do without, ``exact``
the same outputs in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # the 16 latent tokens of two samples: latency
        dict(name="gate_norm_32", kind="norm", rows=32, cols=1152, group=16, norm="layer", post="none", gate=True, lens=False, residual=1.0,
             xdtype="bf16", hdtype="bf16"),
        # between the attention and the MLP of a diffusion-transformer block: 32 images of 256 tokens
        dict(name="gate_norm_dit", kind="norm", rows=8192, cols=1152, group=256, norm="layer", post="none", gate=True, lens=False,
             residual=1.0, xdtype="bf16", hdtype="bf16"),
        # the 32x32 level at a full batch of 64 images, a norm behind the block as well, the residual stream in fp32
        dict(name="gate_norm_post_64k", kind="norm", rows=65536, cols=512, group=1024, norm="rms", post="rms", gate=True, lens=False,
             residual=0.7071, xdtype="f32", hdtype="bf16"),
        # gradient of the diffusion-transformer block's
        dict(name="gate_norm_grad_dit", kind="norm_grad", rows=8192, cols=1152, group=256, norm="layer", post="none", gate=True, lens=False,
             residual=1.0, xdtype="bf16", hdtype="bf16"),
        # the same at eight times the batch
        dict(name="gate_norm_grad_64k", kind="norm_grad", rows=65536, cols=1152, group=256, norm="layer", post="none", gate=True, lens=False,
             residual=1.0, xdtype="bf16", hdtype="bf16"),
        # text tokens of ragged lengths between two norms, no condition
        dict(name="gate_norm_grad_text", kind="norm_grad", rows=64 * 77, cols=1000, group=77, norm="rms", post="rms", gate=False, lens=True,
             residual=1.0, xdtype="f32", hdtype="bf16"),
        # class labels of a batch: latency
        dict(name="embed_labels", kind="embed", tokens=64, classes=1001, dim=1152, ids="uniform", dtype="bf16", outdtype="bf16",
             scale=1.0, accumulate=False),
        # captions of 77 tokens for 256 images
        dict(name="embed_text", kind="embed", tokens=256 * 77, classes=32768, dim=768, ids="padded", dtype="bf16", outdtype="bf16",
             scale=27.7, accumulate=False),
        # gradient of the class table, added to the one of earlier micro-batches
        dict(name="embed_grad_labels", kind="embed_grad", tokens=64, classes=1001, dim=1152, ids="uniform", dtype="bf16", outdtype="f32",
             scale=1.0, accumulate=True),
        # gradient of the captions' table, most of the tokens padding of one id
        dict(name="embed_grad_text", kind="embed_grad", tokens=256 * 77, classes=32768, dim=768, ids="padded", dtype="bf16", outdtype="bf16",
             scale=27.7, accumulate=False),
        # low-rank factors of 28 blocks (rank 8): many small tensors
        dict(name="clip_factors", kind="clip", tensors=280, largest=36864, total=5_000_000, dtype="f32", outdtype="f32", max_norm=1.0),
        # as many tensors and elements as a diffusion transformer of 28 blocks of width 1152 has: bf16 gradients, fp32 for the optimizer
        dict(name="clip_dit", kind="clip", tensors=287, largest=6 * 1152 * 1152, total=675_000_000, dtype="bf16", outdtype="f32", max_norm=1.0),
    ]


# ------------------------------------------------------------------------------------------------------ drawn cases

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "norm_grad", "embed", "embed_grad", "embed_grad", "clip"])
    if kind in ("norm", "norm_grad"):
        cols = rng.choice([64, 128, 200, 320, 512, 640, 768, 1000, 1152, 1152, 1280, 2048, 2304, 4096])
        rows = _log_int(rng, 1, 65536 * 1152 // (2 * cols))
        group = rng.choice([0, 1, 16, 77, 256, 1024, _log_int(rng, 1, max(2, rows))])
        xdtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(kind=kind, rows=rows, cols=cols, group=group, norm=rng.choice(["layer", "layer", "rms"]),
                    post=rng.choice(["none", "none", "layer", "rms"]), gate=rng.random() < 0.7, lens=group > 1 and rng.random() < 0.3,
                    residual=rng.choice([1.0, 1.0, 0.7071]), xdtype=xdtype,
                    hdtype="bf16" if xdtype == "bf16" else rng.choice(["f32", "bf16"]))
    if kind in ("embed", "embed_grad"):
        dim = rng.choice([64, 200, 320, 768, 1152, 2048])
        tokens = _log_int(rng, 1, min(262144, 33_000_000 // dim))
        return dict(kind=kind, tokens=tokens, classes=_log_int(rng, 2, 60_000_000 // dim if dim > 320 else 131072), dim=dim,
                    ids=rng.choice(["uniform", "skewed", "padded"]), dtype=rng.choice(["bf16", "f32"]), outdtype=rng.choice(["bf16", "f32"]),
                    scale=rng.choice([1.0, math.sqrt(dim)]), accumulate=kind == "embed_grad" and rng.random() < 0.4)
    tensors, total = _log_int(rng, 1, 1500), _log_int(rng, 1000, 200_000_000)
    return dict(kind="clip", tensors=tensors, largest=_log_int(rng, 500, 8_000_000), total=total, dtype=rng.choice(["bf16", "f32"]),
                outdtype=rng.choice(["bf16", "f32"]), max_norm=rng.choice([0.1, 1.0, 1e6]))


# --------------------------------------------------------------------------------------- what a program has in hand

def _groups(case):
    return -(-case["rows"] // case["group"]) if case["group"] else 1


def _lengths(case):
    """Rows that are there of each group of a padded batch: from none (a dropped caption) to all; the first is full."""
    n = _groups(case)
    return [case["group"] * (n - i) // n for i in range(n)] if n > 1 else [case["group"]]


def _probabilities(case):
    """How often a token takes each id, in order of frequency."""
    V = case["classes"]
    if case["ids"] == "uniform":
        return np.full(V, 1.0 / V)
    p = 1.0 / (np.arange(V) + 10.0)
    return p / p.sum()


def _sizes(case):
    """Elements of the tensors: odd, small and large ones, at most `largest` each and about `total` together."""
    n, most = case["tensors"], case["largest"]
    share = np.random.default_rng(n).dirichlet(np.full(n, 0.7)) * case["total"]
    return [int(min(max(1, round(s)), most)) for s in share]


def _starts(sizes):
    """Where tensors of these sizes begin in one buffer, and its end."""
    return [0] + np.cumsum([-(-n // 8) * 8 for n in sizes]).tolist()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    state = dict(case)
    if case["kind"] in ("norm", "norm_grad"):
        rows, cols, groups = case["rows"], case["cols"], _groups(case)
        xt, ht = DTYPES[case["xdtype"]], DTYPES[case["hdtype"]]
        x, h = randn(rows, cols), randn(rows, cols)
        # a few channels of the residual stream are far larger than the rest, and the stream has a mean
        x[:, torch.randperm(cols, generator=gen, device="cuda")[: max(1, cols // 100)]] *= 12.0
        x += 0.5
        # gate, shift and scale of every sample, slices of one modulation
        mod = 0.3 * randn(groups, 3 * cols)
        order = torch.randperm(groups, generator=gen, device="cuda")
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")[order].contiguous() if case["lens"] else None
        state.update(x=x.to(xt), h=h.to(ht), gate=mod[:, :cols] if case["gate"] else None, bias=mod[:, cols: 2 * cols], weight=mod[:, 2 * cols:],
                     post_weight=1.0 + 0.2 * randn(cols) if case["post"] != "none" else None, lens=lens)
        x = h = None
        if case["kind"] == "norm":
            state.update(x_out=torch.empty((rows, cols), dtype=xt, device="cuda"), y=torch.empty((rows, cols), dtype=ht, device="cuda"),
                         stats=torch.empty((rows, 4), device="cuda"))
            return state
        x_out, _, stats = _gate_norm(state)
        dmod = torch.empty((groups, 3 * cols), device="cuda")
        del state["x"]
        state.update(x_out=x_out, stats=stats, dx_out=randn(rows, cols).to(xt), dy=randn(rows, cols).to(ht),
                     dx=torch.empty((rows, cols), dtype=xt, device="cuda"), dh=torch.empty((rows, cols), dtype=ht, device="cuda"),
                     dgate=dmod[:, :cols] if case["gate"] else None, dbias=dmod[:, cols: 2 * cols], dweight=dmod[:, 2 * cols:],
                     dpost_weight=torch.empty(cols, device="cuda") if case["post"] != "none" else None)
        return state
    if case["kind"] in ("embed", "embed_grad"):
        T, V, dim = case["tokens"], case["classes"], case["dim"]
        cdf = torch.from_numpy(np.cumsum(_probabilities(case))).cuda()
        ids = torch.searchsorted(cdf, torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)).clamp_(0, V - 1)
        ids = torch.randperm(V, generator=gen, device="cuda")[ids]
        if case["ids"] == "padded":                        # captions of up to 77 tokens, the last id behind each
            ends = torch.randint(4, 78, (-(-T // 77), 1), generator=gen, device="cuda")
            ids[(torch.arange(77, device="cuda")[None] >= ends).flatten()[:T]] = V - 1
        table = 0.02 * randn(V, dim)
        state.update(ids=ids.to(torch.int32))
        if case["kind"] == "embed":
            state.update(table=table.to(DTYPES[case["dtype"]]), out=torch.empty((T, dim), dtype=DTYPES[case["outdtype"]], device="cuda"))
        else:
            table = table.to(DTYPES[case["outdtype"]])
            state.update(dout=randn(T, dim).to(DTYPES[case["dtype"]]), before=table if case["accumulate"] else None,
                         dtable=torch.empty_like(table))
        return state
    dt, odt = DTYPES[case["dtype"]], DTYPES[case["outdtype"]]
    # gradients of different layers differ in size
    grads = [torch.randn((n,), generator=gen, device="cuda", dtype=dt).mul_(10.0 ** -(1 + i % 4)) for i, n in enumerate(_sizes(case))]
    # the optimizer's gradients lie in one buffer, each tensor on a multiple of 8 elements
    starts = _starts([g.numel() for g in grads])
    flat = torch.zeros(starts[-1], dtype=odt, device="cuda")
    state.update(grads=grads, flat=flat, outs=[flat[a: a + g.numel()] for a, g in zip(starts, grads)], norm=torch.empty(1, device="cuda"))
    return state


# ----------------------------------------------------------------------------------------------------- plain forms

def _of_rows(s, v):
    """A group's vector for every row (one vector without groups)."""
    return v if s["group"] == 0 else v[torch.arange(s["rows"], device="cuda") // s["group"]]


def _there(s):
    """[rows, 1]: rows inside their group's length."""
    row = torch.arange(s["rows"], device="cuda")
    return (row % s["group"] < s["lens"][row // s["group"]])[:, None]


def _moments(x, norm):
    """Mean and 1 / standard deviation of each row; a norm without a mean takes 0."""
    mean = x.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(x[:, :1])
    return mean, ((x - mean).square().mean(-1, keepdim=True) + EPS).rsqrt()


def _gate_norm(s):
    x, t = s["x"].float(), s["h"].float()
    p_mean, p_inv = torch.zeros_like(x[:, :1]), torch.ones_like(x[:, :1])
    if s["post"] != "none":
        p_mean, p_inv = _moments(t, s["post"])
        t = (t - p_mean) * p_inv * s["post_weight"]
    if s["gate"] is not None:
        t = _of_rows(s, s["gate"]) * t
    x = s["residual"] * x + t
    mean, inv = _moments(x, s["norm"])
    y = (x - mean) * inv * (1.0 + _of_rows(s, s["weight"])) + _of_rows(s, s["bias"])
    stats = torch.cat((mean, inv, p_mean, p_inv), 1)
    if s["lens"] is not None:
        there = _there(s)
        x, y, stats = (torch.where(there, v, torch.zeros_like(v)) for v in (x, y, stats))
    return x.to(s["x"].dtype), y.to(s["h"].dtype), stats


def _centred(g, xh, norm):
    """g without its parts along the row's ones (a norm with a mean) and along xh."""
    less = xh * (g * xh).mean(-1, keepdim=True)
    return g - less - g.mean(-1, keepdim=True) if norm == "layer" else g - less


def _group_sums(s, v):
    if s["group"] == 0:
        return v.sum(0, keepdim=True)
    n, pad = _groups(s), _groups(s) * s["group"] - s["rows"]
    return torch.nn.functional.pad(v, (0, 0, 0, pad)).reshape(n, s["group"], -1).sum(1)


def _gate_norm_grad(s):
    x, h, dy, d = (s[n].float() for n in ("x_out", "h", "dy", "dx_out"))
    mean, inv, p_mean, p_inv = s["stats"].split(1, 1)
    xh = (x - mean) * inv
    d = d + inv * _centred(dy * (1.0 + _of_rows(s, s["weight"])), xh, s["norm"])
    if s["lens"] is not None:
        there = _there(s)
        d, xh, dy, h = (torch.where(there, v, torch.zeros_like(v)) for v in (d, xh, dy, h))
    hh = (h - p_mean) * p_inv if s["post"] != "none" else h
    t = hh * s["post_weight"] if s["post"] != "none" else h
    u = _of_rows(s, s["gate"]) * d if s["gate"] is not None else d
    found = {"dx": (s["residual"] * d).to(s["x_out"].dtype), "dweight": _group_sums(s, dy * xh), "dbias": _group_sums(s, dy)}
    if s["gate"] is not None:
        found["dgate"] = _group_sums(s, d * t)
    if s["post"] != "none":
        found["dpost_weight"] = (u * hh).sum(0)
        u = p_inv * _centred(u * s["post_weight"], hh, s["post"])
    return dict(found, dh=u.to(s["h"].dtype))


def _embed_grad(s):
    dtable = torch.zeros(s["dtable"].shape, device="cuda").index_add_(0, s["ids"], s["dout"].float()) * s["scale"]
    return (dtable if s["before"] is None else dtable + s["before"].float()).to(s["dtable"].dtype)


def _clip(s):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    coefficient = (s["max_norm"] / (norm + EPS)).clamp(max=1.0).float()
    flat = torch.zeros_like(s["flat"])
    for a, g in zip(_starts([g.numel() for g in s["grads"]]), s["grads"]):
        flat[a: a + g.numel()] = (g.float() * coefficient).to(flat.dtype)
    return {"norm": norm.float().reshape(1), "grads": flat}


def _plain(s):
    if s["kind"] == "norm":
        return dict(zip(("x_out", "y", "stats"), _gate_norm(s)))
    if s["kind"] == "norm_grad":
        return _gate_norm_grad(s)
    if s["kind"] == "embed":
        return (s["table"][s["ids"].long()].float() * s["scale"]).to(s["out"].dtype)
    return _embed_grad(s) if s["kind"] == "embed_grad" else _clip(s)


# ----------------------------------------------------------------------------------------------- the framework's calls

def _workspace(s, size, *args):
    """The workspace of these sizes, which a program allocates once."""
    if "workspace" not in s:
        s["workspace"] = torch.empty((max(16, size(*args)),), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own(s):
    from paper_2512_05746_b200 import binding as hq
    norms = {"layer": hq.HQ_NORM_LAYER, "rms": hq.HQ_NORM_RMS, "none": hq.HQ_NORM_NONE}
    if s["kind"] == "norm":
        hq.hq_gate_norm(s["x"], s["h"], s["gate"], s["weight"], s["bias"], s["x_out"], s["y"], s["stats"], rows_per_group=s["group"],
                        lens=s["lens"], post=norms[s["post"]], post_weight=s["post_weight"], norm=norms[s["norm"]], weight_plus=1.0,
                        residual_scale=s["residual"], eps=EPS)
        return {"x_out": s["x_out"], "y": s["y"], "stats": s["stats"]}
    if s["kind"] == "norm_grad":
        ws = _workspace(s, hq.hq_gate_norm_bwd_workspace_size, s["rows"], s["cols"], s["group"])
        hq.hq_gate_norm_bwd(s["x_out"], s["h"], s["stats"], s["gate"], s["weight"], s["dx_out"], s["dy"], s["dx"], s["dh"], s["dgate"],
                            s["dweight"], s["dbias"], ws, rows_per_group=s["group"], lens=s["lens"], post=norms[s["post"]],
                            post_weight=s["post_weight"], dpost_weight=s["dpost_weight"], norm=norms[s["norm"]], weight_plus=1.0,
                            residual_scale=s["residual"])
        names = ["dx", "dweight", "dbias"] + ["dgate"] * (s["gate"] is not None) + ["dpost_weight"] * (s["post"] != "none") + ["dh"]
        return {n: s[n] for n in names}
    if s["kind"] == "embed":
        hq.hq_embedding(s["ids"], s["table"], s["out"], scale=s["scale"])
        return s["out"]
    if s["kind"] == "embed_grad":
        ws = _workspace(s, hq.hq_embedding_bwd_workspace_size, s["tokens"], s["classes"], s["dim"])
        hq.hq_embedding_bwd(s["ids"], s["dout"], s["dtable"], ws, scale=s["scale"], base=s["before"])
        return s["dtable"]
    if "list" not in s:                            # laid out once for tensors that stay where they are
        s["list"] = hq.GradList(s["grads"], s["outs"])
    ws = _workspace(s, hq.hq_grad_workspace_size)
    hq.hq_grad_clip(s["list"], s["max_norm"], s["norm"], ws, eps=EPS)
    return {"norm": s["norm"], "grads": s["flat"]}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work and exactness

def work(case):
    if case["kind"] in ("norm", "norm_grad"):
        cols, sx, sh = case["cols"], SIZES[case["xdtype"]], SIZES[case["hdtype"]]
        rows = case["rows"]
        there = sum(min(n, max(0, rows - i * case["group"])) for i, n in enumerate(_lengths(case))) if case["lens"] else rows
        vectors = 4 * cols * (_groups(case) * (2 + case["gate"]) + (case["post"] != "none")) + (4 * _groups(case) if case["lens"] else 0)
        if case["kind"] == "norm":
            return {"bytes": cols * (there + rows) * (sx + sh) + 16 * rows + vectors, "flops": 16 * there * cols}
        return {"bytes": cols * (2 * there + rows) * (sx + sh) + 16 * there + 2 * vectors, "flops": 30 * there * cols}
    if case["kind"] in ("embed", "embed_grad"):
        T, V, dim, s, so = case["tokens"], case["classes"], case["dim"], SIZES[case["dtype"]], SIZES[case["outdtype"]]
        distinct = int(round(float((1.0 - (1.0 - _probabilities(case)) ** T).sum())))
        if case["kind"] == "embed":
            return {"bytes": 4 * T + s * distinct * dim + so * T * dim, "flops": T * dim}
        return {"bytes": 4 * T + s * T * dim + (2 if case["accumulate"] else 1) * so * V * dim, "flops": T * dim}
    n = sum(_sizes(case))
    return {"bytes": n * (SIZES[case["dtype"]] + SIZES[case["outdtype"]]) + 4, "flops": 3 * n}


def exact(case, seed):
    """From the definitions, in 64 bits, group by group: the gradient of a norm as projections of the row, sums over the tokens of an id as
    differences of running sums over the sorted tokens, the norm of the gradients by torch's vector norm."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["kind"] in ("norm", "norm_grad"):
        rows, cols, step = case["rows"], case["cols"], case["group"] or case["rows"]
        names = ("x_out", "y", "stats") if case["kind"] == "norm" else ("dx", "dh")
        found = {n: torch.zeros(((rows, 4) if n == "stats" else (rows, cols)), dtype=f64, device="cuda") for n in names}
        sums = {n: torch.zeros((_groups(case), cols), dtype=f64, device="cuda") for n in ("dgate", "dweight", "dbias", "dpost_weight")}
        pw = None if s["post_weight"] is None else s["post_weight"].to(f64)
        if _groups(case) > 40000:                          # taken one by one below
            return None
        lens = s["lens"].tolist() if case["lens"] else None
        one = torch.ones(cols, dtype=f64, device="cuda") / math.sqrt(cols)
        for g, first in enumerate(range(0, rows, step)):
            n = min(step, rows - first, lens[g] if lens else rows)
            if n == 0:
                continue
            at = slice(first, first + n)
            gate = 1.0 if s["gate"] is None else s["gate"][g].to(f64)
            gain = s["weight"][g].to(f64) + 1.0
            h = s["h"][at].to(f64)
            if case["kind"] == "norm":
                p_mean, p_inv = torch.zeros((n, 1), dtype=f64, device="cuda"), torch.ones((n, 1), dtype=f64, device="cuda")
                if case["post"] != "none":
                    p_mean = h.sum(1, keepdim=True) / cols if case["post"] == "layer" else p_mean
                    p_inv = 1.0 / torch.sqrt(torch.linalg.vector_norm(h - p_mean, dim=1, keepdim=True) ** 2 / cols + EPS)
                    h = (h - p_mean) * (p_inv * pw)
                z = torch.addcmul(s["x"][at].to(f64) * case["residual"], h, gate * torch.ones(cols, dtype=f64, device="cuda"))
                mean = z.sum(1, keepdim=True) / cols if case["norm"] == "layer" else torch.zeros((n, 1), dtype=f64, device="cuda")
                inv = 1.0 / torch.sqrt(torch.linalg.vector_norm(z - mean, dim=1, keepdim=True) ** 2 / cols + EPS)
                found["x_out"][at] = z
                found["y"][at] = s["bias"][g].to(f64) + gain * inv * (z - mean)
                found["stats"][at] = torch.cat((mean, inv, p_mean, p_inv), 1)
                continue
            mean, inv, p_mean, p_inv = s["stats"][at].to(f64).split(1, 1)
            dy, axis = s["dy"][at].to(f64), (s["x_out"][at].to(f64) - mean) * inv
            v = dy * gain
            less = axis * (torch.einsum("rc,rc->r", v, axis)[:, None] / cols)
            v = v - less - (torch.outer(v @ one, one) if case["norm"] == "layer" else 0.0)
            d = s["dx_out"][at].to(f64) + inv * v
            found["dx"][at] = case["residual"] * d
            sums["dweight"][g], sums["dbias"][g] = torch.einsum("rc,rc->c", dy, axis), dy.sum(0)
            if case["post"] == "none":
                sums["dgate"][g], found["dh"][at] = torch.einsum("rc,rc->c", d, h), d * gate
                continue
            axis = (h - p_mean) * p_inv
            sums["dgate"][g], sums["dpost_weight"][g] = torch.einsum("rc,rc->c", d, axis) * pw, torch.einsum("rc,rc->c", d, axis) * gate
            v = d * (gate * pw)
            less = axis * (torch.einsum("rc,rc->r", v, axis)[:, None] / cols)
            found["dh"][at] = p_inv * (v - less - (torch.outer(v @ one, one) if case["post"] == "layer" else 0.0))
        if case["kind"] == "norm":
            return found
        answer = {"dx": found["dx"], "dweight": sums["dweight"], "dbias": sums["dbias"]}
        if case["gate"]:
            answer["dgate"] = sums["dgate"]
        if case["post"] != "none":
            answer["dpost_weight"] = sums["dpost_weight"].sum(0)
        return dict(answer, dh=found["dh"])
    if case["kind"] == "embed":
        return torch.nn.functional.embedding(s["ids"].long(), s["table"].to(f64)) * case["scale"]
    if case["kind"] == "embed_grad":
        order = torch.argsort(s["ids"], stable=True)
        ids, counts = torch.unique_consecutive(s["ids"][order], return_counts=True)
        ends = counts.cumsum(0)
        table = torch.zeros(s["dtable"].shape, dtype=f64, device="cuda") if s["before"] is None else s["before"].to(f64).clone()
        for c in range(0, case["dim"], 64):                # differences of running sums, some columns at a time
            run_sum = torch.nn.functional.pad(s["dout"][:, c: c + 64].to(f64)[order].cumsum(0), (0, 0, 1, 0))
            table[ids.long(), c: c + 64] += (run_sum[ends] - run_sum[ends - counts]) * case["scale"]
        return table
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g, dtype=f64) for g in s["grads"]]))
    factor = min(1.0, case["max_norm"] / (float(norm) + EPS))
    return {"norm": norm.reshape(1), "grads": torch.cat([torch.nn.functional.pad(g, (0, -g.numel() % 8)).to(f64) * factor for g in s["grads"]])}
