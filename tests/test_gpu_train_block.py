"""The operators around a transformer block's linears as a training step runs them: one step against 64-bit differentiation, other streams,
captured graphs, calls that overlap, offsets beyond 2^31."""
import math

import pytest
import torch

from train_block_reference import F32, backward, embedding_grad, forward, unit

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


def reference_step(p, labels, x, target, attention, Nb, heads):
    """Loss and gradients of the step in 64 bits by torch's differentiation."""
    p = {n: v.double().requires_grad_() for n, v in p.items()}
    C, rows = x.shape[1], x.shape[0]
    mod = (p["table"][labels.long()] * 1.5) @ p["w_mod"]
    each = lambda i: mod[:, i * C: (i + 1) * C].repeat_interleave(rows // Nb, 0)  # noqa: E731
    ln = lambda v: (v - v.mean(-1, keepdim=True)) / (v.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()  # noqa: E731
    rms = lambda v: v / (v.square().mean(-1, keepdim=True) + EPS).sqrt()  # noqa: E731
    x = x.double().requires_grad_()
    qkv = (ln(x) * (1 + each(0)) + each(1)) @ p["w_qkv"]
    if attention:
        q, k, v = (t.reshape(Nb, -1, heads, C // heads).transpose(1, 2) for t in qkv.split(C, 1))
        o = (torch.softmax(q @ k.transpose(-1, -2) / math.sqrt(C // heads), -1) @ v).transpose(1, 2).reshape(rows, C)
    else:
        o = qkv[:, :C] * qkv[:, C: 2 * C] + qkv[:, 2 * C:]
    x1 = x + each(2) * (o @ p["w_o"])
    h = torch.nn.functional.silu((ln(x1) * (1 + each(3)) + each(4)) @ p["w_1"]) @ p["w_2"]
    x2 = x1 + each(5) * (rms(h) * p["post"])
    loss = (x2 * target.double()).sum()
    return loss.detach(), dict(zip(list(p) + ["x"], torch.autograd.grad(loss, list(p.values()) + [x])))


def step(hq, p, labels, x, target, attention, Nb, heads):
    """The same with the library's operators in fp32 around torch's products, attention in bf16."""
    rows, C = x.shape
    per, new = rows // Nb, lambda *s, t=F: torch.empty(s, dtype=t, device="cuda")
    cond = new(Nb, C)
    hq.hq_embedding(labels, p["table"], cond, scale=1.5)
    mod = cond @ p["w_mod"]
    part = lambda m, i: m[:, i * C: (i + 1) * C]  # noqa: E731
    y0, s0 = new(rows, C), new(rows, 4)
    hq.hq_gate_norm(x, None, None, part(mod, 0), part(mod, 1), None, y0, s0, rows_per_group=per, weight_plus=1.0)
    qkv = y0 @ p["w_qkv"]
    if attention:
        b = qkv.to(BF)
        o, lse = new(rows, C, t=BF), new(Nb, heads, per)
        q, k, v = b[:, :C], b[:, C: 2 * C], b[:, 2 * C:]
        hq.hq_attention_fwd(q, k, v, Nb, heads, heads, o, lse)
        of = o.float()
    else:
        q, k, v = (qkv[:, i * C: (i + 1) * C] for i in range(3))
        of = q * k + v
    h1, x1, y1, s1 = of @ p["w_o"], new(rows, C), new(rows, C), new(rows, 4)
    hq.hq_gate_norm(x, h1, part(mod, 2), part(mod, 3), part(mod, 4), x1, y1, s1, rows_per_group=per, weight_plus=1.0)
    z = y1 @ p["w_1"]
    a = torch.nn.functional.silu(z)
    h2, x2, s2 = a @ p["w_2"], new(rows, C), new(rows, 4)
    hq.hq_gate_norm(x1, h2, part(mod, 5), None, None, x2, None, s2, rows_per_group=per, post=hq.HQ_NORM_RMS, post_weight=p["post"], norm=hq.HQ_NORM_NONE)
    # backward
    ws = new(hq.hq_gate_norm_bwd_workspace_size(rows, C, per), t=torch.uint8)
    g = {n: new(*v.shape) for n, v in p.items()}
    dmod, dh2, dx = new(Nb, 6 * C), new(rows, C), target.clone()
    hq.hq_gate_norm_bwd(None, h2, s2, part(mod, 5), None, dx, None, dx, dh2, part(dmod, 5), None, None, ws, rows_per_group=per, post=hq.HQ_NORM_RMS,
                        post_weight=p["post"], dpost_weight=g["post"], norm=hq.HQ_NORM_NONE)
    g["w_2"] = a.t() @ dh2
    sig = torch.sigmoid(z)
    dz = (dh2 @ p["w_2"].t()) * (sig * (1 + z * (1 - sig)))
    g["w_1"] = y1.t() @ dz
    dh1 = new(rows, C)
    hq.hq_gate_norm_bwd(x1, h1, s1, part(mod, 2), part(mod, 3), dx, dz @ p["w_1"].t(), dx, dh1, part(dmod, 2), part(dmod, 3), part(dmod, 4), ws,
                        rows_per_group=per, weight_plus=1.0)
    g["w_o"] = of.t() @ dh1
    do = dh1 @ p["w_o"].t()
    if attention:
        dqkv = new(rows, 3 * C, t=BF)
        aws = new(hq.hq_attention_bwd_workspace_size(Nb, per, per, heads, heads, C // heads), t=torch.uint8)
        hq.hq_attention_bwd(q, k, v, o, lse, do.to(BF), Nb, heads, heads, dqkv[:, :C], dqkv[:, C: 2 * C], dqkv[:, 2 * C:], aws)
        dqkv = dqkv.float()
    else:
        dqkv = torch.cat((do * k, do * q, do), 1)
    g["w_qkv"] = y0.t() @ dqkv
    hq.hq_gate_norm_bwd(x, None, s0, None, part(mod, 0), dx, dqkv @ p["w_qkv"].t(), dx, None, None, part(dmod, 0), part(dmod, 1), ws, rows_per_group=per,
                        weight_plus=1.0)
    g["w_mod"] = cond.t() @ dmod
    ews = new(hq.hq_embedding_bwd_workspace_size(Nb, p["table"].shape[0], C), t=torch.uint8)
    hq.hq_embedding_bwd(labels, dmod @ p["w_mod"].t(), g["table"], ews, scale=1.5)
    return (x2.double() * target.double()).sum(), dict(g, x=dx)


@pytest.mark.parametrize("attention", [False, True])
def test_a_step(hq, attention):
    """Without attention every rounding is fp32's, and every product (of at most 128 terms) is summed in fp32 or better with torch's default;
    a gradient passes some 40 operations: 2^-24 x 128 x 40 of its norm bounds them with room.  With attention some ten roundings to bf16 stand
    between a parameter and the loss and back (q k v, the weights twice, the output, its gradient, dS, dq dk dv): 2^-8 each, all in one
    direction."""
    torch.backends.cuda.matmul.allow_tf32 = False
    gen = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    Nb, per, C, heads = 3, 20, 64, 2
    p = dict(table=rand(11, C), w_mod=0.05 * rand(C, 6 * C), w_qkv=rand(C, 3 * C) / 8, w_o=rand(C, C) / 8, w_1=rand(C, 2 * C) / 8, w_2=rand(2 * C, C) / 11,
             post=1 + 0.2 * rand(C))
    labels = torch.tensor([7, 2, 7], dtype=torch.int32, device="cuda")
    x, target = rand(Nb * per, C), rand(Nb * per, C)
    loss, want = reference_step(p, labels, x, target, attention, Nb, heads)
    got_loss, got = step(hq, p, labels, x, target, attention, Nb, heads)
    tolerance = 10 * unit(BF) if attention else 128 * 40 * F32
    assert set(got) == set(want)
    for name, w in want.items():
        assert float((got[name].double() - w).norm()) <= tolerance * float(w.norm()), name
    assert abs(float(got_loss - loss)) <= tolerance * float(x.norm() * target.norm())
    # and the step's clipping
    grads = [got[n] for n in p]
    total = math.sqrt(sum(float(v.double().square().sum()) for v in grads))
    before = [v.clone() for v in grads]
    norm, ws = torch.empty(1, device="cuda"), torch.empty((hq.hq_grad_workspace_size(),), dtype=torch.uint8, device="cuda")
    hq.hq_grad_clip(grads, 0.5 * total, norm, ws, eps=0.0)
    assert abs(float(norm) - total) <= 8 * F32 * total
    for b, v in zip(before, grads):
        assert bool(((v.double() - 0.5 * b.double()).abs() <= 12 * F32 * b.double().abs()).all())


class Calls:
    """One call of everything on buffers of its own; run() writes them, results() copies them."""

    def __init__(self, hq, seed, rows=900, cols=512, per=128, tokens=700):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
        self.hq, self.per, groups = hq, per, -(-rows // per)
        new = lambda *s, t=F: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
        self.x, self.h, self.mod, self.pw = rand(rows, cols), rand(rows, cols).to(BF), 0.3 * rand(groups, 3 * cols), 1 + 0.2 * rand(cols)
        self.cols, self.x_out, self.y, self.stats = cols, new(rows, cols), new(rows, cols, t=BF), new(rows, 4)
        self.dxo, self.dy = rand(rows, cols), rand(rows, cols).to(BF)
        self.dx, self.dh, self.dmod, self.dpw = new(rows, cols), new(rows, cols, t=BF), new(groups, 3 * cols), new(cols)
        self.ws = [new(n, t=torch.uint8) for n in (hq.hq_gate_norm_bwd_workspace_size(rows, cols, per), hq.hq_embedding_bwd_workspace_size(tokens, 50, cols),
                                                   hq.hq_grad_workspace_size())]
        self.ids = torch.randint(0, 50, (tokens,), generator=gen, device="cuda").to(torch.int32)
        self.table, self.emb, self.dtable = rand(50, cols), new(tokens, cols), new(50, cols)
        self.clipped = [new(50, cols), new(groups, 3 * cols), new(cols)]
        self.list, self.norm = hq.GradList([self.dtable, self.dmod, self.dpw], self.clipped), new(1)

    def run(self, stream=None):
        hq, c = self.hq, self.cols
        kw = dict(rows_per_group=self.per, post=hq.HQ_NORM_LAYER, post_weight=self.pw, weight_plus=1.0, stream=stream)
        part = lambda m: (m[:, :c], m[:, c: 2 * c], m[:, 2 * c:])  # noqa: E731
        gate, weight, bias = part(self.mod)
        hq.hq_gate_norm(self.x, self.h, gate, weight, bias, self.x_out, self.y, self.stats, **kw)
        hq.hq_gate_norm_bwd(self.x_out, self.h, self.stats, gate, weight, self.dxo, self.dy, self.dx, self.dh, *part(self.dmod), self.ws[0], dpost_weight=self.dpw, **kw)
        hq.hq_embedding(self.ids, self.table, self.emb, scale=2.0, stream=stream)
        hq.hq_embedding_bwd(self.ids, self.emb, self.dtable, self.ws[1], scale=2.0, stream=stream)
        hq.hq_grad_clip(self.list, 1.0, self.norm, self.ws[2], stream=stream)

    def results(self):
        return [t.clone() for t in [self.x_out, self.y, self.stats, self.dx, self.dh, self.dmod, self.dpw, self.emb, self.dtable, self.norm] + self.clipped]


def same(a, b):
    return all(torch.equal(s, t) for s, t in zip(a, b))


def test_other_streams_and_overlapping_calls(hq):
    alone = []
    for seed in range(4):
        c = Calls(hq, seed)
        c.run()
        alone.append(c.results())
    torch.cuda.synchronize()
    calls, streams = [Calls(hq, seed) for seed in range(4)], [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            c.run(stream=s)                        # given
    torch.cuda.synchronize()
    assert all(same(c.results(), a) for c, a in zip(calls, alone))
    calls = [Calls(hq, seed) for seed in range(4)]
    torch.cuda.synchronize()
    for c, s in zip(calls, streams):
        with torch.cuda.stream(s):                 # the current one
            c.run()
    torch.cuda.synchronize()
    assert all(same(c.results(), a) for c, a in zip(calls, alone))


def test_captured_and_replayed(hq):
    """Two graphs, each with buffers and workspaces of its own, replayed on two streams at once with other inputs."""
    fresh = []
    for seed in (10, 11):
        c = Calls(hq, seed)
        c.run()
        fresh.append((c, c.results()))
    graphs, calls = [], [Calls(hq, seed) for seed in (0, 1)]
    for c in calls:
        c.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
        graphs.append(g)
    for c, (other, _) in zip(calls, fresh):
        for name in ("x", "h", "mod", "pw", "dxo", "dy", "ids", "table"):
            getattr(c, name).copy_(getattr(other, name))
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(same(c.results(), want) for c, (_, want) in zip(calls, fresh))


def test_one_workspace_for_calls_one_after_the_other(hq):
    ws = torch.empty((max(hq.hq_embedding_bwd_workspace_size(5000, 3000, 1152), hq.hq_gate_norm_bwd_workspace_size(5000, 1152, 0)),), dtype=torch.uint8, device="cuda")
    for seed, sizes in enumerate([(900, 512, 128, 700), (30, 1152, 7, 5000), (5000, 64, 1, 10), (900, 512, 128, 700)]):
        rows, cols, per, tokens = sizes
        a, b = Calls(hq, seed, rows, cols, per, tokens), Calls(hq, seed, rows, cols, per, tokens)
        a.run()
        b.ws[0] = b.ws[1] = ws
        b.run()
        assert same(a.results(), b.results())


def test_offsets_beyond_32_bits(hq):
    """Matrices whose last rows lie more than 2^31 elements (2^32 bytes) behind their first."""
    rows, ld, cols, per = 540_000, 4096, 64, 1000
    big = torch.empty((rows, ld), dtype=BF, device="cuda")
    for t in (big[:, :cols], big[:, 1024: 1024 + cols], big[:, 2048: 2048 + cols], big[:, 3000: 3000 + cols]):
        t.copy_(torch.randn((rows, cols), device="cuda"))
    x, h, dxo, dy = big[:, :cols], big[:, 1024: 1024 + cols], big[:, 2048: 2048 + cols], big[:, 3000: 3000 + cols]
    mod = 0.3 * torch.randn((rows // per, 3 * cols), device="cuda")
    gate, weight, bias = mod[:, :cols], mod[:, cols: 2 * cols], mod[:, 2 * cols:]
    x_out, y, stats = big[:, 512: 512 + cols], big[:, 600: 600 + cols], torch.empty((rows, 4), device="cuda")
    kw = dict(rows_per_group=per, weight_plus=1.0)
    hq.hq_gate_norm(x, h, gate, weight, bias, x_out, y, stats, **kw)
    dmod, ws = torch.empty_like(mod), torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")
    dx, dh = big[:, 704: 704 + cols], big[:, 800: 800 + cols]
    hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, dxo, dy, dx, dh, dmod[:, :cols], dmod[:, cols: 2 * cols], dmod[:, 2 * cols:], ws, **kw)
    for at in (slice(0, 2 * per), slice(rows - 2 * per, rows)):
        g = slice(at.start // per, at.stop // per)
        want = forward(x[at].double(), h[at].double(), gate[g], weight[g], bias[g], per, plus=1.0)
        assert bool(((y[at].double() - want[1]).abs() <= unit(BF) * want[1].abs() + 128 * F32 * want[4]).all())
        found = backward(x_out[at].double(), h[at].double(), stats[at], gate[g], weight[g], dxo[at].double(), dy[at].double(), per, plus=1.0)
        for name, got in (("dx", dx[at]), ("dh", dh[at]), ("dgate", dmod[g, :cols]), ("dweight", dmod[g, cols: 2 * cols])):
            ref, size = found[name]
            assert bool(((got.double() - ref).abs() <= unit(got.dtype) * ref.abs() + 256 * F32 * size).all()), name
    del x, h, dxo, dy, x_out, y, dx, dh
    # the same memory as a table and as tokens' rows
    V, dim = rows, 128
    table = big[:, :dim]
    ids = torch.randint(0, V, (3000,), device="cuda")
    ids[:2], ids[-1] = torch.tensor([V - 1, 0], device="cuda"), V - 1
    out = torch.empty((3000, dim), dtype=BF, device="cuda")
    hq.hq_embedding(ids, table, out)
    assert torch.equal(out, table[ids])
    dout = torch.randint(-4, 5, (3000, dim), device="cuda").to(BF)
    ews = torch.empty((hq.hq_embedding_bwd_workspace_size(3000, V, dim),), dtype=torch.uint8, device="cuda")
    hq.hq_embedding_bwd(ids, dout, big[:, 1024: 1024 + dim], ews)
    assert torch.equal(big[:, 1024: 1024 + dim].double(), embedding_grad(ids, dout, V, 1.0)[0])
    tokens = torch.randint(0, 9, (V,), device="cuda").to(torch.int32)
    rows_of = big[:, 2048: 2048 + dim]
    rows_of.copy_(torch.randint(-2, 3, (V, dim), device="cuda"))
    dtable = torch.empty((9, dim), device="cuda")
    ews = torch.empty((hq.hq_embedding_bwd_workspace_size(V, 9, dim),), dtype=torch.uint8, device="cuda")
    hq.hq_embedding_bwd(tokens, rows_of, dtable, ews)
    assert torch.equal(dtable.double(), embedding_grad(tokens, rows_of, 9, 1.0)[0])
    del table, rows_of
    flat = big.view(-1)                            # 2.2 G gradients
    flat.fill_(0.5)
    norm, gws = torch.empty(1, device="cuda"), torch.empty((hq.hq_grad_workspace_size(),), dtype=torch.uint8, device="cuda")
    hq.hq_grad_clip([flat], 1.0, norm, gws, eps=0.0)
    want = 0.5 * math.sqrt(flat.numel())
    assert abs(float(norm) - want) <= 8 * F32 * want
    value = torch.tensor(0.5 / want).to(BF).cuda()
    assert bool((flat[:100] == value).all()) and bool((flat[-100:] == value).all()) and bool((flat[2 ** 31 - 50: 2 ** 31 + 50] == value).all())


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_ids_off_the_16_byte_border(hq, shift):
    for dtype in (torch.int32, torch.int64):
        ids = torch.randint(0, 40, (5000 + shift,), device="cuda").to(dtype)[shift:]
        dout = torch.randint(-4, 5, (5000, 64), device="cuda").to(BF)
        dtable = torch.empty((40, 64), device="cuda")
        ws = torch.empty((hq.hq_embedding_bwd_workspace_size(5000, 40, 64),), dtype=torch.uint8, device="cuda")
        hq.hq_embedding_bwd(ids, dout, dtable, ws)
        assert torch.equal(dtable.double(), embedding_grad(ids, dout, 40, 1.0)[0])
