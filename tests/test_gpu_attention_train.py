"""Attention with its row statistic, and its gradient, against 64-bit arithmetic with element-wise bounds: lengths around the tile
edges, widths that do not fill them, shared heads, causal masks that leave rows empty, padded batches with anything behind the
lengths, pitches, streams, captured graphs, and the same bits on every run."""
import math

import pytest
import torch

from attention_train_reference import backward, forward, visible

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


def make(seed, Nb, Lq, Lk, H, G, dh, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda rows, heads, m=1.0: (m * torch.randn((rows, heads * dh), generator=gen, device="cuda")).to(BF)  # noqa: E731
    return r(Nb * Lq, H, scale), r(Nb * Lk, G), r(Nb * Lk, G), r(Nb * Lq, H)


def workspace(n):
    return torch.empty((max(16, n),), dtype=torch.uint8, device="cuda").fill_(0xFF)      # NaN, should anything read before it writes


def fwd(hq, q, k, v, Nb, H, G, **kw):
    Lq, Lk, dh = q.shape[0] // Nb, k.shape[0] // Nb, q.shape[1] // H
    out, lse = torch.full((Nb * Lq, H * dh), math.nan, dtype=BF, device="cuda"), torch.full((Nb, H, Lq), math.nan, device="cuda")
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ws = workspace(hq.hq_attention_fwd_workspace_size(Nb, Lq, Lk, H, G, dh))
    torch.cuda.synchronize()                     # the call may run on another stream than the fills
    hq.hq_attention_fwd(q, k, v, Nb, H, G, out, lse, ws, dev_status=status, **kw)
    torch.cuda.synchronize()
    hq.hq_check_status(status)
    return out, lse


def bwd(hq, q, k, v, out, lse, dout, Nb, H, G, **kw):
    Lq, Lk, dh = q.shape[0] // Nb, k.shape[0] // Nb, q.shape[1] // H
    grads = [torch.full((Nb * L, h * dh), math.nan, dtype=BF, device="cuda") for L, h in ((Lq, H), (Lk, G), (Lk, G))]
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    ws = workspace(hq.hq_attention_bwd_workspace_size(Nb, Lq, Lk, H, G, dh))
    torch.cuda.synchronize()
    hq.hq_attention_bwd(q, k, v, out, lse, dout, Nb, H, G, *grads, ws, dev_status=status, **kw)
    torch.cuda.synchronize()
    hq.hq_check_status(status)
    return grads


def within(got, want, bound, what):
    diff = (got.double() - want).abs()
    worst = (diff / bound).max().item()
    assert bool(torch.isfinite(got.float()).all()), what
    assert worst <= 1.0, (what, worst, diff.max().item())


def check(hq, q, k, v, dout, Nb, H, G, causal=False, q_lens=None, k_lens=None, scale=None):
    dh = q.shape[1] // H
    sc = dh ** -0.5 if scale is None else scale
    kw = dict(causal=causal, q_lens=q_lens, k_lens=k_lens)
    out, lse = fwd(hq, q, k, v, Nb, H, G, scale=scale, **kw)
    want, want_lse, bound, lse_bound = forward(q, k, v, Nb, H, G, sc, **kw)
    within(out, want, bound, "out")
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert bool(((lse.double() - want_lse).abs() <= lse_bound)[~empty].all())
    grads = bwd(hq, q, k, v, out, lse, dout, Nb, H, G, scale=scale, **kw)
    wants, bounds = backward(q, k, v, out, lse, dout, Nb, H, G, sc, **kw)
    for name, got, w, b in zip(("dq", "dk", "dv"), grads, wants, bounds):
        within(got, w, b, name)
    return out, lse, grads


SHAPES = [                                       # Nb, Lq, Lk, heads, kv_heads, dh
    (1, 1, 1, 1, 1, 8), (2, 1, 300, 2, 1, 64), (1, 300, 1, 2, 2, 64), (2, 64, 64, 2, 2, 64), (1, 127, 129, 2, 2, 40),
    (1, 128, 128, 1, 1, 128), (2, 129, 127, 3, 3, 72), (1, 256, 256, 2, 2, 96), (1, 257, 385, 4, 2, 128), (2, 200, 77, 6, 1, 80),
    (1, 513, 640, 2, 2, 32), (1, 640, 513, 2, 1, 48), (3, 65, 191, 2, 2, 56), (1, 383, 130, 2, 1, 120), (1, 1100, 900, 1, 1, 64),
    (1, 2000, 60, 2, 1, 64), (1, 40, 2000, 2, 1, 96), (1, 2100, 150, 2, 1, 128), (2, 1111, 200, 4, 1, 72)]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(hq, shape, causal):
    Nb, Lq, Lk, H, G, dh = shape
    q, k, v, dout = make(Lq * 7 + Lk + dh, *shape)
    check(hq, q, k, v, dout, Nb, H, G, causal=causal)


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_scale_and_peaked_rows(hq, scale):
    q, k, v, dout = make(5, 1, 260, 300, 2, 2, 64, scale=3.0)
    check(hq, q, k, v, dout, 1, 2, 2, scale=scale)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dh,H,G", [(64, 2, 1), (72, 2, 2), (128, 2, 1)])
@pytest.mark.parametrize("garbage", [math.nan, math.inf])
@pytest.mark.parametrize("Lq,Lk", [(260, 300), (250, 100), (2100, 140)])
def test_padded_batch(hq, causal, dh, H, G, garbage, Lq, Lk):
    """Lengths of 0, 1, around the tiles' edges and beyond the matrix (clamped); what lies behind them is never read into a result."""
    ql = torch.tensor([Lq, 0, 1, 128, 129, Lq - 5, 100, 9999, Lq], dtype=torch.int32, device="cuda")
    kl = torch.tensor([Lk, 50, 0, min(129, Lk), min(128, Lk - 1), 1, Lk - 1, 9999, -3], dtype=torch.int32, device="cuda")
    Nb = ql.numel()
    q, k, v, dout = make(11 + dh, Nb, Lq, Lk, H, G, dh)
    clean = check(hq, q, k, v, dout, Nb, H, G, causal=causal, q_lens=ql, k_lens=kl)
    iq, ik = torch.arange(Lq, device="cuda")[None], torch.arange(Lk, device="cuda")[None]
    dead_q, dead_k = (iq >= ql.clamp(0, Lq)[:, None]).flatten(), (ik >= kl.clamp(0, Lk)[:, None]).flatten()
    for t, dead in ((q, dead_q), (dout, dead_q), (k, dead_k), (v, dead_k)):
        t[dead] = garbage
    kw = dict(causal=causal, q_lens=ql, k_lens=kl)
    out, lse = fwd(hq, q, k, v, Nb, H, G, **kw)
    grads = bwd(hq, q, k, v, out, lse, dout, Nb, H, G, **kw)
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
    for got, want, dead in zip(grads, clean[2], (dead_q, dead_k, dead_k)):
        assert torch.equal(got, want)
        assert not got[dead].any()


def test_causal_rows_without_keys(hq):
    """More queries than keys under the causal mask: the first queries see nothing, and what they hold has no part."""
    Nb, Lq, Lk, H, G, dh = 2, 300, 130, 2, 1, 64
    q, k, v, dout = make(3, Nb, Lq, Lk, H, G, dh)
    out, lse, grads = check(hq, q, k, v, dout, Nb, H, G, causal=True)
    blind = (torch.arange(Lq, device="cuda") < Lq - Lk).repeat(Nb)
    assert not out[blind].any() and bool((lse[:, :, : Lq - Lk] == -math.inf).all()) and not grads[0][blind].any()
    q[blind], dout[blind] = math.nan, math.inf
    out2, lse2 = fwd(hq, q, k, v, Nb, H, G, causal=True)
    again = bwd(hq, q, k, v, out2, lse2, dout, Nb, H, G, causal=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and all(torch.equal(a, b) for a, b in zip(grads, again))


def test_slices_of_a_fused_projection(hq):
    """Queries, keys and values as columns of one matrix, gradients into the columns of another; what lies beside them stays."""
    Nb, L, H, G, dh = 2, 200, 4, 2, 48
    width = (H + 2 * G) * dh + 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn((Nb * L, width), generator=gen, device="cuda").to(BF)
    cut = (slice(0, H * dh), slice(H * dh, (H + G) * dh), slice((H + G) * dh, (H + 2 * G) * dh))
    q, k, v = (qkv[:, c] for c in cut)
    dout = torch.randn((Nb * L, H * dh), generator=gen, device="cuda").to(BF)
    out, lse, grads = check(hq, q.contiguous(), k.contiguous(), v.contiguous(), dout, Nb, H, G)
    wide_out, wide_lse = torch.full((Nb * L, H * dh + 8), 7.0, dtype=BF, device="cuda"), torch.empty((Nb, H, L), device="cuda")
    hq.hq_attention_fwd(q, k, v, Nb, H, G, wide_out[:, : H * dh], wide_lse, workspace(hq.hq_attention_fwd_workspace_size(Nb, L, L, H, G, dh)))
    assert torch.equal(wide_out[:, : H * dh], out) and bool((wide_out[:, H * dh:] == 7).all()) and torch.equal(wide_lse, lse)
    dqkv = torch.full((Nb * L, width), 7.0, dtype=BF, device="cuda")
    ws = workspace(hq.hq_attention_bwd_workspace_size(Nb, L, L, H, G, dh))
    hq.hq_attention_bwd(q, k, v, wide_out[:, : H * dh], wide_lse, dout, Nb, H, G, *(dqkv[:, c] for c in cut), ws)
    for c, g in zip(cut, grads):
        assert torch.equal(dqkv[:, c], g)
    assert bool((dqkv[:, -16:] == 7).all())


def test_against_differences(hq):
    """The kernels' gradients along random directions against central differences of the 64-bit forward."""
    Nb, Lq, Lk, H, G, dh = 2, 150, 140, 4, 2, 40
    q, k, v, dout = make(21, Nb, Lq, Lk, H, G, dh)
    sc = dh ** -0.5
    out, lse = fwd(hq, q, k, v, Nb, H, G, causal=True)
    grads = bwd(hq, q, k, v, out, lse, dout, Nb, H, G, causal=True)
    exact_out, exact_lse, _, _ = forward(q, k, v, Nb, H, G, sc, causal=True)
    # D comes from the rounded out: how far that moves the gradient is what the formula gives with either
    rounded, bounds = backward(q, k, v, out, lse, dout, Nb, H, G, sc, causal=True)
    true, _ = backward(q, k, v, exact_out, exact_lse, dout, Nb, H, G, sc, causal=True)
    loss = lambda *t: (forward(*t, Nb, H, G, sc, causal=True)[0] * dout.double()).sum()  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = 1e-5
    for which in range(3):
        base = [t.double() for t in (q, k, v)]
        d = torch.randn(base[which].shape, generator=gen, device="cuda", dtype=torch.float64)
        lo, hi = list(base), list(base)
        lo[which], hi[which] = base[which] - h * d, base[which] + h * d
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        got = (grads[which].double() * d).sum()
        allowed = (bounds[which] * d.abs()).sum() + ((rounded[which] - true[which]).abs() * d.abs()).sum() + 1e-6 * slope.abs() + 1e-6
        assert abs(got - slope) <= allowed, which
        assert abs((true[which] * d).sum() - slope) <= 1e-6 * (1 + slope.abs() + (true[which] * d).abs().sum()), which


@pytest.mark.parametrize("dh,L,Lk", [(64, 700, 700), (128, 700, 700), (64, 700, 90), (64, 1500, 90), (128, 1500, 200)])
def test_same_bits_on_every_run_and_stream(hq, dh, L, Lk):
    Nb, H, G = 2, 4, 2
    q, k, v, dout = make(9, Nb, L, Lk, H, G, dh)
    out, lse = fwd(hq, q, k, v, Nb, H, G, causal=True)
    first = bwd(hq, q, k, v, out, lse, dout, Nb, H, G, causal=True)
    side = torch.cuda.Stream()
    for stream in (None, side, side, None):
        o, l = fwd(hq, q, k, v, Nb, H, G, causal=True, stream=stream)
        again = bwd(hq, q, k, v, o, l, dout, Nb, H, G, causal=True, stream=stream)
        assert torch.equal(o, out) and torch.equal(l, lse)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_calls_that_overlap(hq):
    """Training steps of four widths at the same time, each on a stream and a workspace of its own: the bits of the calls one by one."""
    steps = []
    for seed, (Nb, L, Lk, H, G, dh) in enumerate([(4, 500, 500, 8, 8, 64), (2, 700, 700, 8, 2, 128), (8, 900, 77, 4, 4, 40), (3, 300, 300, 6, 3, 72)]):
        q, k, v, dout = make(50 + seed, Nb, L, Lk, H, G, dh)
        out, lse = fwd(hq, q, k, v, Nb, H, G, causal=True)
        want = [out, lse, *bwd(hq, q, k, v, out, lse, dout, Nb, H, G, causal=True)]
        got = [torch.full_like(t, math.nan) for t in want]
        ws = workspace(hq.hq_attention_bwd_workspace_size(Nb, L, Lk, H, G, dh))
        steps.append((q, k, v, dout, Nb, H, G, want, got, ws, torch.zeros((1,), dtype=torch.int32, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for q, k, v, dout, Nb, H, G, want, got, ws, status, stream in steps:
            hq.hq_attention_fwd(q, k, v, Nb, H, G, got[0], got[1], causal=True, dev_status=status, stream=stream)
            hq.hq_attention_bwd(q, k, v, got[0], got[1], dout, Nb, H, G, *got[2:], ws, causal=True, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    for *_, want, got, ws, status, stream in steps:
        hq.hq_check_status(status)
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("Lk", [190, 100])
def test_captured_and_replayed(hq, Lk):
    """A forward and backward pass in one graph, replayed on inputs and lengths that change in place."""
    Nb, L, H, G, dh = 3, 190, 2, 2, 72
    q, k, v, dout = make(31, Nb, L, Lk, H, G, dh)
    ql, kl = (torch.tensor([a, 60, 99], dtype=torch.int32, device="cuda") for a in (190, Lk))
    out, lse = torch.empty((Nb * L, H * dh), dtype=BF, device="cuda"), torch.empty((Nb, H, L), device="cuda")
    grads = [torch.empty_like(t) for t in (q, k, v)]
    ws = workspace(max(hq.hq_attention_bwd_workspace_size(Nb, L, Lk, H, G, dh), hq.hq_attention_fwd_workspace_size(Nb, L, Lk, H, G, dh)))

    def step():
        hq.hq_attention_fwd(q, k, v, Nb, H, G, out, lse, ws, q_lens=ql, k_lens=kl)
        hq.hq_attention_bwd(q, k, v, out, lse, dout, Nb, H, G, *grads, ws, q_lens=ql, k_lens=kl)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (32, 33):
        for old, new in zip((q, k, v, dout), make(seed, Nb, L, Lk, H, G, dh)):
            old.copy_(new)
        ql.copy_(torch.tensor([seed, 190, 0], dtype=torch.int32))
        kl.copy_(torch.tensor([Lk, seed, 5], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = check(hq, q, k, v, dout, Nb, H, G, q_lens=ql, k_lens=kl)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and all(torch.equal(a, b) for a, b in zip(grads, want[2]))


@pytest.mark.parametrize("Lk", [300, 100])
def test_offsets_past_32_bits(hq, Lk):
    """Rows 4 Mi elements apart: the last ones lie beyond 2^31 elements."""
    Nb, L, H, G, dh = 2, 300, 1, 1, 64
    pitch = 1 << 22
    q, k, v, dout = make(41, Nb, L, Lk, H, G, dh)
    want = check(hq, q, k, v, dout, Nb, H, G)
    wide = torch.empty((Nb * L, pitch), dtype=BF, device="cuda")               # 5 GB
    rows = [Nb * n for n in (L, Lk, Lk, L, L, L, Lk, Lk)]
    cols = [wide[Nb * L - n:, 64 * i: 64 * (i + 1)] for i, n in enumerate(rows)]
    for c, t in zip(cols, (q, k, v, dout)):
        c.copy_(t)
    lse = torch.empty((Nb, H, L), device="cuda")
    hq.hq_attention_fwd(*cols[:3], Nb, H, G, cols[4], lse, workspace(hq.hq_attention_fwd_workspace_size(Nb, L, Lk, H, G, dh)))
    ws = workspace(hq.hq_attention_bwd_workspace_size(Nb, L, Lk, H, G, dh))
    hq.hq_attention_bwd(*cols[:3], cols[4], lse, cols[3], Nb, H, G, *cols[5:], ws)
    assert torch.equal(cols[4], want[0]) and all(torch.equal(a, b) for a, b in zip(cols[5:], want[2]))


def test_agrees_with_the_inference_attention(hq):
    """The same inputs through hq_attention: both within the bound of 64-bit arithmetic."""
    Nb, L, H, dh = 2, 256, 4, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn((Nb * L, 3 * H * dh), generator=gen, device="cuda").to(BF)
    q, k, v = qkv.chunk(3, 1)
    out, _ = fwd(hq, q, k, v, Nb, H, H)
    old = torch.empty((Nb * L, H * dh), dtype=BF, device="cuda")
    hq.hq_attention(qkv, Nb, H, old)
    want, _, bound, _ = forward(q, k, v, Nb, H, H, dh ** -0.5)
    within(out, want, bound, "out")
    within(old, want, 2 * bound, "hq_attention")


@pytest.mark.parametrize("dh,H,G", [(40, 8, 4), (64, 8, 8), (72, 8, 8), (128, 8, 2)])
@pytest.mark.parametrize("Lq,Lk,lens", [(2, 2, False), (300, 130, False), (200, 200, True), (2100, 140, False), (2100, 140, True)])
def test_queries_that_see_one_key(hq, dh, H, G, Lq, Lk, lens):
    """Under the causal mask the query that sees the first key only has a weight of 1 whatever its score: with the gradients of all other
    outputs zero, dq and dk are zero, to the bit, and dv is not."""
    ql, kl = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([Lq, 77, 2, 90], [Lk, 77, 2, 70])) if lens else (None, None)
    Nb = 4 if lens else 2
    q, k, v, dout = make(61 + dh, Nb, Lq, Lk, H, G, dh)
    one = (visible(Nb, Lq, Lk, True, ql, kl, "cuda").sum(-1) == 1).flatten()
    assert one.sum() == Nb
    dout[~one] = 0
    _, _, (dq, dk, dv) = check(hq, q, k, v, dout, Nb, H, G, causal=True, q_lens=ql, k_lens=kl)
    assert not dq.any() and not dk.any() and dv.any()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("of", ["queries", "keys"])
@pytest.mark.parametrize("Lq,Lk,H,G,dh", [(260, 77, 4, 4, 40), (2100, 140, 2, 1, 64), (300, 300, 3, 1, 72), (2100, 140, 2, 1, 128)])
def test_lengths_of_one_side(hq, Lq, Lk, H, G, dh, of, causal):
    """Text tokens of several lengths under images of one (k_lens alone), and padded queries on keys of one length (q_lens alone); what
    lies behind the lengths may be anything."""
    L = Lk if of == "keys" else Lq
    lens = torch.tensor([L, 0, 1, L // 2, L - 1], dtype=torch.int32, device="cuda")
    Nb = lens.numel()
    q, k, v, dout = make(81 + dh, Nb, Lq, Lk, H, G, dh)
    kw = dict(causal=causal, q_lens=lens if of == "queries" else None, k_lens=lens if of == "keys" else None)
    clean = check(hq, q, k, v, dout, Nb, H, G, **kw)
    dead = (torch.arange(L, device="cuda")[None] >= lens[:, None]).flatten()
    for t in (q, dout) if of == "queries" else (k, v):
        t[dead] = math.nan
    out, lse = fwd(hq, q, k, v, Nb, H, G, **kw)
    grads = bwd(hq, q, k, v, out, lse, dout, Nb, H, G, **kw)
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1]) and all(torch.equal(a, b) for a, b in zip(grads, clean[2]))
    for g in grads[:1] if of == "queries" else grads[1:]:
        assert not g[dead].any()
