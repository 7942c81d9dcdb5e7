"""The norm of queries and keys with the position rotation, and its gradient, against 64-bit arithmetic (torch's differentiation of the
plain formula) and against differences; and a block's attention forward and backward as a training step runs them."""
import math

import pytest
import torch

from attention_train_reference import backward, forward, rope

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


def tables(npos, rot):
    if rot == 0:
        return None, None
    angle = torch.arange(npos, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))
    return angle.cos().float().cuda(), angle.sin().float().cuda()


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def run(hq, rows, H, G, dh, rot, dtype, interleaved, gamma, npos, positions, pad=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(rows * 31 + dh + seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    qkv = rand(rows, (H + G) * dh + pad).to(dtype)
    q, k = qkv[:, : H * dh], (qkv[:, H * dh: (H + G) * dh] if G else None)
    gq, gk = (1 + 0.3 * rand(dh), 1 + 0.3 * rand(dh)) if gamma else (None, None)
    cos, sin = tables(npos, rot)
    pos = torch.randint(-2, npos + 2, (rows,), generator=gen, device="cuda").to(torch.int32) if positions else None
    outs = torch.full((rows, (H + G) * dh + pad), math.nan, dtype=dtype, device="cuda")
    grads_out = rand(rows, (H + G) * dh).to(dtype)
    dqkv = torch.full_like(outs, math.nan)
    part = lambda t: (t[:, : H * dh], t[:, H * dh: (H + G) * dh] if G else None)  # noqa: E731
    hq.hq_qk_norm_rope(q, k, H, G, gq, gk, EPS, cos, sin, *part(outs), positions=pos, interleaved=interleaved)
    dg = [torch.full((dh,), math.nan, device="cuda") if gamma and n else None for n in (H, G)]
    ws = torch.empty((hq.hq_qk_norm_rope_bwd_workspace_size(rows, H, G, dh),), dtype=torch.uint8, device="cuda").fill_(0xFF)
    hq.hq_qk_norm_rope_bwd(q, k, H, G, gq, gk, EPS, cos, sin, *part(grads_out), *part(dqkv), *dg, ws, positions=pos, interleaved=interleaved)
    u, f = unit(dtype), 2.0 ** -23
    for x, heads, g, y, go, dx, dgamma in zip((q, k), (H, G), (gq, gk), part(outs), part(grads_out), part(dqkv), dg):
        if x is None:
            continue
        leaves = [x.double().clone().requires_grad_()] + ([g.double().clone().requires_grad_()] if g is not None else [])
        want = rope(leaves[0], heads, leaves[1] if g is not None else None, EPS, cos, sin, pos, interleaved)
        grads = torch.autograd.grad(want, leaves, go.double())
        # fp32 arithmetic on values of size at most |a| + |b| of a pair (a head's largest bounds both), one rounding at the end
        big = lambda t: t.detach().abs().reshape(rows, heads, dh).amax(-1, keepdim=True).expand(-1, -1, dh).flatten(1)  # noqa: E731
        bound = u * want.detach().abs() + 64 * f * big(want)
        assert bool(((y.double() - want.detach()).abs() <= bound).all())
        # the gradient's terms: gamma u and xh mean(gamma u xh), both at most max|gamma| |go| sqrt(2) / rms(x) (norms over the head)
        inv = (x.double().reshape(rows, heads, dh).square().mean(-1, keepdim=True) + EPS).rsqrt()
        gmax = 1.0 if g is None else g.abs().max().item()
        size = (inv * gmax * 2 * go.double().reshape(rows, heads, dh).norm(dim=-1, keepdim=True)).expand(-1, -1, dh).flatten(1)
        bound = u * grads[0].abs() + 64 * f * size
        assert bool(((dx.double() - grads[0]).abs() <= bound).all())
        if dgamma is not None:
            # every term |u xh| <= 2 max|go| |xh|, summed in fp32 over rows x heads terms by a tree of runs
            xh = (x.double().reshape(rows, heads, dh) * inv).abs()
            terms = (xh * 2 * go.double().abs().reshape(rows, heads, dh).amax(-1, keepdim=True)).sum((0, 1))
            assert bool(((dgamma.double() - grads[1]).abs() <= (16 + math.sqrt(rows * heads)) * f * terms + 1e-12).all())
    if pad:
        assert bool(outs[:, -pad:].isnan().all()) and bool(dqkv[:, -pad:].isnan().all())
    return outs, dqkv, dg


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,H,G,dh,rot", [(1, 1, 1, 8, 8), (3, 8, 8, 64, 64), (33, 4, 2, 72, 72), (257, 16, 1, 128, 64), (100, 3, 3, 40, 20),
                                             (70, 5, 5, 48, 48), (19, 2, 1, 120, 36), (64, 6, 6, 96, 96), (40, 2, 2, 16, 2), (40, 2, 2, 80, 0),
                                             (300, 7, 3, 128, 128), (9, 40, 40, 32, 32)])
def test_against_64_bits(hq, rows, H, G, dh, rot, interleaved, dtype):
    run(hq, rows, H, G, dh, rot, dtype, interleaved, True, 50, True)
    run(hq, rows, H, G, dh, rot, dtype, interleaved, False, 16, False, pad=16)


def test_many_rows(hq):
    run(hq, 20011, 8, 2, 64, 64, torch.bfloat16, False, True, 1024, False)


def test_queries_alone(hq):
    run(hq, 130, 4, 0, 64, 64, torch.bfloat16, False, True, 130, False)


def test_same_bits_and_in_place(hq):
    args = (1000, 8, 8, 64, 64, torch.bfloat16, False, True, 250, False)
    a, b = run(hq, *args), run(hq, *args)
    for x, y in zip(a[:2], b[:2]):
        assert torch.equal(x, y)
    assert all(torch.equal(x, y) for x, y in zip(a[2], b[2]))
    gen = torch.Generator(device="cuda").manual_seed(8)
    for interleaved, dh in ((False, 64), (True, 64), (False, 72)):
        q, k = (torch.randn((90, 4 * dh), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        cos, sin = tables(90, dh)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        hq.hq_qk_norm_rope(q, k, 4, 4, None, None, EPS, cos, sin, qo, ko, interleaved=interleaved)
        dq, dk = torch.empty_like(q), torch.empty_like(k)
        hq.hq_qk_norm_rope_bwd(q, k, 4, 4, None, None, EPS, cos, sin, qo, ko, dq, dk, None, None, None, interleaved=interleaved)
        q2, k2, g = q.clone(), k.clone(), qo.clone()
        hq.hq_qk_norm_rope_bwd(q2, k2, 4, 4, None, None, EPS, cos, sin, g, ko, g, k2, None, None, None, interleaved=interleaved)
        assert torch.equal(g, dq) and torch.equal(k2, dk)
        hq.hq_qk_norm_rope(q2, k, 4, 4, None, None, EPS, cos, sin, q2, k, interleaved=interleaved)
        assert torch.equal(q2, qo) and torch.equal(k, ko)


def test_zero_rows_and_zero_heads_values(hq):
    """A head of zeros: the norm divides by sqrt(eps); no rows at all: nothing but cleared sums."""
    q = torch.zeros((4, 128), device="cuda")
    cos, sin = tables(4, 64)
    out = torch.full_like(q, math.nan)
    hq.hq_qk_norm_rope(q, None, 2, 0, None, None, EPS, cos, sin, out, None)
    assert not out.any()
    dg = torch.full((64,), math.nan, device="cuda")
    hq.hq_qk_norm_rope_bwd(q[:0], None, 2, 0, None, None, EPS, cos, sin, q[:0], None, q[:0], None, dg, None, None)
    assert not dg.any()


def test_gradient_against_differences(hq):
    rows, H, dh = 30, 2, 48
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, go = (torch.randn((rows, H * dh), generator=gen, device="cuda") for _ in range(2))
    gamma, (cos, sin) = 1 + 0.2 * torch.randn(dh, generator=gen, device="cuda"), tables(rows, 32)
    dq, dg = torch.empty_like(q), torch.empty_like(gamma)
    ws = torch.empty((hq.hq_qk_norm_rope_bwd_workspace_size(rows, H, 0, dh),), dtype=torch.uint8, device="cuda")
    hq.hq_qk_norm_rope_bwd(q, None, H, 0, gamma, None, EPS, cos, sin, go, None, dq, None, dg, None, ws)
    loss = lambda x, g: (rope(x, H, g, EPS, cos, sin, None, False) * go.double()).sum()  # noqa: E731
    h = 1e-6
    for which, grad in ((0, dq), (1, dg)):
        base = [q.double(), gamma.double()]
        d = torch.randn(base[which].shape, generator=gen, device="cuda", dtype=torch.float64)
        lo, hi = list(base), list(base)
        lo[which], hi[which] = base[which] - h * d, base[which] + h * d
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        # fp32 gradients: 64 units of each term's size at most; differences in 64 bits with a step of 1e-6: 1e-8 of the loss's terms
        allowed = 64 * 2.0 ** -23 * (grad.abs().double() * d.abs()).sum() + 1e-4 * math.sqrt(d.numel())
        assert abs((grad.double() * d).sum() - slope) <= allowed


@pytest.mark.parametrize("graph", [False, True])
def test_a_block_s_attention_forward_and_backward(hq, graph):
    """As a training step runs them: fused projection -> norm + rotation -> attention -> gradient back to the projection's output,
    every step against 64 bits on what the step before left."""
    Nb, L, H, G, dh = 2, 150, 4, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(6)
    bf = torch.bfloat16
    qkv, dout = torch.randn((Nb * L, (H + 2 * G) * dh), generator=gen, device="cuda").to(bf), torch.randn((Nb * L, H * dh), generator=gen, device="cuda").to(bf)
    gq, gk = (1 + 0.2 * torch.randn(dh, generator=gen, device="cuda") for _ in range(2))
    cos, sin = tables(L, dh)
    cut = (slice(0, H * dh), slice(H * dh, (H + G) * dh), slice((H + G) * dh, (H + 2 * G) * dh))
    q, k, v = (qkv[:, c] for c in cut)
    qn, kn = torch.empty((Nb * L, H * dh), dtype=bf, device="cuda"), torch.empty((Nb * L, G * dh), dtype=bf, device="cuda")
    out, lse = torch.empty_like(dout), torch.empty((Nb, H, L), device="cuda")
    dqn, dkn, dqkv, dgq, dgk = torch.empty_like(qn), torch.empty_like(kn), torch.empty_like(qkv), torch.empty_like(gq), torch.empty_like(gk)
    ws = torch.empty((max(hq.hq_attention_fwd_workspace_size(Nb, L, L, H, G, dh), hq.hq_attention_bwd_workspace_size(Nb, L, L, H, G, dh),
                          hq.hq_qk_norm_rope_bwd_workspace_size(Nb * L, H, G, dh)),), dtype=torch.uint8, device="cuda")

    def step():
        hq.hq_qk_norm_rope(q, k, H, G, gq, gk, EPS, cos, sin, qn, kn)
        hq.hq_attention_fwd(qn, kn, v, Nb, H, G, out, lse, ws)
        hq.hq_attention_bwd(qn, kn, v, out, lse, dout, Nb, H, G, dqn, dkn, dqkv[:, cut[2]], ws)
        hq.hq_qk_norm_rope_bwd(q, k, H, G, gq, gk, EPS, cos, sin, dqn, dkn, dqkv[:, cut[0]], dqkv[:, cut[1]], dgq, dgk, ws)
    step()
    if graph:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for t in (qn, kn, out, lse, dqkv, dgq, dgk):
            t.zero_()
        g.replay()
    torch.cuda.synchronize()
    u = 2.0 ** -8
    for x, heads, gm, y in ((q, H, gq, qn), (k, G, gk, kn)):
        want = rope(x, heads, gm, EPS, cos, sin, None, False)
        assert bool(((y.double() - want).abs() <= u * want.abs() + 1e-4).all())
    want, _, bound, _ = forward(qn, kn, v, Nb, H, G, dh ** -0.5)
    assert bool(((out.double() - want).abs() <= bound).all())
    wants, bounds = backward(qn, kn, v, out, lse, dout, Nb, H, G, dh ** -0.5)
    for got, w, b in ((dqn, wants[0], bounds[0]), (dkn, wants[1], bounds[1]), (dqkv[:, cut[2]], wants[2], bounds[2])):
        assert bool(((got.double() - w).abs() <= b).all())
    for x, heads, gm, go, dx, dg in ((q, H, gq, dqn, dqkv[:, cut[0]], dgq), (k, G, gk, dkn, dqkv[:, cut[1]], dgk)):
        leaves = [x.double().clone().requires_grad_(), gm.double().clone().requires_grad_()]
        gx, gg = torch.autograd.grad(rope(leaves[0], heads, leaves[1], EPS, cos, sin, None, False), leaves, go.double())
        size = go.double().abs().max() * 64 * 2.0 ** -23 * math.sqrt(dh) * 8
        assert bool(((dx.double() - gx).abs() <= u * gx.abs() + size).all())
        assert bool(((dg.double() - gg).abs() <= 1e-4 * gg.abs().max()).all())


def check_gradient(hq, q, k, H, G, gq, gk, eps, cos, sin, pos, interleaved, wanted=(True, True), stream=None):
    """Forward and gradient of the given inputs against 64 bits, element by element, with the bounds of `run`; returns what was computed."""
    rows, dtype, dh = q.shape[0], q.dtype, q.shape[1] // H
    gen = torch.Generator(device="cuda").manual_seed(rows + dh)
    grads_out = [torch.randn((rows, n * dh), generator=gen, device="cuda").to(dtype) for n in (H, G)]
    outs, dx = ([torch.full((rows, n * dh), math.nan, dtype=dtype, device="cuda") for n in (H, G)] for _ in range(2))
    dg = [torch.full((dh,), math.nan, device="cuda") if want else None for want in wanted]
    ws = torch.empty((hq.hq_qk_norm_rope_bwd_workspace_size(rows, H, G, dh),), dtype=torch.uint8, device="cuda").fill_(0xFF)
    torch.cuda.synchronize()                     # the calls may run on another stream than the fills
    hq.hq_qk_norm_rope(q, k, H, G, gq, gk, eps, cos, sin, *outs, positions=pos, interleaved=interleaved, stream=stream)
    hq.hq_qk_norm_rope_bwd(q, k, H, G, gq, gk, eps, cos, sin, *grads_out, *dx, *dg, ws, positions=pos, interleaved=interleaved, stream=stream)
    torch.cuda.synchronize()
    u, f = unit(dtype), 2.0 ** -23
    for x, heads, g, y, go, d, dgamma in zip((q, k), (H, G), (gq, gk), outs, grads_out, dx, dg):
        leaves = [x.double().clone().requires_grad_(), g.double().clone().requires_grad_()]
        want = rope(leaves[0], heads, leaves[1], eps, cos, sin, pos, interleaved)
        grads = torch.autograd.grad(want, leaves, go.double())
        by_head = lambda t: t.double().reshape(rows, heads, dh)  # noqa: E731
        whole = lambda t: t.expand(-1, -1, dh).flatten(1)  # noqa: E731
        bound = u * want.detach().abs() + 64 * f * whole(by_head(want.detach()).abs().amax(-1, keepdim=True))
        assert bool(((y.double() - want.detach()).abs() <= bound).all())
        inv = (by_head(x).square().mean(-1, keepdim=True) + eps).rsqrt()
        bound = u * grads[0].abs() + 64 * f * whole(inv * g.abs().max().item() * 2 * by_head(go).norm(dim=-1, keepdim=True))
        assert bool(((d.double() - grads[0]).abs() <= bound).all())
        if dgamma is not None:
            terms = ((by_head(x) * inv).abs() * 2 * by_head(go).abs().amax(-1, keepdim=True)).sum((0, 1))
            assert bool(((dgamma.double() - grads[1]).abs() <= (16 + math.sqrt(rows * heads)) * f * terms + 1e-12).all())
    return outs + dx + dg


def block_inputs(rows, H, G, dh, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return rand(rows, H * dh).to(dtype), rand(rows, G * dh).to(dtype), 1 + 0.3 * rand(dh), 1 + 0.3 * rand(dh)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,H,G,dh", [(5, 3, 6, 64), (33, 6, 3, 64), (7, 1, 1, 128), (3, 2, 2, 72), (9, 1, 2, 32), (1, 5, 1, 40)])
def test_no_epsilon(hq, rows, H, G, dh, dtype):
    """eps = 0 on rows that are not zero: lanes without a head or a row, which divide by the norm of nothing, have no part in gamma's sums."""
    q, k, gq, gk = block_inputs(rows, H, G, dh, dtype, 71)
    check_gradient(hq, q, k, H, G, gq, gk, 0.0, *tables(rows, dh // 2), None, True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("garbage", [math.nan, math.inf])
@pytest.mark.parametrize("H,G", [(3, 6), (1, 2)])
def test_table_rows_that_no_token_takes(hq, interleaved, garbage, H, G):
    """Whatever the first row of the tables holds, where no token stands there."""
    rows, dh, npos = 37, 64, 20
    q, k, gq, gk = block_inputs(rows, H, G, dh, torch.bfloat16, 72)
    cos, sin = tables(npos, dh)
    pos = (torch.arange(rows, device="cuda") % (npos - 1) + 1).to(torch.int32)
    want = check_gradient(hq, q, k, H, G, gq, gk, EPS, cos, sin, pos, interleaved)
    cos[0], sin[0] = garbage, garbage
    got = check_gradient(hq, q, k, H, G, gq, gk, EPS, cos, sin, pos, interleaved)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def off_by_one_float(t):
    """The same values, dense, at an address that is a multiple of 4 bytes and no more."""
    wide = torch.empty((t.numel() + 1,), dtype=t.dtype, device=t.device)
    wide[1:] = t.flatten()
    return wide[1:].view(t.shape)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dh,rot", [(32, 32), (64, 64), (64, 16), (72, 48), (128, 128)])
def test_tables_off_the_16_byte_boundary(hq, dh, rot, interleaved, dtype):
    rows, H, G = 45, 3, 2
    q, k, gq, gk = block_inputs(rows, H, G, dh, dtype, 73)
    cos, sin = (off_by_one_float(t) for t in tables(20, rot))
    assert cos.is_contiguous() and cos.data_ptr() % 16 == 4
    check_gradient(hq, q, k, H, G, off_by_one_float(gq), off_by_one_float(gk), EPS, cos, sin, None, interleaved)


@pytest.mark.parametrize("wanted", [(True, False), (False, True), (False, False)])
def test_gradient_of_one_gamma(hq, wanted):
    q, k, gq, gk = block_inputs(300, 4, 2, 64, torch.bfloat16, 74)
    args = (hq, q, k, 4, 2, gq, gk, EPS, *tables(300, 64), None, False)
    both, some = check_gradient(*args), check_gradient(*args, wanted=wanted)
    assert all(b is None or torch.equal(a, b) for a, b in zip(both, some))
    assert [b is not None for b in some[4:]] == list(wanted)


def test_streams_and_calls_that_overlap(hq):
    """On another stream, and steps of several widths at the same time, each with a workspace of its own: the bits of the calls one by one."""
    steps = []
    for seed, (rows, H, G, dh, dtype) in enumerate([(30000, 8, 8, 64, torch.bfloat16), (20, 8, 8, 64, torch.bfloat16),
                                                    (9000, 6, 3, 72, torch.float32), (5000, 16, 2, 128, torch.bfloat16)]):
        q, k, gq, gk = block_inputs(rows, H, G, dh, dtype, 75 + seed)
        table, stream = tables(250, dh), torch.cuda.Stream()
        want = check_gradient(hq, q, k, H, G, gq, gk, EPS, *table, None, False, stream=stream)
        # the gradients of the outputs that check_gradient drew
        gen = torch.Generator(device="cuda").manual_seed(rows + dh)
        go = [torch.randn((rows, n * dh), generator=gen, device="cuda").to(dtype) for n in (H, G)]
        got = [torch.full_like(t, math.nan) for t in want]
        ws = torch.empty((hq.hq_qk_norm_rope_bwd_workspace_size(rows, H, G, dh),), dtype=torch.uint8, device="cuda").fill_(0xFF)
        steps.append(((q, k, H, G, gq, gk, EPS, *table), go, want, got, ws, stream))
    torch.cuda.synchronize()
    for _ in range(5):
        for args, go, _, got, ws, stream in steps:
            hq.hq_qk_norm_rope(*args, *got[:2], stream=stream)
            hq.hq_qk_norm_rope_bwd(*args, *go, *got[2:], ws, stream=stream)
    torch.cuda.synchronize()
    for _, _, want, got, _, _ in steps:
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_past_32_bits(hq, dtype):
    """Rows 4 Mi elements apart: the last ones lie beyond 2^31 elements."""
    rows, H, G, dh = 600, 2, 1, 64
    q, k, gq, gk = block_inputs(rows, H, G, dh, dtype, 76)
    args = (H, G, gq, gk, EPS, *tables(rows, dh))
    want = check_gradient(hq, q, k, *args, None, False)
    gen = torch.Generator(device="cuda").manual_seed(rows + dh)
    go = [torch.randn((rows, n * dh), generator=gen, device="cuda").to(dtype) for n in (H, G)]
    wide = torch.empty((rows, 1 << 22), dtype=dtype, device="cuda")            # 5 or 10 GB
    cols = [wide[:, 128 * i: 128 * i + t.shape[1]] for i, t in enumerate([q, k, *go, *want[:4]])]
    for c, t in zip(cols, (q, k, *go)):
        c.copy_(t)
    dg = [torch.empty_like(gq) for _ in range(2)]
    ws = torch.empty((hq.hq_qk_norm_rope_bwd_workspace_size(rows, H, G, dh),), dtype=torch.uint8, device="cuda")
    hq.hq_qk_norm_rope(*cols[:2], *args, *cols[4:6])
    hq.hq_qk_norm_rope_bwd(*cols[:2], *args, *cols[2:4], *cols[6:], *dg, ws)
    assert all(torch.equal(a, b) for a, b in zip(want, cols[4:] + dg))
