"""The gated residual with the norms before and after a block, and its gradient, against 64-bit arithmetic and against differences."""
import math

import pytest
import torch

from train_block_reference import F32, backward, forward, masked, there, unit

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
KINDS = {"layer": 0, "rms": 1, "none": 2}
# Steps of fp32 arithmetic behind one result: a row's sums run over 8 values of a thread, 32 lanes and up to 16 warps (below 32 additions),
# the square root, quotient and products of a norm a dozen more; two norms follow one another.
STEPS = 128


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


def modulation(rand, groups, cols, per):
    mod = 0.4 * rand(groups, 3 * cols)
    return mod[:, :cols], mod[:, cols: 2 * cols], mod[:, 2 * cols:]


def inputs(rows, cols, per, xt, ht, seed=0, pad=0, lens=None, mean=0.5):
    gen = torch.Generator(device="cuda").manual_seed(rows * 31 + cols + seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    groups = -(-rows // per) if per else 1
    x, h = rand(rows, cols + pad) + mean, 2 * rand(rows, cols + pad)
    x[:, 3] *= 40                                  # one channel far larger than the rest
    if lens is not None:                           # what stands behind the lengths is anything
        gone = ~there(rows, per, lens)[:, 0]
        x[gone], h[gone] = math.nan, math.inf
    return x.to(xt)[:, :cols], h.to(ht)[:, :cols], rand, modulation(rand, groups, cols, per)


def run(hq, rows, cols, per=0, norm="layer", post="none", xt=BF, ht=BF, gated=True, lens=None, plus=1.0, residual=0.7, pad=0, affine=True, seed=0):
    x, h, rand, (gate, bias, weight) = inputs(rows, cols, per, xt, ht, seed, pad, lens)
    pw = 1 + 0.3 * rand(cols) if post != "none" else None
    gate = gate if gated else None
    weight, bias = (weight, bias) if affine and norm != "none" else (None, None)
    kw = dict(rows_per_group=per, lens=lens, post=KINDS[post], post_weight=pw, norm=KINDS[norm], weight_plus=plus, residual_scale=residual)
    nan = lambda t, n=cols + pad: torch.full((rows, n), math.nan, dtype=t, device="cuda")  # noqa: E731
    xo_, y_ = nan(xt), nan(ht)
    x_out, y, stats = xo_[:, :cols], (y_[:, :cols] if norm != "none" else None), torch.full((rows, 4), math.nan, device="cuda")
    hq.hq_gate_norm(x, h, gate, weight, bias, x_out, y, stats, **kw)
    keep = there(rows, per, lens)
    w64 = masked(x.double(), keep), masked(h.double(), keep)
    want = forward(*w64, gate, weight, bias, per, post, pw, norm, plus, residual)
    checks = [("x_out", x_out, want[0], want[3])] + ([("y", y, want[1], want[4])] if norm != "none" else [])
    for name, got, ref, size in checks:
        bound = masked(unit(got.dtype) * ref.abs() + STEPS * F32 * size, keep)
        assert bool(((got.double() - masked(ref, keep)).abs() <= bound).all()), name
    stat_size = torch.cat((want[3].amax(-1, keepdim=True), want[2][:, 1:2] * (1 + (want[2][:, 1:2] * want[3].amax(-1, keepdim=True))),
                           h.double().abs().amax(-1, keepdim=True), want[2][:, 3:4]), 1)
    assert bool(((stats.double() - masked(want[2], keep)).abs() <= masked(STEPS * F32 * stat_size, keep)).all())
    # the gradient, from these results
    dx_out, dy = rand(rows, cols).to(xt), rand(rows, cols).to(ht) if norm != "none" else None
    if lens is not None:
        dx_out[~keep[:, 0]] = math.nan
        if dy is not None:
            dy[~keep[:, 0]] = math.inf
    groups = -(-rows // per) if per else 1
    dx_, dh_, dmod = nan(xt), nan(ht), torch.full((groups, 3 * cols), math.nan, device="cuda")
    dx, dh = dx_[:, :cols], dh_[:, :cols]
    dgate = dmod[:, :cols] if gated else None
    dbias, dweight = (dmod[:, cols: 2 * cols], dmod[:, 2 * cols:]) if norm != "none" else (None, None)
    dpw = torch.full((cols,), math.nan, device="cuda") if post != "none" else None
    ws = torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda").fill_(0xFF)
    del kw["post"]
    hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, dx_out, dy, dx, dh, dgate, dweight, dbias, ws, post=KINDS[post], dpost_weight=dpw, **kw)
    found = backward(x_out.double(), h.double(), stats, gate, weight, dx_out.double(), None if dy is None else dy.double(), per, lens, post, pw, norm,
                     plus, residual)
    for name, got in (("dx", dx), ("dh", dh), ("dgate", dgate), ("dweight", dweight), ("dbias", dbias), ("dpost_weight", dpw)):
        if got is None:
            continue
        ref, size = found[name]
        # sums over rows: one rounding a row and a joining step, in the worst order
        steps = STEPS + (math.sqrt(rows) * 4 if name[1] != "x" and name != "dh" else 0)
        out = unit(got.dtype) if name in ("dx", "dh") else F32
        assert bool(((got.double() - ref).abs() <= out * ref.abs() + steps * F32 * size + 1e-30).all()), name
    if pad:
        assert all(bool(t[:, cols:].isnan().all()) for t in (xo_, dx_, dh_)) and (norm == "none" or bool(y_[:, cols:].isnan().all()))
    return [t for t in (x_out, y, stats, dx, dh, dgate, dweight, dbias, dpw) if t is not None]


@pytest.mark.parametrize("xt,ht", [(BF, BF), (F, BF), (F, F), (BF, F)])
@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "rms"), ("layer", "rms"), ("rms", "layer"), ("layer", "layer"), ("rms", "none")])
@pytest.mark.parametrize("rows,cols,per", [(1, 8, 0), (37, 264, 5), (260, 1152, 64), (75, 2056, 0)])
def test_against_64_bits(hq, rows, cols, per, norm, post, xt, ht):
    run(hq, rows, cols, per, norm, post, xt, ht)


@pytest.mark.parametrize("rows,cols,per", [(3, 16, 1), (1000, 64, 1), (33, 256, 7), (513, 248, 100), (129, 768, 129), (300, 1000, 77), (40, 4096, 13),
                                           (9, 4088, 2), (2000, 320, 1999), (5000, 512, 0), (7, 1280, 1000000), (77, 72, 10), (500, 128, 6), (41, 8, 3)])
def test_shapes(hq, rows, cols, per):
    run(hq, rows, cols, per, pad=8)
    run(hq, rows, cols, per, "rms", "rms", F, BF, pad=16)


@pytest.mark.parametrize("rows,cols,per", [(33, 4096, 0), (21, 3848, 4), (9, 3584, 1)])
def test_widest_rows_of_fp32(hq, rows, cols, per):
    run(hq, rows, cols, per, xt=F, ht=F)
    run(hq, rows, cols, per, "rms", "layer", F, F, gated=False)


def test_groups_larger_than_all_rows(hq):
    a, b = run(hq, 50, 128, (1 << 63) - 1), run(hq, 50, 128, 50)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_many_rows(hq):
    run(hq, 20011, 1152, 256)
    run(hq, 70001, 64, 0, "rms", "layer", F, F)
    run(hq, 33000, 128, 3, "layer", "rms")


@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "rms")])
@pytest.mark.parametrize("rows,cols,per", [(154, 256, 77), (1000, 1152, 77), (33, 64, 4), (64, 2304, 16), (100, 128, 11), (90, 56, 7), (70, 120, 64)])
def test_lengths(hq, rows, cols, per, norm, post):
    groups = -(-rows // per)
    lens = torch.tensor([(i * 5) % (per + 3) - 1 for i in range(groups)], dtype=torch.int32, device="cuda")     # none, negative, all, too many
    run(hq, rows, cols, per, norm, post, lens=lens)
    run(hq, rows, cols, per, norm, post, lens=torch.zeros_like(lens))


@pytest.mark.parametrize("cols", [64, 1152])
def test_vectors_of_empty_groups_hold_anything(hq, cols):
    rows, per = 200, 20
    lens = torch.tensor([0, 20, 3, 0, 0, 7, 20, 0, 1, 0], dtype=torch.int32, device="cuda")
    x, h, rand, mod = inputs(rows, cols, per, F, BF, lens=lens)
    pw, dxo, dy = 1 + 0.3 * rand(cols), rand(rows, cols), rand(rows, cols).to(BF)
    results = []
    for fill in (0.0, math.nan, math.inf):
        gate, bias, weight = (torch.where((lens == 0)[:, None], torch.full_like(m, fill), m) for m in mod)
        x_out, y, stats, dx, dh = torch.empty_like(x), torch.empty_like(h), torch.empty((rows, 4), device="cuda"), torch.empty_like(x), torch.empty_like(h)
        kw = dict(rows_per_group=per, lens=lens, post=1, post_weight=pw, weight_plus=1.0)
        hq.hq_gate_norm(x, h, gate, weight, bias, x_out, y, stats, **kw)
        sums = [torch.empty((10, cols), device="cuda") for _ in range(3)] + [torch.empty(cols, device="cuda")]
        ws = torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")
        hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, dxo, dy, dx, dh, *sums[:3], ws, dpost_weight=sums[3], **kw)
        results.append([x_out, y, stats, dx, dh] + sums)
        assert all(bool(t.isfinite().all()) for t in results[-1]) and all(bool((s[lens == 0] == 0).all()) for s in sums[:3])
    assert all(torch.equal(a, b) for r in results[1:] for a, b in zip(results[0], r))


def test_parts_of_the_operator(hq):
    run(hq, 130, 640, 32, norm="none")             # the residual alone
    run(hq, 130, 640, 32, norm="none", post="layer", xt=F, gated=False)
    run(hq, 130, 640, 32, gated=False, affine=False, plus=3.0, residual=1.0)
    run(hq, 130, 640, 32, gated=False, post="rms", plus=0.0, residual=-2.0)


def test_norm_alone(hq):
    """h None: x_out is x; nothing but y, and the gradient from dy and, in a residual stream, from what else uses x."""
    rows, cols, per = 90, 1152, 30
    x, _, rand, (_, bias, weight) = inputs(rows, cols, per, BF, BF)
    y, stats = torch.empty_like(x), torch.empty((rows, 4), device="cuda")
    hq.hq_gate_norm(x, None, None, weight, bias, None, y, stats, rows_per_group=per, weight_plus=1.0)
    want = forward(x.double(), None, None, weight, bias, per, plus=1.0)
    assert bool(((y.double() - want[1]).abs() <= unit(BF) * want[1].abs() + STEPS * F32 * want[4]).all())
    assert bool((stats[:, 2] == 0).all()) and bool((stats[:, 3] == 1).all())
    dy, later = rand(rows, cols).to(BF), rand(rows, cols).to(BF)
    ws = torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")
    for dx_out in (None, later):
        dx, dw = torch.empty_like(x), torch.empty((3, cols), device="cuda")
        hq.hq_gate_norm_bwd(x, None, stats, None, weight, dx_out, dy, dx, None, None, dw, None, ws, rows_per_group=per, weight_plus=1.0)
        found = backward(x.double(), None, stats, None, weight, None if dx_out is None else dx_out.double(), dy.double(), per, plus=1.0)
        for name, got in (("dx", dx), ("dweight", dw)):
            ref, size = found[name]
            assert bool(((got.double() - ref).abs() <= unit(got.dtype) * ref.abs() + 2 * STEPS * F32 * size).all())


def test_what_is_not_wanted(hq):
    """Gradients left out change nothing in the others; without sums over rows no workspace is needed."""
    rows, cols, per = 200, 512, 50
    x, h, rand, (gate, bias, weight) = inputs(rows, cols, per, BF, BF)
    pw = 1 + 0.3 * rand(cols)
    x_out, y, stats = torch.empty_like(x), torch.empty_like(h), torch.empty((rows, 4), device="cuda")
    kw = dict(rows_per_group=per, post=1, post_weight=pw, weight_plus=1.0)
    hq.hq_gate_norm(x, h, gate, weight, bias, x_out, y, stats, **kw)
    hq.hq_gate_norm(x, h, gate, weight, bias, None, y2 := torch.empty_like(h), None, **kw)
    assert torch.equal(y, y2)
    dxo, dy = rand(rows, cols).to(BF), rand(rows, cols).to(BF)
    ws = torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")
    outs = lambda: [torch.empty_like(x), torch.empty_like(h)] + [torch.empty((4, cols), device="cuda") for _ in range(3)] + [torch.empty(cols, device="cuda")]  # noqa: E731
    full = outs()
    call = lambda o, w: hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, dxo, dy, *o[:5], w, dpost_weight=o[5], **kw)  # noqa: E731
    call(full, ws)
    for left in range(6):
        some = outs()
        some[left] = None
        call(some, ws)
        for a, b in zip(some, full):
            assert a is None or torch.equal(a, b)
        only = [None] * 6
        only[left] = outs()[left]
        call(only, ws if left > 1 else None)
        assert torch.equal(only[left], full[left])


def test_same_bits_and_in_place(hq):
    for args in ((3000, 1152, 100), (513, 96, 9)):
        a, b = run(hq, *args), run(hq, *args)
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    rows, cols, per = 3000, 1152, 256
    for xt, ht in ((BF, BF), (F, BF)):
        x, h, rand, (gate, bias, weight) = inputs(rows, cols, per, xt, ht)
        x_out, y, stats = torch.empty_like(x), torch.empty_like(h), torch.empty((rows, 4), device="cuda")
        kw = dict(rows_per_group=per, weight_plus=1.0)
        hq.hq_gate_norm(x, h, gate, weight, bias, x_out, y, stats, **kw)
        x2, h2 = x.clone(), h.clone()
        hq.hq_gate_norm(x2, h2, gate, weight, bias, x2, h2, None, **kw)
        assert torch.equal(x2, x_out) and torch.equal(h2, y)
        dxo, dy = rand(rows, cols).to(xt), rand(rows, cols).to(ht)
        dx, dh = torch.empty_like(x), torch.empty_like(h)
        hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, dxo, dy, dx, dh, None, None, None, None, **kw)
        for into in ("dy", "h"):
            dxo2, dy2, h2 = dxo.clone(), dy.clone(), h.clone()
            hq.hq_gate_norm_bwd(x_out, h2, stats, gate, weight, dxo2, dy2, dxo2, dy2 if into == "dy" else h2, None, None, None, None, **kw)
            assert torch.equal(dxo2, dx) and torch.equal(dy2 if into == "dy" else h2, dh)


def test_against_differences(hq):
    """The loss sum(x_out a) + sum(y b) along random directions of every input, by central differences of the kernel's own fp32 results
    summed in fp64.  Step e: the cubic term is e^2 / 6 of the third derivative (values and derivatives of size one: 1e-5 relative at e = 2^-8);
    fp32 results are off by 2^-24 of values up to 8 each, random in sign, over a step of 2 e: sqrt(n) 2^-21 / (2 e)."""
    rows, cols, per, e = 48, 256, 16, 2.0 ** -8
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    for norm, post in (("layer", "layer"), ("rms", "rms"), ("layer", "none")):
        x, h, gate, weight, bias, pw = rand(rows, cols), rand(rows, cols), rand(3, cols), 0.3 * rand(3, cols), rand(3, cols), 1 + 0.3 * rand(cols)
        a, b = rand(rows, cols), rand(rows, cols)
        kw = dict(rows_per_group=per, post=KINDS[post], norm=KINDS[norm], weight_plus=1.0, residual_scale=0.8)
        x_out, y, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((rows, 4), device="cuda")
        leaves = dict(x=x, h=h, gate=gate, weight=weight, bias=bias, post_weight=pw)

        def loss(v):
            hq.hq_gate_norm(v["x"], v["h"], v["gate"], v["weight"], v["bias"], x_out, y, stats, post_weight=v["post_weight"] if post != "none" else None, **kw)
            return ((x_out.double() * a.double()).sum() + (y.double() * b.double()).sum()).item()

        loss(leaves)
        got = dict(x=torch.empty_like(x), h=torch.empty_like(x), gate=torch.empty_like(gate), weight=torch.empty_like(gate), bias=torch.empty_like(gate),
                   post_weight=torch.empty(cols, device="cuda"))
        ws = torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")
        hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, a, b, got["x"], got["h"], got["gate"], got["weight"], got["bias"], ws,
                            post_weight=pw if post != "none" else None, dpost_weight=got["post_weight"] if post != "none" else None, **kw)
        for name, v in leaves.items():
            if name == "post_weight" and post == "none":
                continue
            way = rand(*v.shape)
            up, down = loss(dict(leaves, **{name: v + e * way})), loss(dict(leaves, **{name: v - e * way}))
            want = (got[name].double() * way.double()).sum().item()
            size = (got[name].double() * way.double()).square().sum().sqrt().item()
            noise = math.sqrt(2 * rows * cols) * 2.0 ** -21 / (2 * e)
            cubic = e * e * way.norm().item() * rows               # third derivatives along the direction, each row's of size |direction|^3 / rows
            assert abs((up - down) / (2 * e) - want) <= noise + cubic + 1e-3 * size, (name, norm, post)
