"""The norm of all gradients and clipping by it, against 64-bit arithmetic."""
import math

import pytest
import torch

from train_block_reference import F32, unit

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


@pytest.fixture(scope="module")
def ws(hq):
    return torch.empty((hq.hq_grad_workspace_size(),), dtype=torch.uint8, device="cuda").fill_(0xFF)


def norm_of(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check(hq, ws, grads, max_norm, outs=None):
    want = norm_of(grads)
    before = [g.clone() for g in grads]
    factor = min(1.0, max_norm / (want + EPS))
    norm, coef, alone = (torch.full((1,), math.nan, device="cuda") for _ in range(3))
    listed = hq.GradList(grads, outs)
    hq.hq_grad_norm(listed, alone, ws)
    hq.hq_grad_clip(listed, max_norm, norm, ws, eps=EPS, coef=coef)
    # 8 squares in fp32 (4 roundings each in the worst order), the rest in fp64, one rounding
    assert abs(float(norm) - want) <= 8 * F32 * want and torch.equal(norm, alone)
    assert abs(float(coef) - factor) <= 10 * F32 * factor
    for b, g, o in zip(before, grads, grads if outs is None else outs):
        ref = b.double() * factor
        assert bool(((o.double() - ref).abs() <= (unit(o.dtype) + 12 * F32) * ref.abs() + 2.0 ** -149).all())
        assert outs is None or torch.equal(b, g)
        if factor == 1.0 and o.dtype == b.dtype:
            assert torch.equal(o, b)


def tensors(sizes, dtypes, gen, offset=0):
    """Dense tensors `offset` elements behind a 16-byte border, with room behind them that nothing may write."""
    rooms = [torch.full((n + offset + 9,), 7.0, dtype=dtypes[i % len(dtypes)], device="cuda") for i, n in enumerate(sizes)]
    for r, n, i in zip(rooms, sizes, range(len(sizes))):
        r[offset: offset + n] = (torch.randn(n, generator=gen, device="cuda") * 10.0 ** -(i % 5)).to(r.dtype)
    return rooms, [r[offset: offset + n] for r, n in zip(rooms, sizes)]


@pytest.mark.parametrize("offset", [0, 1, 3, 4, 5])
@pytest.mark.parametrize("dtypes", [(F,), (BF,), (F, BF)])
@pytest.mark.parametrize("sizes", [(1,), (7, 8, 9), (2048, 2047, 2049, 5000), (0, 3, 0, 100000, 0), tuple(range(1, 300, 7))])
def test_against_64_bits(hq, ws, sizes, dtypes, offset):
    gen = torch.Generator(device="cuda").manual_seed(len(sizes) + offset)
    for max_norm in (0.5, 1e9, math.inf, 0.0):
        rooms, grads = tensors(sizes, dtypes, gen, offset)
        check(hq, ws, grads, max_norm)
        for other in ((BF,), (F,), (BF, F)):
            outs_room, outs = tensors(sizes, other, gen, (offset * 2) % 7)
            check(hq, ws, grads, max_norm, outs)
            for r, n in list(zip(rooms, sizes)) + [(q, n + (offset * 2) % 7 - offset) for q, n in zip(outs_room, sizes)]:
                assert bool((r[n + offset:] == 7).all())
            for r, o in ((rooms, offset), (outs_room, (offset * 2) % 7)):
                assert all(bool((t[:o] == 7).all()) for t in r)


@pytest.mark.parametrize("n", [31, 32, 33, 256, 257, 1087, 1088, 1089, 1099, 1100, 1101, 2300, 6001])
def test_numbers_of_tensors(hq, ws, n):
    gen = torch.Generator(device="cuda").manual_seed(n)
    flat = torch.randn(n * 40, generator=gen, device="cuda")
    grads = [flat[i * 40: i * 40 + 1 + (i * 7) % 40] for i in range(n)]
    check(hq, ws, grads, 3.0)


def test_large(hq, ws):
    gen = torch.Generator(device="cuda").manual_seed(1)
    _, grads = tensors((40_000_003, 17, 9_999_999), (BF, F), gen)
    check(hq, ws, grads, 1.0, [torch.empty(g.shape, device="cuda") for g in grads])
    check(hq, ws, grads, 1.0)


def test_no_gradients(hq, ws):
    check(hq, ws, [], 1.0)
    check(hq, ws, [torch.empty((0, 5), device="cuda")], 1.0)
    check(hq, ws, [torch.zeros((100, 5), device="cuda")], 1.0)


@pytest.mark.parametrize("size", [1e-44, 1e-30, 1e-21, 1e-17, 1e-5, 1e17, 1e25, 3e38])
def test_range(hq, ws, size):
    """Squares that fp32 does not hold."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = torch.rand(5000, generator=gen, device="cuda") * size
    if size == 1e17:                               # both ends in one tensor
        g[::16] = 1e-30
    norm = torch.empty(1, device="cuda")
    hq.hq_grad_norm([g], norm, ws)
    want = norm_of([g])
    assert abs(float(norm) - want) <= 8 * F32 * want + 2.0 ** -149 if want < 3.4e38 else math.isinf(float(norm))


def test_not_finite(hq, ws):
    for bad, coef_wanted in ((math.inf, 0.0), (math.nan, math.nan)):
        g, h = torch.ones(3000, device="cuda"), torch.ones(50, dtype=BF, device="cuda")
        g[1234] = bad
        norm, coef = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        hq.hq_grad_clip([g, h], 1.0, norm, ws, coef=coef)
        assert not math.isfinite(float(norm)) and (float(coef) == coef_wanted or math.isnan(coef_wanted) and math.isnan(float(coef)))
        if coef_wanted == 0.0:
            assert bool((h == 0).all()) and math.isnan(float(g[1234])) and float(g.nan_to_num().abs().max()) == 0.0
        else:
            assert bool(h.isnan().all()) and bool(g.isnan().all())


def test_layouts_and_same_bits(hq, ws):
    gen = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    grads = [rand(64, 48).t(), rand(8, 3, 3, 16).permute(0, 3, 1, 2), rand(5), rand(1, 7, 1), torch.tensor(2.5, device="cuda")]
    check(hq, ws, [g.clone(memory_format=torch.preserve_format) for g in grads], 2.0)
    results = []
    for _ in range(2):
        copies = [g.clone(memory_format=torch.preserve_format) for g in grads] + [rand(1), ]
        copies[-1].fill_(0.125)
        norm = torch.empty(1, device="cuda")
        hq.hq_grad_clip(copies, 2.0, norm, ws)
        results.append([norm] + copies)
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_refuses(hq, ws):
    g, norm = torch.ones(100, device="cuda"), torch.empty(1, device="cuda")
    for bad in ([g[::2]], [g, g], [g, g[50:]], [g.cpu()], [torch.ones((4, 4), device="cuda").expand(3, 4, 4)]):
        with pytest.raises(ValueError):
            hq.GradList(bad)
    with pytest.raises(TypeError):
        hq.GradList([g.half()])
    for outs in ([g[:50]], [g.view(10, 10)], [], [torch.ones(100)], [g.view(torch.int32)], [torch.as_strided(g, (100,), (1,), 0).view(BF)[:100]]):
        with pytest.raises((ValueError, TypeError)):
            hq.GradList([g], outs)
    with pytest.raises(ValueError):
        hq.GradList([g[:50], g[50:]], [torch.ones(50, device="cuda"), g[:50]])         # one's output is the other's gradient
    hq.GradList([g[:50], g[50:]], [g[:50], torch.ones(50, device="cuda")])
    for bad in (dict(norm=torch.empty(2, device="cuda")), dict(norm=torch.empty(1)), dict(ws=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            hq.hq_grad_clip([g], 1.0, bad.get("norm", norm), bad.get("ws", ws))
    for max_norm, eps in ((-1.0, 0.0), (math.nan, 0.0), (1.0, -1.0)):
        with pytest.raises(hq.HqError):
            hq.hq_grad_clip([g], max_norm, norm, ws, eps=eps)
    with pytest.raises(hq.HqError):
        hq.hq_grad_clip([g], 1.0, norm, ws[:100])
    assert bool((g == 1).all())
