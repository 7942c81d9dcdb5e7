"""The embedding lookup with scaling, and the gradient of its table by sorted tokens, against 64-bit arithmetic."""
import math

import pytest
import torch

from train_block_reference import F32, embedding_grad, unit

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


def tokens_of(T, V, how, gen):
    """Token ids: all over the table and beyond it on both sides, half of one id, or all of one id."""
    ids = torch.randint(-2, V + 2, (T,), generator=gen, device="cuda")
    if how == "half":
        ids[torch.rand(T, generator=gen, device="cuda") < 0.5] = V // 2
    elif how == "one":
        ids.fill_(V - 1)
    elif how == "outside":
        ids.fill_(V)
    elif how == "runs":
        ids = (torch.arange(T, device="cuda") // 40) % V
    return ids


@pytest.mark.parametrize("tt,ot", [(BF, BF), (F, BF), (BF, F), (F, F)])
@pytest.mark.parametrize("T,V,dim", [(1, 1, 8), (64, 1001, 1152), (1000, 50, 64), (333, 7, 2048), (40, 9, 2056), (77, 100, 5000), (5000, 3000, 200)])
def test_lookup(hq, T, V, dim, tt, ot):
    gen = torch.Generator(device="cuda").manual_seed(T + dim)
    store = torch.randn((V, dim + 8), generator=gen, device="cuda").to(tt)
    store[:, dim:] = math.nan
    table = store[:, :dim]
    for dtype in (torch.int32, torch.int64):
        ids = tokens_of(T, V, "all", gen).to(dtype)
        if dtype == torch.int64 and T > 2:
            ids[1], ids[2] = 2 ** 40 + 1, -2 ** 40             # no id modulo 2^32
        room = torch.full((T, dim + 16), math.nan, dtype=ot, device="cuda")
        hq.hq_embedding(ids, table, room[:, :dim], scale=1.7)
        ok = (ids >= 0) & (ids < V)
        want = torch.where(ok[:, None], table.double()[ids.clamp(0, V - 1).long()], torch.zeros((), dtype=torch.float64, device="cuda")) * 1.7
        # one product in fp32 (the scale is rounded to it, too), one rounding
        assert bool(((room[:, :dim].double() - want).abs() <= (unit(ot) + 3 * F32) * want.abs()).all())
        assert bool(room[:, dim:].isnan().all())


def grad(hq, ids, dout, V, dtable_type, scale=1.7, base=None, into=None):
    T, dim = ids.numel(), dout.shape[-1]
    ws = torch.empty((hq.hq_embedding_bwd_workspace_size(T, V, dim),), dtype=torch.uint8, device="cuda").fill_(0xFF)
    dtable = torch.full((V, dim), math.nan, dtype=dtable_type, device="cuda") if into is None else into
    hq.hq_embedding_bwd(ids, dout, dtable, ws, scale=scale, base=base)
    return dtable


def check(hq, T, V, dim, how, dt, gt, dtype=torch.int32, with_base=False, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(T + dim + V + seed)
    ids = tokens_of(T, V, how, gen).to(dtype)
    store = torch.randn((T, dim + 8), generator=gen, device="cuda").to(dt)
    dout = store[:, :dim]
    base = torch.randn((V, dim), generator=gen, device="cuda").to(gt) if with_base else None
    want, size = embedding_grad(ids, dout, V, 1.7, base)
    got = grad(hq, ids, dout, V, gt, base=base)
    most = int(torch.bincount(ids[(ids >= 0) & (ids < V)].long(), minlength=1).max()) if T else 0
    # a sum of `most` terms at worst, in fp32, then scale and base: each step half a rounding of the sum so far
    bound = unit(gt) * want.abs() + (8 + 2 * math.sqrt(most) + most / 16) * F32 * size
    assert bool(((got.double() - want).abs() <= bound).all())
    assert torch.equal(got, grad(hq, ids, dout, V, gt, base=base))             # the same bits
    if with_base:                                  # in place
        assert torch.equal(got, grad(hq, ids, dout, V, gt, base=base, into=base))
    return got


@pytest.mark.parametrize("dt,gt", [(BF, BF), (F, BF), (BF, F), (F, F)])
@pytest.mark.parametrize("how", ["all", "half", "one", "runs", "outside"])
@pytest.mark.parametrize("T,V,dim", [(1, 1, 8), (64, 1001, 1152), (1000, 50, 64), (3000, 7, 2056), (2500, 300000, 16), (33, 2, 5000), (128, 40, 320), (129, 40, 320), (100, 9, 16384)])
def test_gradient(hq, T, V, dim, how, dt, gt):
    check(hq, T, V, dim, how, dt, gt)
    check(hq, T, V, dim, how, dt, gt, torch.int64, with_base=True)


@pytest.mark.parametrize("T,V,dim,how", [(20011, 32768, 768, "half"), (100003, 1001, 64, "all"), (65536, 3, 128, "all"), (131072, 150000, 64, "half"),
                                         (30000, 1, 1152, "one"), (40000, 5000, 320, "runs")])
def test_gradient_of_many_tokens(hq, T, V, dim, how):
    check(hq, T, V, dim, how, BF, BF)
    check(hq, T, V, dim, how, BF, F, torch.int64, with_base=True)


@pytest.mark.parametrize("T", [1, 100, 1000, 4096, 4097, 9000])
def test_every_size_of_the_counters(hq, T):
    """Slices of the ids of every size up to the largest: shared memory on both sides of what a kernel has without asking."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    dout = torch.randint(-4, 5, (T, 8), generator=gen, device="cuda").to(BF)
    for slice_of in list(range(1, 256, 3)) + list(range(256, 1030, 51)):
        ids = torch.randint(0, 148 * slice_of, (T,), generator=gen, device="cuda").to(torch.int32)
        assert torch.equal(grad(hq, ids, dout, 148 * slice_of, F, scale=1.0).double(), embedding_grad(ids, dout, 148 * slice_of, 1.0)[0])


@pytest.mark.parametrize("n", list(range(1, 80, 3)) + [127, 128, 129, 1023, 1024, 1025])
def test_runs_at_the_borders_of_spans(hq, n):
    """Ids of n tokens each, and one of n between others: sums that end, begin and go on at every place of a span."""
    V, dim = 40, 64
    gen = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.repeat_interleave(torch.arange(V, device="cuda"), torch.tensor([n if v % 3 else (v % 7) for v in range(V)], device="cuda"))
    ids = ids[torch.randperm(ids.numel(), generator=gen, device="cuda")].to(torch.int32)
    dout = torch.randint(-8, 9, (ids.numel(), dim), generator=gen, device="cuda").to(BF)          # whole numbers: every order gives the sum itself
    assert torch.equal(grad(hq, ids, dout, V, F, scale=1.0).double(), embedding_grad(ids, dout, V, 1.0)[0])


def test_no_tokens(hq):
    base = torch.randn((30, 64), device="cuda").to(BF)
    ids, dout = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 64), dtype=BF, device="cuda")
    assert bool((grad(hq, ids, dout, 30, BF) == 0).all()) and torch.equal(grad(hq, ids, dout, 30, BF, base=base), base)
    hq.hq_embedding(ids, base, dout)


def test_shapes_of_ids(hq):
    table, ids = torch.randn((100, 64), device="cuda"), torch.randint(0, 100, (6, 7), device="cuda")
    out = torch.empty((6, 7, 64), device="cuda")
    hq.hq_embedding(ids, table, out, scale=0.5)
    assert torch.equal(out, table[ids] * 0.5)
    dtable = torch.empty_like(table)
    ws = torch.empty((hq.hq_embedding_bwd_workspace_size(42, 100, 64),), dtype=torch.uint8, device="cuda")
    hq.hq_embedding_bwd(ids, out, dtable, ws)
    want, size = embedding_grad(ids, out, 100, 1.0)
    assert bool(((dtable.double() - want).abs() <= 16 * F32 * size).all())
    with pytest.raises(ValueError):
        hq.hq_embedding(ids, table, out.view(7, 6, 64))


def test_gradient_of_the_class_table(hq):
    """The gradient of what hq_class_embed_add adds: differences of its own results, exact where every number is whole."""
    table, labels = torch.zeros((11, 64), dtype=BF, device="cuda"), torch.tensor([3, 0, 10, 3], dtype=torch.int32, device="cuda")
    weights = torch.randint(-4, 5, (4, 64), device="cuda").to(BF)
    ws = torch.empty((hq.hq_embedding_bwd_workspace_size(4, 11, 64),), dtype=torch.uint8, device="cuda")
    dtable = torch.empty((11, 64), device="cuda")
    hq.hq_embedding_bwd(labels, weights, dtable, ws)
    for v in range(11):
        table.zero_()
        table[v] = 1
        emb = torch.zeros((4, 64), dtype=BF, device="cuda")
        hq.hq_class_embed_add(emb, table, labels)
        assert torch.equal((emb.float() * weights.float()).sum(0), dtable[v])
