"""Calls of the operators around a transformer block's linears that their documentation allows and that are seldom made: lengths of any value,
host threads beside one another, workspaces of a larger batch, labels outside their table, gradients without elements, lists of gradients
that were let go, very many groups."""
import threading
import warnings

import pytest
import torch

from test_gpu_gate_norm import run
from train_block_reference import embedding_grad

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
LEAST, MOST = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


@pytest.mark.parametrize("norm,post", [("layer", "none"), ("rms", "rms")])
@pytest.mark.parametrize("rows,cols,per", [(300, 256, 50), (5000, 64, 1000), (33, 1152, 30), (20000, 128, 20000)])
def test_lengths_of_any_value(hq, rows, cols, per, norm, post):
    """Groups of several batches and of several teams: a length is clamped before anything is counted from it."""
    groups = -(-rows // per)
    for values in ((LEAST, MOST), (LEAST + 1, 0, LEAST + per // 2), (LEAST + per, MOST - 1, -1, LEAST + per - 1)):
        lens = torch.tensor([values[i % len(values)] for i in range(groups)], dtype=torch.int32, device="cuda")
        run(hq, rows, cols, per, norm, post, lens=lens)


def side_by_side(calls, times):
    """Every call `times` over in a host thread and on a stream of its own; what the first that failed raised."""
    failed, start = [], threading.Barrier(len(calls))

    def work(call):
        try:
            stream = torch.cuda.Stream()
            start.wait(60)
            for i in range(times):
                call(stream)
                if i % 64 == 63:
                    stream.synchronize()
            stream.synchronize()
        except Exception as e:                     # shown by the test's own thread
            failed.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    if failed:
        raise failed[0]


def gate_norm_calls(hq, cols, xt, ht):
    """Forward and gradient on buffers of their own, and the results."""
    rows, per = 64, 16
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, h, mod = rand(rows, cols).to(xt), rand(rows, cols).to(ht), 0.3 * rand(4, 3 * cols)
    gate, weight, bias = mod[:, :cols], mod[:, cols: 2 * cols], mod[:, 2 * cols:]
    x_out, y, stats, dx, dh = torch.empty_like(x), torch.empty_like(h), torch.empty((rows, 4), device="cuda"), torch.empty_like(x), torch.empty_like(h)
    dxo, dy, dmod = rand(rows, cols).to(xt), rand(rows, cols).to(ht), torch.empty_like(mod)
    ws = torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")
    kw = dict(rows_per_group=per, weight_plus=1.0)

    def call(stream):
        hq.hq_gate_norm(x, h, gate, weight, bias, x_out, y, stats, stream=stream, **kw)
        hq.hq_gate_norm_bwd(x_out, h, stats, gate, weight, dxo, dy, dx, dh, dmod[:, :cols], dmod[:, cols: 2 * cols], dmod[:, 2 * cols:], ws, stream=stream, **kw)
    return call, (x_out, y, stats, dx, dh, dmod)


@pytest.mark.parametrize("xt,ht,widths", [(BF, BF, (4096, 2048, 3000)), (F, F, (2048, 1024, 3584)), (F, BF, (4096, 1536, 2304))])
def test_gate_norm_in_host_threads(hq, xt, ht, widths):
    """Other widths of one type in other threads: none takes from a launch of another the shared memory that it asked for."""
    made = [gate_norm_calls(hq, c, xt, ht) for c in widths]
    alone = []
    for call, out in made:
        call(None)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in out])
    side_by_side([call for call, _ in made], 1500)
    assert all(torch.equal(a, b) for (_, out), want in zip(made, alone) for a, b in zip(out, want))


@pytest.mark.parametrize("sizes", [((300, 100, 2048), (300, 100, 1152), (300, 100, 1664)), ((200, 150000, 8), (200, 40000, 8), (5000, 90000, 8)),
                                   ((100, 150000, 8), (128, 40000, 8), (3, 90000, 8))])
def test_embedding_in_host_threads(hq, sizes):
    made = []
    for tokens, classes, dim in sizes:
        gen = torch.Generator(device="cuda").manual_seed(classes + dim)
        ids = torch.randint(0, classes, (tokens,), generator=gen, device="cuda").to(torch.int32)
        dout = torch.randint(-4, 5, (tokens, dim), generator=gen, device="cuda").to(BF)
        dtable = torch.empty((classes, dim), device="cuda")
        ws = torch.empty((hq.hq_embedding_bwd_workspace_size(tokens, classes, dim),), dtype=torch.uint8, device="cuda")
        made.append((lambda stream, a=(ids, dout, dtable, ws): hq.hq_embedding_bwd(*a, stream=stream), dtable, embedding_grad(ids, dout, classes, 1.0)[0]))
    side_by_side([call for call, _, _ in made], 1500)
    assert all(torch.equal(got.double(), want) for _, got, want in made)


def test_gate_norm_in_the_workspace_of_a_larger_batch(hq):
    """Of 1152 columns 7992 rows make more parts than 8192."""
    cols, per = 1152, 256
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x, dy, stats, weight = rand(8192, cols).to(BF), rand(8192, cols).to(BF), rand(8192, 4), rand(32, cols)
    largest = torch.empty((hq.hq_gate_norm_bwd_workspace_size(8192, cols, per),), dtype=torch.uint8, device="cuda")
    for rows in (8192, 7992, 7991, 5000, 33):
        groups, results = -(-rows // per), []
        for ws in (largest, torch.empty((hq.hq_gate_norm_bwd_workspace_size(rows, cols, per),), dtype=torch.uint8, device="cuda")):
            dx, dw, db = torch.empty_like(x[:rows]), torch.empty((groups, cols), device="cuda"), torch.empty((groups, cols), device="cuda")
            hq.hq_gate_norm_bwd(x[:rows], None, stats[:rows], None, weight[:groups], None, dy[:rows], dx, None, None, dw, db, ws, rows_per_group=per)
            results.append((dx, dw, db))
        assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dt", [BF, F])
def test_embedding_in_the_workspace_of_a_larger_batch(hq, dt):
    """Of 768 channels 8400 tokens make more spans than 16000."""
    classes, dim = 32768, 768
    gen = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, classes, (16000,), generator=gen, device="cuda").to(torch.int32)
    ids[torch.rand(16000, generator=gen, device="cuda") < 0.5] = 5
    dout = torch.randint(-4, 5, (16000, dim), generator=gen, device="cuda").to(dt)
    largest = torch.empty((hq.hq_embedding_bwd_workspace_size(16000, classes, dim),), dtype=torch.uint8, device="cuda")
    for tokens in (16000, 8400, 4927, 1500, 129, 100):
        dtable = torch.empty((classes, dim), device="cuda")
        hq.hq_embedding_bwd(ids[:tokens], dout[:tokens], dtable, largest)
        assert torch.equal(dtable.double(), embedding_grad(ids[:tokens], dout[:tokens], classes, 1.0)[0])


def test_gradient_of_the_class_table_with_labels_outside(hq):
    """hq_class_embed_add takes them for the first or last class: its table's gradient is that of the clamped labels; as ids they have no part."""
    classes = 11
    labels = torch.tensor([3, -1, 0, 11, 10, 3, LEAST, MOST], dtype=torch.int32, device="cuda")
    weights = torch.arange(1, 9, device="cuda").view(8, 1).expand(8, 64).to(BF).contiguous()
    ws = torch.empty((hq.hq_embedding_bwd_workspace_size(8, classes, 64),), dtype=torch.uint8, device="cuda")
    clamped, dropped = torch.empty((classes, 64), device="cuda"), torch.empty((classes, 64), device="cuda")
    hq.hq_embedding_bwd(labels.clamp(0, classes - 1), weights, clamped, ws)
    hq.hq_embedding_bwd(labels, weights, dropped, ws)
    table = torch.zeros((classes, 64), dtype=BF, device="cuda")
    for v in range(classes):
        table.zero_()
        table[v] = 1
        emb = torch.zeros((8, 64), dtype=BF, device="cuda")
        hq.hq_class_embed_add(emb, table, labels)
        assert torch.equal((emb.float() * weights.float()).sum(0), clamped[v])
    assert torch.equal(dropped.double(), embedding_grad(labels, weights, classes, 1.0)[0]) and not torch.equal(dropped, clamped)


def test_gradients_without_elements(hq):
    ws, norm = torch.empty((hq.hq_grad_workspace_size(),), dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    g = torch.full((9,), 2.0, device="cuda")
    empty = [torch.empty(s, device="cuda") for s in ((5, 0), (2, 0, 3), (0,))]
    hq.hq_grad_clip([empty[0], g, empty[1], empty[2]], 3.0, norm, ws, eps=0.0)
    assert float(norm) == 6.0 and bool((g == 1.0).all())
    out = torch.empty(9, device="cuda")
    hq.hq_grad_clip(hq.GradList([empty[0], g], [torch.empty((5, 0), device="cuda"), out]), 1.5, norm, ws, eps=0.0)
    assert float(norm) == 3.0 and bool((out == 0.5).all()) and bool((g == 1.0).all())


def test_a_list_of_gradients_that_were_let_go(hq):
    """Gradients of an earlier step in a list that was kept: the call says so.  Gradients that stay, views and copies in the list alone do not."""
    ws, norm = torch.empty((hq.hq_grad_workspace_size(),), dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    params = [torch.nn.Parameter(torch.randn(50, device="cuda")) for _ in range(3)]
    optimizer = torch.optim.SGD(params, lr=0.1)

    def backward():
        sum((p * p).sum() for p in params).backward()

    with warnings.catch_warnings():
        warnings.simplefilter("error")
        backward()
        kept = hq.GradList([p.grad for p in params])
        for _ in range(3):
            hq.hq_grad_norm(kept, norm, ws)
            hq.hq_grad_clip(kept, 1.0, norm, ws)
            optimizer.zero_grad(set_to_none=False)
            backward()
        for grads in ([p.grad.view(5, 10) for p in params], [p.grad.clone() for p in params], [p.grad.detach() for p in params]):
            other = hq.GradList(grads)
            del grads
            hq.hq_grad_clip(other, 1.0, norm, ws)
        hq.hq_grad_clip([p.grad for p in params], 1.0, norm, ws)
    optimizer.zero_grad()
    backward()
    for call in (lambda: hq.hq_grad_norm(kept, norm, ws), lambda: hq.hq_grad_clip(kept, 1.0, norm, ws)):
        with pytest.warns(RuntimeWarning, match="3 of the list's gradients"):
            call()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        hq.hq_grad_clip(hq.GradList([p.grad for p in params]), 1.0, norm, ws)
    params[1].grad = torch.ones(50, device="cuda")
    before = hq.GradList([p.grad for p in params])
    params[1].grad = None
    with pytest.warns(RuntimeWarning, match="1 of the list's gradients"):
        hq.hq_grad_clip(before, 1.0, norm, ws)


@pytest.mark.parametrize("rows,cols,per", [(500_003, 64, 3), (300_007, 128, 1), (400_001, 72, 2)])
def test_very_many_groups(hq, rows, cols, per):
    """More groups than teams by far: most are one team's, and the join takes those at the borders of two."""
    run(hq, rows, cols, per, "layer", "none")
    run(hq, rows, cols, per, "rms", "layer", F, BF)
    groups = -(-rows // per)
    lens = torch.arange(groups, dtype=torch.int32, device="cuda") % (per + 2)
    run(hq, rows, cols, per, "layer", "rms", lens=lens)
