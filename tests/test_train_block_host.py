"""Refusals of the gated residual with its norms, of the embedding and of gradient clipping, before anything reaches a GPU: the C entry points
on addresses that are never read, and the binding on tensors of other shapes, types and devices; and the formulas the GPU tests compare with,
against torch's differentiation and against differences."""
import ctypes as C

import pytest
import torch

from train_block_reference import backward, embedding_grad, forward

OK, INVALID, SHAPE, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4, 5
FAKE, ODD, HALF = C.c_void_p(0x1000), C.c_void_p(0x1004), C.c_void_p(0x1008)
LAYER, RMS, NONE = 0, 1, 2
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import build
    build.build()
    from paper_2512_05746_b200 import binding
    return binding


def norm(hq, **change):
    a = dict(x=FAKE, ldx=64, xdt=1, h=FAKE, ldh=64, hdt=1, rows=8, cols=64, per=4, lens=None, post=NONE, post_weight=None, gate=FAKE, ld_gate=64,
             residual=1.0, norm=LAYER, weight=FAKE, ld_weight=64, bias=FAKE, ld_bias=64, plus=1.0, eps=1e-6, x_out=FAKE, ldx_out=64, y=FAKE,
             ldy=64, stats=None, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_gate_norm(*a.values())


def norm_bwd(hq, **change):
    a = dict(x=FAKE, ldx=64, xdt=1, h=FAKE, ldh=64, hdt=1, stats=FAKE, rows=8, cols=64, per=4, lens=None, post=NONE, post_weight=None, gate=FAKE,
             ld_gate=64, residual=1.0, norm=LAYER, weight=FAKE, ld_weight=64, plus=1.0, dx_out=FAKE, lddx_out=64, dy=FAKE, lddy=64, dx=FAKE,
             lddx=64, dh=FAKE, lddh=64, dpost=None, dgate=FAKE, ld_dgate=64, dweight=FAKE, ld_dweight=64, dbias=FAKE, ld_dbias=64, ws=FAKE,
             ws_bytes=1 << 30, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_gate_norm_bwd(*a.values())


@pytest.mark.parametrize("call", [norm, norm_bwd])
@pytest.mark.parametrize("change,want", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=-8), SHAPE), (dict(per=-1), SHAPE), (dict(cols=60), UNSUPPORTED),
    (dict(cols=4104, ldx=4104, ldh=4104), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(xdt=2), INVALID), (dict(hdt=-1), INVALID),
    (dict(post=3), INVALID), (dict(norm=-1), INVALID), (dict(per=0, lens=FAKE), INVALID), (dict(post_weight=FAKE), INVALID),
    (dict(post=RMS, post_weight=ODD), ALIGNMENT), (dict(residual=NAN), INVALID), (dict(residual=INF), INVALID), (dict(plus=NAN), INVALID),
    (dict(h=None), INVALID), (dict(h=None, gate=None, residual=0.5), INVALID), (dict(h=None, gate=None, post=RMS), INVALID),
    (dict(x=None), INVALID), (dict(x=HALF), ALIGNMENT), (dict(h=HALF), ALIGNMENT), (dict(ldx=56), SHAPE), (dict(ldh=60), SHAPE), (dict(ldx=68), ALIGNMENT),
    (dict(xdt=0, ldx=66), ALIGNMENT), (dict(ldx=1 << 30), UNSUPPORTED), (dict(ldh=1 << 33), UNSUPPORTED), (dict(gate=HALF), ALIGNMENT), (dict(ld_gate=60), SHAPE), (dict(ld_gate=66), ALIGNMENT),
    (dict(weight=ODD), ALIGNMENT), (dict(ld_weight=0), SHAPE), (dict(stats=HALF), ALIGNMENT)])
def test_gate_norm_refuses(hq, call, change, want):
    assert call(hq, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(rows=0), OK), (dict(rows=0, x=None, h=FAKE), OK), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(y=None), INVALID),
    (dict(norm=NONE), INVALID), (dict(norm=NONE, y=None), INVALID), (dict(norm=NONE, y=None, weight=None), INVALID),
    (dict(norm=NONE, y=None, weight=None, bias=None, x_out=None), INVALID), (dict(x_out=HALF), ALIGNMENT), (dict(ldx_out=8), SHAPE),
    (dict(ldy=66), ALIGNMENT), (dict(bias=HALF), ALIGNMENT), (dict(ld_bias=63), SHAPE)])
def test_gate_norm_s_own(hq, change, want):
    assert norm(hq, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(rows=0), OK), (dict(dy=None), INVALID), (dict(norm=NONE), INVALID), (dict(norm=NONE, dy=None, weight=None, dweight=None, dbias=None, dx_out=None), INVALID),
    (dict(norm=NONE, dy=None), INVALID), (dict(h=None, gate=None), INVALID), (dict(h=None, gate=None, dgate=None), INVALID), (dict(dpost=FAKE), INVALID),
    (dict(stats=None), INVALID), (dict(dx_out=HALF), ALIGNMENT), (dict(lddx=66), ALIGNMENT), (dict(lddh=32), SHAPE), (dict(dgate=HALF), ALIGNMENT),
    (dict(ld_dweight=32), SHAPE), (dict(ld_dbias=66), ALIGNMENT), (dict(post=RMS, dpost=HALF), ALIGNMENT), (dict(rows=1000, per=500, ws=None), INVALID),
    (dict(rows=1000, per=500, ws=HALF), ALIGNMENT), (dict(rows=1000, per=500, ws_bytes=64), WORKSPACE), (dict(post=RMS, dpost=FAKE, ws=None), INVALID)])
def test_gate_norm_gradient_s_own(hq, change, want):
    assert norm_bwd(hq, **change) == want


def embed(hq, **change):
    a = dict(ids=FAKE, id_bytes=4, tokens=5, table=FAKE, tdt=1, classes=10, dim=64, ld=64, scale=1.0, out=FAKE, odt=1, ldo=64, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_embedding(*a.values())


def embed_bwd(hq, **change):
    a = dict(ids=FAKE, id_bytes=4, tokens=5, out=FAKE, odt=1, ldo=64, classes=10, dim=64, scale=1.0, base=None, ld_base=64, table=FAKE, tdt=1, ld=64,
             ws=FAKE, ws_bytes=1 << 30, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_embedding_bwd(*a.values())


@pytest.mark.parametrize("call", [embed, embed_bwd])
@pytest.mark.parametrize("change,want", [
    (dict(tokens=-1), SHAPE), (dict(classes=0), SHAPE), (dict(dim=0), SHAPE), (dict(dim=60), UNSUPPORTED), (dict(dim=65544, ld=65544, ldo=65544), UNSUPPORTED),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(classes=1 << 31), UNSUPPORTED), (dict(id_bytes=2), INVALID), (dict(tdt=2), INVALID), (dict(odt=7), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(ids=None), INVALID), (dict(table=None), INVALID), (dict(out=None), INVALID),
    (dict(ids=C.c_void_p(0x1002)), ALIGNMENT), (dict(id_bytes=8, ids=ODD), ALIGNMENT), (dict(table=HALF), ALIGNMENT), (dict(out=HALF), ALIGNMENT),
    (dict(ld=56), SHAPE), (dict(ldo=0), SHAPE), (dict(ldo=68), ALIGNMENT), (dict(ld=1 << 30), UNSUPPORTED), (dict(ldo=1 << 32), UNSUPPORTED)])
def test_embedding_refuses(hq, call, change, want):
    assert call(hq, **change) == want


def test_embedding_s_own(hq):
    assert embed(hq, tokens=0, ids=None, table=None, out=None) == OK
    for change, want in ((dict(base=HALF), ALIGNMENT), (dict(base=FAKE, ld_base=32), SHAPE), (dict(base=FAKE, ld_base=72), SHAPE), (dict(ws=None), INVALID),
                         (dict(ws=HALF), ALIGNMENT), (dict(ws_bytes=64), WORKSPACE), (dict(tokens=0, table=None), INVALID)):
        assert embed_bwd(hq, **change) == want, change


class Tensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("count", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32)]


@pytest.mark.parametrize("change,want", [
    (dict(n=-1), SHAPE), (dict(tensors=None), INVALID), (dict(norm=None), INVALID), (dict(ws=None), INVALID), (dict(norm=C.c_void_p(0x1002)), ALIGNMENT),
    (dict(ws=ODD), ALIGNMENT), (dict(ws_bytes=100), WORKSPACE), (dict(max_norm=-1.0), INVALID), (dict(max_norm=NAN), INVALID), (dict(eps=-1.0), INVALID),
    (dict(coef=C.c_void_p(0x1001)), ALIGNMENT), (dict(count=-1), SHAPE), (dict(count=(1 << 40) + 1), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(grad=None), INVALID), (dict(grad=0x1002), ALIGNMENT), (dict(grad=0x1001, dtype=1), ALIGNMENT), (dict(out=0x2002), ALIGNMENT),
    (dict(out=0x2000, out_dtype=5), INVALID), (dict(out=0x1000, out_dtype=1), INVALID)])
def test_clipping_refuses(hq, change, want):
    t = dict(grad=0x1000, out=None, count=5, dtype=0, out_dtype=0)
    a = dict(tensors=(Tensor * 1)(Tensor(**{k: change.get(k, v) for k, v in t.items()})), n=1, max_norm=1.0, eps=1e-6, norm=FAKE, coef=None, ws=FAKE,
             ws_bytes=1 << 20, stream=None)
    assert not set(change) - set(a) - set(t)
    a.update({k: v for k, v in change.items() if k in a})
    assert hq.lib.hq_grad_clip(*a.values()) == want
    if not set(change) & {"max_norm", "eps", "coef"}:
        assert hq.lib.hq_grad_norm(a["tensors"], a["n"], a["norm"], a["ws"], a["ws_bytes"], None) == want


def test_workspace_sizes(hq):
    assert hq.hq_gate_norm_bwd_workspace_size(1, 8, 0) >= 7 * 8 * 4 and hq.hq_gate_norm_bwd_workspace_size(0, 8, 0) == 0
    assert hq.hq_embedding_bwd_workspace_size(100, 10, 64) >= 100 * 8 + 11 * 4
    assert hq.hq_embedding_bwd_workspace_size(0, 10, 64) >= 11 * 4
    for bad in ((-1, 8, 0), (1, 4104, 0), (1, 12, 0), (1, 8, -1)):
        with pytest.raises(hq.HqError):
            hq.hq_gate_norm_bwd_workspace_size(*bad)
    for bad in ((-1, 10, 64), (1, 0, 64), (1, 10, 60)):
        with pytest.raises(hq.HqError):
            hq.hq_embedding_bwd_workspace_size(*bad)
    assert hq.hq_grad_workspace_size() > 0
    assert hq.lib.hq_grad_workspace_size(None) == hq.lib.hq_gate_norm_bwd_workspace_size(1, 8, 0, None) == hq.lib.hq_embedding_bwd_workspace_size(1, 1, 8, None) == INVALID


def test_binding_refuses(hq):
    x, vec, bf = torch.zeros((8, 64)), torch.zeros((2, 64)), torch.bfloat16
    for bad in (dict(h=x[:4]), dict(h=x.t()), dict(gate=vec[:1]), dict(weight=vec.to(bf)), dict(bias=torch.zeros((2, 32))), dict(x_out=x.to(bf)),
                dict(y=x.to(bf)), dict(stats=torch.zeros((8, 3))), dict(lens=torch.zeros(2)), dict(lens=torch.zeros(3, dtype=torch.int32)),
                dict(post_weight=torch.zeros(32)), dict(per=-4), dict(per=0), dict(x=None), dict(gate=torch.zeros(64)), dict()):
        a = dict(dict(x=x, h=x, gate=vec, weight=vec, bias=vec, x_out=x, y=x, stats=None, per=4, lens=None, post_weight=None), **bad)
        with pytest.raises(ValueError):            # the last: everything fits, but the tensors are the host's
            hq.hq_gate_norm(a["x"], a["h"], a["gate"], a["weight"], a["bias"], a["x_out"], a["y"], a["stats"], rows_per_group=a["per"], lens=a["lens"],
                            post_weight=a["post_weight"])
    for bad in (dict(dy=x[:4]), dict(dx=x.to(bf)), dict(dh=x.to(bf)), dict(dgate=vec[:1]), dict(stats=None, dx_out=x.t()), dict(dweight=vec.double()), dict()):
        a = dict(dict(x_out=x, h=x, stats=torch.zeros((8, 4)), dx_out=x, dy=x, dx=x, dh=x, dgate=vec, dweight=vec, dbias=vec), **bad)
        with pytest.raises(ValueError):
            hq.hq_gate_norm_bwd(a["x_out"], a["h"], a["stats"], vec, vec, a["dx_out"], a["dy"], a["dx"], a["dh"], a["dgate"], a["dweight"], a["dbias"],
                                None, rows_per_group=4)
    with pytest.raises(TypeError):
        hq.hq_gate_norm(x.half(), None, None, None, None, None, x.half())
    with pytest.raises(OverflowError):
        hq.hq_gate_norm(x, x, None, None, None, x, x, norm=1 << 32)
    ids, table, out = torch.zeros(8, dtype=torch.int32), torch.zeros((10, 64)), torch.zeros((8, 64))
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (dict(ids=ids.float()), dict(ids=ids[:4]), dict(ids=torch.zeros(16, dtype=torch.int32)[::2]), dict(out=out[:, :32]), dict(out=out.t()),
                dict(table=table[:, ::2]), dict(ids=ids.view(2, 4)), dict()):
        a = dict(dict(ids=ids, table=table, out=out), **bad)
        with pytest.raises(ValueError):
            hq.hq_embedding(a["ids"], a["table"], a["out"])
        with pytest.raises(ValueError):
            hq.hq_embedding_bwd(a["ids"], a["out"], a["table"], ws)
    with pytest.raises(ValueError):
        hq.hq_embedding_bwd(ids, out, table, ws, base=table.to(bf))
    with pytest.raises(ValueError):
        hq.GradList([x])                           # the host's


@pytest.mark.parametrize("kind,post", [("layer", "none"), ("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("none", "none")])
@pytest.mark.parametrize("per", [0, 4, 5])
def test_the_formula_of_the_gradient(kind, post, per):
    """The formula's gradient (from the statistics) is torch's of the forward formula."""
    gen = torch.Generator().manual_seed(per + len(kind))
    rows, cols, groups = 13, 24, -(-13 // per) if per else 1
    rand = lambda *s: torch.randn(s, generator=gen, dtype=torch.float64)  # noqa: E731
    names = ["x", "h", "gate", "weight", "bias", "post_weight"]
    leaves = dict(zip(names, (rand(rows, cols), rand(rows, cols), rand(groups, cols), rand(groups, cols), rand(groups, cols), rand(cols))))
    for v in leaves.values():
        v.requires_grad_()
    pw = leaves["post_weight"] if post != "none" else None
    out, y, stats, _, _ = forward(leaves["x"], leaves["h"], leaves["gate"], leaves["weight"], leaves["bias"], per, post, pw, kind, 1.0, 0.7)
    a, b = rand(rows, cols), rand(rows, cols)
    loss = (out * a).sum() + ((y * b).sum() if y is not None else 0.0)
    used = [n for n in names if (kind != "none" or n not in ("weight", "bias")) and (post != "none" or n != "post_weight")]
    want = dict(zip(used, torch.autograd.grad(loss, [leaves[n] for n in used])))
    leaves = {n: v.detach() for n, v in leaves.items()}
    found = backward(out.detach(), leaves["h"], stats.detach(), leaves["gate"], leaves["weight"], a, b if y is not None else None, per, None, post,
                     pw.detach() if pw is not None else None, kind, 1.0, 0.7)
    for n in used:
        assert torch.allclose(found["d" + n][0], want[n], rtol=1e-10, atol=1e-12), n


def test_the_formula_of_the_embedding_s_gradient():
    gen = torch.Generator().manual_seed(1)
    table, ids = torch.randn((9, 8), generator=gen, dtype=torch.float64, requires_grad=True), torch.randint(0, 9, (40,), generator=gen)
    a = torch.randn((40, 8), generator=gen, dtype=torch.float64)
    want, = torch.autograd.grad((table[ids] * 1.5 * a).sum(), table)
    assert torch.allclose(embedding_grad(ids, a, 9, 1.5)[0], want, rtol=1e-12)
