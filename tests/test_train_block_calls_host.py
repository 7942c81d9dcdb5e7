"""What the calls around a transformer block's linears promise of their arguments, where no GPU is needed: workspaces of a larger batch, outputs
in place, gradients without elements, clipping without a norm."""
import pytest
import torch

from test_train_block_host import ALIGNMENT, HALF, SHAPE, C, norm, norm_bwd


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import build
    build.build()
    from paper_2512_05746_b200 import binding
    return binding


def sizes_up_to(most):
    """All small numbers, then some of every size, both sides of multiples among them."""
    some = set(range(0, 3000))
    n = 3000
    while n < most:
        some |= {n - 1, n, n + 1, n // 512 * 512, n // 128 * 128 + 1}
        n += max(7, n // 60)
    return sorted(some) + [most]


@pytest.mark.parametrize("cols", [8, 64, 72, 128, 136, 256, 512, 1000, 1152, 1280, 2304, 4096])
def test_a_workspace_of_the_gated_residual_does_for_fewer_rows(hq, cols):
    for per in (0, 1, 77):
        sizes = [hq.hq_gate_norm_bwd_workspace_size(rows, cols, per) for rows in sizes_up_to(600_000)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("classes,dim", [(2, 8), (7, 64), (1001, 64), (50, 320), (1001, 1152), (32768, 768), (300, 2048), (300, 2056), (9, 16384), (11, 65536)])
def test_a_workspace_of_the_embedding_does_for_fewer_tokens(hq, classes, dim):
    sizes = [hq.hq_embedding_bwd_workspace_size(tokens, classes, dim) for tokens in sizes_up_to(600_000)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))


AT = [C.c_void_p(0x100000 * (i + 1)) for i in range(8)]        # never read: every call is refused, the last check's of `stats` where no other does


def test_in_place_with_another_pitch(hq):
    """Rows written at other places than they are read from lie on rows that another thread block still has to read."""
    apart = dict(x=AT[0], h=AT[1], x_out=AT[2], y=AT[3], stats=HALF)
    assert norm(hq, **apart, ldx_out=72, ldy=72) == norm(hq, **dict(apart, x_out=AT[0], y=AT[1])) == ALIGNMENT
    for change in (dict(x_out=AT[0], ldx_out=72), dict(x_out=AT[0], ldx=72), dict(y=AT[1], ldy=128), dict(y=AT[1], ldh=80)):
        assert norm(hq, **dict(apart, **change)) == SHAPE, change
        assert norm(hq, **dict(apart, rows=1, per=1, **change)) == ALIGNMENT, change
    apart = dict(x=AT[0], h=AT[1], dx_out=AT[2], dy=AT[3], dx=AT[4], dh=AT[5], stats=HALF)
    assert norm_bwd(hq, **apart, lddx=72, lddh=72) == ALIGNMENT
    for same in (dict(dx=AT[2]), dict(dh=AT[3]), dict(dh=AT[1])):
        assert norm_bwd(hq, **dict(apart, **same)) == ALIGNMENT
    for change in (dict(dx=AT[2], lddx=72), dict(dh=AT[3], lddh=72), dict(dh=AT[1], ldh=72), dict(dh=AT[3], lddy=128)):
        assert norm_bwd(hq, **dict(apart, **change)) == SHAPE, change
        assert norm_bwd(hq, **dict(apart, rows=1, per=1, **change)) == ALIGNMENT, change


def test_layouts_of_gradients(hq):
    """A tensor without elements has a dense layout whatever its strides; others by their strides."""
    for shape in ((0,), (0, 5), (5, 0), (2, 0, 3), (3, 2, 0, 4)):
        assert hq._is_dense(torch.empty(shape)) and hq._is_dense(torch.empty(shape).transpose(0, -1)), shape
    t = torch.empty((4, 6, 5))
    assert hq._is_dense(t) and hq._is_dense(t.permute(2, 0, 1)) and hq._is_dense(t[1:3]) and hq._is_dense(t[:0]) and hq._is_dense(t[:, :1][:1])
    assert not any(hq._is_dense(v) for v in (t[::2], t[:, 1:], t[..., :4], t[:1].expand(4, 6, 5)))


def test_clipping_by_no_norm(hq):
    """None, an option that was not set, is refused: it would leave the gradients as they are."""
    norm, ws = torch.zeros(1), torch.zeros(hq.hq_grad_workspace_size(), dtype=torch.uint8)
    with pytest.raises(TypeError):
        hq.hq_grad_clip([], None, norm, ws)
