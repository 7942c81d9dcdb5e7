"""What the calls around a transformer block's linears promise of their arguments, where no GPU is needed: workspaces of a larger batch."""
import pytest


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
