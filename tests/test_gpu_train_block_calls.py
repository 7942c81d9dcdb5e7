"""Calls of the operators around a transformer block's linears that their documentation allows and that come seldom: lengths of any value."""
import pytest
import torch

from test_gpu_gate_norm import run

pytestmark = pytest.mark.gpu
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
