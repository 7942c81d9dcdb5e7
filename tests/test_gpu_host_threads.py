"""Calls of one kernel in several host threads, each of other sizes and on a stream of its own: none takes from a launch of another the shared
memory that it asked for, and each has the results of the call alone."""
import pytest
import torch

from paper_2512_05746_b200 import inputs
from test_gpu_train_block_calls import side_by_side

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import binding
    return binding


def check(made):
    """made: (call, outputs) of each thread."""
    alone = []
    for call, out in made:
        call(None)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in out])
        for t in out:
            t.zero_()
    side_by_side([call for call, _ in made], 1500)
    assert all(torch.equal(a, b) for (_, out), want in zip(made, alone) for a, b in zip(out, want))


@pytest.mark.parametrize("shapes,xt,yt", [(((4, 512), (4, 256), (4, 768)), F, BF), (((4, 512), (4, 256), (4, 768)), BF, BF), (((8, 320), (5, 400), (16, 128)), F, BF),
                                          (((512, 3), (1024, 3), (256, 3)), BF, F), (((768, 4), (1024, 4), (264, 4)), BF, F)])
@pytest.mark.parametrize("R,pad", [(3, 1), (1, 0)])
def test_direct_convolution(hq, shapes, xt, yt, R, pad):
    made = []
    for C, Cout in shapes:
        gen = torch.Generator(device="cuda").manual_seed(C + Cout)
        x = torch.randn((1, 6, 6, C), generator=gen, device="cuda").to(xt)
        w, y = torch.randn((Cout, R, R, C), generator=gen, device="cuda"), torch.empty((1, 6, 6, Cout), dtype=yt, device="cuda")
        made.append((lambda stream, x=x, w=w, y=y: hq.hq_conv2d_direct(x, w, None, R, 1, pad, y, stream=stream), (y,)))
    check(made)


@pytest.mark.parametrize("had_block,widths", [(4096, (16384, 12288, 4096)), (2048, (16384, 14336, 2048)), (32, (16384, 24576, 49152))])
@pytest.mark.parametrize("xt", [F, BF])
def test_quantization(hq, had_block, widths, xt):
    made = []
    for cols in widths:
        gen = torch.Generator(device="cuda").manual_seed(cols)
        x = torch.randn((20, cols), generator=gen, device="cuda").to(xt)
        codes, scales = torch.empty((20, cols), dtype=torch.uint8, device="cuda"), torch.empty((20,), device="cuda")
        made.append((lambda stream, a=(x, had_block, 4, codes, hq.HQ_CODES_INT8, scales): hq.hq_hadamard_quant(*a, stream=stream), (codes, scales)))
    check(made)


@pytest.mark.parametrize("mode,xt", [("folded", F), ("double", BF)])
def test_small_linear(hq, mode, xt):
    made = []
    for K in (1024, 768, 512):
        gen = torch.Generator(device="cuda").manual_seed(K)
        x = torch.randn((16, K), generator=gen, device="cuda").to(xt)
        pw = hq.hq_weight_prepare(inputs.weights((64, K), seed=K), 4, 256, hq.WEIGHT_MODES[mode], hq.HQ_CODES_INT8).to_device()
        y, ws = torch.empty((16, 64), dtype=BF, device="cuda"), torch.empty((hq.hq_layer_workspace_size(pw, 4, 16),), dtype=torch.uint8, device="cuda")
        made.append((lambda stream, a=(x, pw, None, 4, y, ws): hq.hq_qlinear(*a, stream=stream), (y,)))
    check(made)
