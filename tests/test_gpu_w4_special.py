"""Making 4-bit matrices from values that are no ordinary numbers."""
import numpy as np
import pytest
import torch

from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_groups_that_are_not_finite_stay_so(bad, dtype):
    """NaN or an infinity in a group makes its scale not finite and all its weights
    NaN, here and in the outputs of products; other groups keep their bits."""
    from paper_1905_05233_amd import sequence_ops as S
    m = torch.randn((20, 300), generator=torch.Generator().manual_seed(1)).to(TORCH[dtype]).cuda()
    clean = S.W4Matrix.quantize(m, 64).dequantize(torch.float32)
    m[3, 70], m[17, 299] = bad, bad
    w = S.W4Matrix.quantize(m, 64)
    back = w.dequantize(torch.float32)
    hit = torch.zeros_like(back, dtype=torch.bool)
    hit[3, 64:128] = hit[17, 256:300] = True
    assert bool(torch.isnan(back[hit]).all()) and torch.equal(back[~hit], clean[~hit])
    y = S.matvec_w4(torch.ones((2, 300), device="cuda"), w)
    rows = torch.tensor([3, 17], device="cuda")
    assert bool(torch.isnan(y[:, rows]).all()) and int(torch.isnan(y).sum()) == 4
    zero = S.matvec_w4(torch.zeros((1, 300), device="cuda"), w)
    assert bool(torch.isnan(zero[0, rows]).all()) and not zero[0, :3].any()


def test_scales_below_the_normal_range():
    """There a scale has few bits: codes are clipped at 7 scales to either side."""
    from paper_1905_05233_amd import sequence_ops as S
    tiny = 2.0 ** -133                       # bf16's smallest value
    m = torch.zeros((2, 32))
    m[0, :4] = torch.tensor([9.8, -9.8, 2.0, -1.0]) * tiny     # a scale of 1.4 tiny becomes 1
    w = S.W4Matrix.quantize(m.cuda(), 32)
    back = w.dequantize(torch.float32).cpu().numpy() / tiny
    assert np.array_equal(back[0, :4], [7.0, -7.0, 2.0, -1.0]) and not back[0, 4:].any() and not back[1].any()


def test_the_tensors_memory_is_read_where_it_is():
    """A tensor of a matrix that is given other memory is read there, and checked again."""
    from paper_1905_05233_amd import sequence_ops as S
    m = torch.randn((40, 200), generator=torch.Generator().manual_seed(2)).cuda()
    w, other = S.W4Matrix.quantize(m, 64), S.W4Matrix.quantize(m * 2 - 1, 64)
    x = torch.randn((2, 200), generator=torch.Generator().manual_seed(3)).cuda()
    first, want = S.matvec_w4(x, w), S.matvec_w4(x, other)
    held = w.tiles.detach(), w.scales.detach()
    w.tiles.data, w.scales.data = other.tiles, other.scales
    assert torch.equal(S.matvec_w4(x, w), want) and not torch.equal(first, want)
    w.tiles.data = other.tiles[:2].clone()
    with pytest.raises(ValueError):
        S.matvec_w4(x, w)
    with pytest.raises(ValueError):
        w.dequantize()
    w.tiles.data, w.scales.data = held
    assert torch.equal(S.matvec_w4(x, w), first)
