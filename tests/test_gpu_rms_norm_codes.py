"""The 8-bit codes of the norm are those of the quotient y / s, also where it lies
halfway between two of them."""
import numpy as np
import pytest
import torch

from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


def _halves():
    """The numbers halfway between two neighbours among the e4m3 values, and these."""
    v = np.unique(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy())
    v = v[np.isfinite(v)].astype(np.float64)
    return np.concatenate((v, (v[1:] + v[:-1]) / 2))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [24, 512, 700, 4100, 40000])
def test_codes_are_those_of_the_quotient(C, dtype):
    """Rows of 1 and -1 without eps have a mean square of exactly 1, so the norm's
    output is the weight (or its negative), and scale and quotient follow in fp32."""
    g = np.random.default_rng(C)
    halves = _halves()
    for group in (0, 128):
        size = min(group or C, C)
        for trial in range(12):
            top = np.float32(np.exp(g.uniform(-8, 8)))
            w = (g.choice(halves, C) * (np.float64(top) / 448)).astype(np.float32)
            w[::size] = top
            w = torch.from_numpy(w).to(TORCH[dtype])
            x = torch.from_numpy(g.choice([-1.0, 1.0], (3, C))).to(TORCH[dtype])
            q, scales, _ = S_norm(x.cuda(), w.cuda(), group)
            y = torch.nn.functional.pad(x.float() * w.float(), (0, -C % size)).view(3, -1, size)
            s = y.abs().amax(2) / torch.tensor(448.0)
            assert torch.equal(scales.cpu(), s), (C, dtype, group)
            want = (y / s[:, :, None]).view(3, -1)[:, :C].to(torch.float8_e4m3fn)
            off = (q.cpu().view(torch.uint8) != want.view(torch.uint8)).sum().item()
            assert off == 0, (C, dtype, group, off)


def S_norm(x, w, group):
    from paper_1905_05233_amd import sequence_ops as S
    return S.rms_norm_fp8(x, w, eps=0.0, group=group)


def test_a_scale_of_infinity():
    """Where an output passes fp32's range its group's scale is infinite: the group's finite
    outputs are 0 times it, the infinite one NaN, and other groups are their own."""
    w = torch.full((128,), 2.0, device="cuda")
    x = torch.ones((1, 128), device="cuda")
    clean = S_norm(x, w, 64)
    w[3] = float("inf")
    q, scales, _ = S_norm(x, w, 64)
    assert torch.isinf(scales[0, 0]) and scales[0, 1] == clean[1][0, 1]
    q = q.float()
    assert bool(torch.isnan(q[0, 3])) and not q[0, :3].any() and not q[0, 4:64].any()
    assert torch.equal(q[0, 64:], clean[0].float()[0, 64:])
