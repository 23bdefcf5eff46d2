"""Products with 4-bit weights at the widest layers: whole numbers, whose sums are exact,
and the bound that follows from the order of the sums, for fp32 outputs from every type of x."""
import numpy as np
import pytest
import torch

import sequence_reference as R
import w4_reference as W
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def _np(t):
    return t.double().cpu().numpy()


def _matrix(codes, scales, K):
    from paper_1905_05233_amd import sequence_ops as S
    even = torch.cat((codes, torch.full((codes.shape[0], 1), 15)), 1) if K % 2 else codes
    return S.W4Matrix.from_nibbles((even[:, 0::2] | even[:, 1::2] << 4).to(torch.uint8).cuda(), scales.cuda(), K)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "fp8"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [4096, 25088, 25103])
def test_whole_numbers(K, group, dtype):
    """Small whole numbers, scales that are powers of two (of x in 8 bits too, a row's
    and by groups): the terms' sizes add to less than 2^24 of the smallest step, so every
    sum is exact in fp32, whatever its order."""
    from paper_1905_05233_amd import sequence_ops as S
    print(f"[w4 whole] {K} {group} {dtype}", flush=True)
    g = torch.Generator().manual_seed(K + group)
    rows, groups = 40, -(-K // group)
    codes = torch.randint(0, 16, (rows, K), generator=g)
    scales = (2.0 ** torch.randint(-2, 2, (rows, groups), generator=g)).bfloat16()
    w = _matrix(codes, scales, K)
    full = (codes.numpy() - 8.0) * np.repeat(_np(scales), group, 1)[:, :K]
    for M in (1, 16):
        x = torch.randint(-2, 3, (M, K), generator=g).float()
        for xg in ((1, groups) if dtype == "fp8" else (0,)):
            xs, xv, least = None, _np(x), 0.25
            if xg:
                xs = 2.0 ** torch.randint(-1, 2, (M, xg), generator=g).float()
                xv, least = xv * (_np(xs) if xg == 1 else np.repeat(_np(xs), group, 1)[:, :K]), 0.125
            assert (np.abs(xv) @ np.abs(full).T).max() / least < 2 ** 24
            t = x.to(E4M3 if dtype == "fp8" else TORCH[dtype]).cuda()
            y = S.matvec_w4(t, w, x_scales=None if xs is None else xs.cuda(), dtype=torch.float32)
            assert np.array_equal(_np(y), xv @ full.T), (K, group, dtype, M, xg)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "fp8"])
@pytest.mark.parametrize("shape", [(1, 25088, 64), (16, 25088, 48), (5, 4096, 1000), (3, 1000, 4500), (2, 1409, 4112)], ids=str)
def test_within_the_order_of_the_sums(shape, dtype):
    """fp32 outputs within the bound of sums of the weights themselves, whatever x's type:
    rows in bf16 and e4m3, which meet codes with an offset, must lose nothing to it (their
    products have few bits).  Beside the bound, the size of the error: with a rounding of 0.6 2^-24 of the
    partial sum for each column, and partial sums that grow as the root of their columns,
    a group's sum of 128 is off by 8 * 0.6 2^-24 = 2.8e-7 of its size, and the output by
    as much; 50 sums of groups in a wave add 1.7e-7 and 16 waves 1e-7, together 3.5e-7.
    Three parts of an fp32 value are three roundings a column."""
    from paper_1905_05233_amd import sequence_ops as S
    M, K, rows = shape
    for group in (32, 64, 128):
        print(f"[w4 bound] {shape} {dtype} {group}", flush=True)
        g = torch.Generator().manual_seed(K + group)
        codes = torch.randint(0, 16, (rows, K), generator=g)
        groups = -(-K // group)
        scales = ((torch.rand((rows, groups), generator=g) + 0.5) * 0.1).bfloat16()
        w = _matrix(codes, scales, K)
        x = torch.randn((M, K), generator=g)
        for xg in ((1, groups) if dtype == "fp8" else (0,)):
            xs = None
            if xg:
                t = (x * 40).to(E4M3)
                xs = torch.rand((M, xg), generator=g) + 0.1
                xv = _np(t.float()) * (_np(xs) if xg == 1 else np.repeat(_np(xs), group, 1)[:, :K])
            else:
                t = x.to(TORCH[dtype])
                xv = _np(t)
            want, bound = W.product(xv, codes.numpy() - 8.0, _np(scales), group, 3 if dtype == "f32" else 1, 0)
            y = S.matvec_w4(t.cuda(), w, x_scales=None if xs is None else xs.cuda(), dtype=torch.float32)
            R.assert_close(_np(y), want, bound, "f32", (shape, dtype, group, xg))
            rms = np.sqrt(np.mean(want ** 2))
            off = np.sqrt(np.mean((_np(y) - want) ** 2)) / rms
            print(f"    off by {off:.2e} of the outputs' size, the bound {bound.mean() / rms:.2e}", flush=True)
            assert off <= 4e-7 * np.sqrt(3 if dtype == "f32" else 1)
