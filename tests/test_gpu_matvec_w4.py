"""Products with 4-bit weights on the GPU against the 64-bit reference, and the
making and unmaking of such matrices."""
import numpy as np
import pytest
import torch

import sequence_reference as R
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)

E4M3 = torch.float8_e4m3fn
# rows of x, columns, rows of the matrix
SHAPES = [(1, 1, 1), (1, 8, 16), (3, 33, 17), (1, 127, 100), (2, 128, 64), (5, 129, 31), (16, 512, 48), (17, 300, 20),
          (1, 1536, 512), (4, 4096, 130), (8, 1000, 257), (1, 25088, 64), (40, 256, 16), (16, 4099, 1)]


def _np(t):
    return t.double().cpu().numpy()


def _matrix(rows, cols, group, seed):
    from paper_1905_05233_amd import sequence_ops as S
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 16, (rows, cols), generator=g)
    groups = -(-cols // group)
    scales = ((torch.rand((rows, groups), generator=g) + 0.5) * 0.1).bfloat16()
    even = torch.cat((codes, torch.full((rows, 1), 15)), 1) if cols % 2 else codes
    nibbles = (even[:, 0::2] | even[:, 1::2] << 4).to(torch.uint8)
    w = S.W4Matrix.from_nibbles(nibbles.cuda(), scales.cuda(), cols)
    ref = (codes.numpy() - 8.0) * np.repeat(_np(scales), group, 1)[:, :cols]
    return w, ref


def _x(M, K, dtype, seed, groups=1):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g)
    if dtype != "fp8":
        x = x.to(TORCH[dtype]).cuda()
        return x, None, _np(x)
    s = torch.rand((M, groups), generator=g) + 0.1
    q = (x * 40).to(E4M3)
    size = -(-K // groups) if groups == 1 else None
    return q.cuda(), s.cuda(), (_np(q.float()), _np(s), size)


def _bound(x, w, K):
    """Whatever the order: a product and a sum for each column, a scale for each
    group, and the codes' offset, which an evaluation may take out of the sums
    afterwards: partial sums of up to (8 + 24) / 1 times |x| a column instead of
    |code - 8| |x|."""
    return (np.abs(x) @ w.T) * (K + 64) * R.U["f32"]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "fp8"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_matvec(shape, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    M, K, rows = shape
    for group in (32, 64, 128):
        print(f"[w4] {shape} {dtype} {group}", flush=True)
        w, ref = _matrix(rows, K, group, seed=K + group)
        groups = -(-K // group)
        scale_max = np.repeat(_np(w.scales).transpose(0, 2, 1).reshape(-1, groups)[:rows], group, 1)[:, :K]
        for xg in ((1, groups) if dtype == "fp8" else (1,)):
            x, xs, xv = _x(M, K, dtype, seed=M, groups=xg)
            if dtype == "fp8":
                xv = xv[0] * (xv[1] if xg == 1 else np.repeat(xv[1], group, 1)[:, :K])
            out = ("f32", "bf16") if dtype in ("f32", "fp8") else (dtype, "f32")
            for od in out:
                y = S.matvec_w4(x, w, x_scales=xs, dtype=TORCH[od])
                R.assert_close(_np(y), xv @ ref.T, _bound(xv, 32 * scale_max, K), od, (shape, dtype, group, od))


# more tiles of 16 rows (with those of 16 rows of x) than the chip has units, odd and even
# in number, by few and many columns
MANY_TILES = [(1, 1000, 4111), (16, 1409, 4097), (3, 900, 4112), (33, 1030, 1400), (5, 512, 4500), (100, 1100, 601)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "fp8"])
@pytest.mark.parametrize("shape", MANY_TILES, ids=str)
def test_matvec_of_many_tiles(shape, dtype):
    """Against the reference, and bit for bit what the same rows of the matrix give
    in a smaller one for one row of x."""
    from paper_1905_05233_amd import sequence_ops as S
    M, K, rows = shape
    for group in (32, 64, 128):
        print(f"[w4 many] {shape} {dtype} {group}", flush=True)
        w, ref = _matrix(rows, K, group, seed=K + group)
        groups = -(-K // group)
        scale_max = np.repeat(_np(w.scales).transpose(0, 2, 1).reshape(-1, groups)[:rows], group, 1)[:, :K]
        for xg in ((1, groups) if dtype == "fp8" else (1,)):
            x, xs, xv = _x(M, K, dtype, seed=M, groups=xg)
            if dtype == "fp8":
                xv = xv[0] * (xv[1] if xg == 1 else np.repeat(xv[1], group, 1)[:, :K])
            y = S.matvec_w4(x, w, x_scales=xs, dtype=torch.float32)
            R.assert_close(_np(y), xv @ ref.T, _bound(xv, 32 * scale_max, K), "f32", (shape, dtype, group, xg))
            first = max(0, rows // 16 - 2) * 16
            part = S.W4Matrix._empty(rows - first, K, group, "cuda")
            part.tiles.copy_(w.tiles[first // 16:])
            part.scales.copy_(w.scales[first // 16:])
            for m in {0, M - 1}:
                one = S.matvec_w4(x[m:m + 1], part, x_scales=None if xs is None else xs[m:m + 1], dtype=torch.float32)
                assert torch.equal(one[0], y[m, first:]), (shape, dtype, group, m)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_matvec_exact_on_small_integers(dtype):
    """Codes, scales that are powers of two and small whole numbers: every sum is
    exact in fp32, whatever its order."""
    from paper_1905_05233_amd import sequence_ops as S
    g = torch.Generator().manual_seed(2)
    for M, K, rows, group in ((1, 777, 50, 64), (16, 256, 33, 128), (7, 4096, 16, 32)):
        codes = torch.randint(0, 16, (rows, K + K % 2), generator=g)
        scales = (2.0 ** torch.randint(-3, 4, (rows, -(-K // group)), generator=g)).bfloat16()
        w = S.W4Matrix.from_nibbles((codes[:, 0::2] | codes[:, 1::2] << 4).to(torch.uint8).cuda(), scales.cuda(), K)
        x = torch.randint(-2, 3, (M, K), generator=g).to(TORCH[dtype]).cuda()
        full = (codes[:, :K].numpy() - 8.0) * np.repeat(_np(scales), group, 1)[:, :K]
        y = S.matvec_w4(x, w, dtype=torch.float32)
        assert np.array_equal(_np(y), _np(x) @ full.T), (M, K, rows, group)
        assert np.array_equal(_np(w.dequantize(torch.float32)), full)


def test_matvec_layouts_and_values():
    from paper_1905_05233_amd import sequence_ops as S
    w, ref = _matrix(40, 200, 64, 5)
    x, _, _ = _x(6, 200, "bf16", 3)
    want = S.matvec_w4(x, w)
    buf = torch.full((6, 211), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, 3:203] = x
    out = torch.full((6, 50), 7.0, dtype=torch.bfloat16, device="cuda")
    S.matvec_w4(buf[:, 3:203], w, y=out[:, 5:45])
    assert torch.equal(out[:, 5:45], want) and bool((out[:, :5] == 7.0).all()) and bool((out[:, 45:] == 7.0).all())
    # one row for all: stride 0
    assert torch.equal(S.matvec_w4(x[:1].expand(6, 200), w), want[:1].expand(6, 40))
    # a row with NaN or infinity poisons itself alone; NaN behind a row's end is not read
    x2 = x.clone()
    x2[2, 17], x2[4, 199] = float("nan"), float("inf")
    y = S.matvec_w4(x2, w)
    assert torch.equal(y[[0, 1, 3, 5]], want[[0, 1, 3, 5]]) and bool(torch.isnan(y[2]).all())
    assert not bool(torch.isfinite(y[4][torch.from_numpy(ref[:, 199] != 0).cuda()]).any())
    assert S.matvec_w4(x[:0], w).shape == (0, 40)
    # the same row alone and among others
    for m in range(6):
        assert torch.equal(S.matvec_w4(x[m:m + 1], w), want[m:m + 1])


def test_matvec_wide_range():
    """fp32 rows whose values differ by many orders keep their small parts."""
    from paper_1905_05233_amd import sequence_ops as S
    w, ref = _matrix(64, 512, 128, 6)
    x = torch.randn((3, 512), generator=torch.Generator().manual_seed(3)) * 10.0 ** torch.linspace(-12, 12, 512)
    x = x[:, torch.randperm(512, generator=torch.Generator().manual_seed(4))].contiguous()
    x[1] *= 1e-20
    x[2] *= 1e20
    scale = np.repeat(_np(w.scales).transpose(0, 2, 1).reshape(-1, 4)[:64], 128, 1)
    y = S.matvec_w4(x.cuda(), w)
    R.assert_close(_np(y), _np(x) @ ref.T, _bound(_np(x), 32 * scale, 512), "f32", "wide")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (17, 33), (16, 128), (50, 300)], ids=str)
def test_quantize(shape, dtype):
    """Scales are bf16(max / 7); every weight is within half a scale, or beyond 7
    scales by what the scale's rounding took."""
    from paper_1905_05233_amd import sequence_ops as S
    m = torch.randn(shape, generator=torch.Generator().manual_seed(1)).to(TORCH[dtype]).cuda()
    m[0, :1] = 0.0
    for group in (32, 64, 128):
        w = S.W4Matrix.quantize(m, group)
        back = _np(w.dequantize(torch.float32))
        C = shape[1]
        tops = np.abs(np.pad(_np(m), ((0, 0), (0, -C % group)))).reshape(shape[0], -1, group).max(2)
        groups = tops.shape[1]
        scales = _np(w.scales).transpose(0, 2, 1).reshape(-1, groups)
        assert (np.abs(scales[:shape[0]] - tops / 7) <= tops / 7 * 2.0 ** -8).all() and not scales[shape[0]:].any()
        s = np.repeat(scales[:shape[0]], group, 1)[:, :C]
        assert (np.abs(back - _np(m)) <= s * (0.5 + 7 * 2.0 ** -8)).all()
        again = S.W4Matrix.quantize(torch.from_numpy(back).float().cuda(), group)
        assert np.abs(_np(again.dequantize(torch.float32)) - back).max() <= 0.02 * np.abs(back).max()


def test_graph_and_stream():
    from paper_1905_05233_amd import sequence_ops as S
    w, _ = _matrix(300, 1000, 64, 8)
    x = torch.randn((4, 1000), device="cuda").bfloat16()
    want = S.matvec_w4(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = S.matvec_w4(x, w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = S.matvec_w4(x, w)
    for k in range(4):
        x.copy_(torch.randn((4, 1000), device="cuda"))
        want = S.matvec_w4(x, w)
        got.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), k


def test_refusals():
    from paper_1905_05233_amd import sequence_ops as S
    w, _ = _matrix(40, 200, 64, 5)
    x = torch.zeros((2, 200), device="cuda")
    with pytest.raises(ValueError):
        S.matvec_w4(x[:, :199], w)
    with pytest.raises(TypeError):
        S.matvec_w4(x.double(), w)
    with pytest.raises(ValueError):
        S.matvec_w4(x.to(E4M3), w)
    with pytest.raises(ValueError):
        S.matvec_w4(x, w, x_scales=torch.ones((2, 1), device="cuda"))
    with pytest.raises(S.N.WinogradError, match="x_scales"):
        S.matvec_w4(x.to(E4M3), w, x_scales=torch.ones((2, 3), device="cuda"))
    with pytest.raises(ValueError):
        S.matvec_w4(x, w, y=torch.zeros((2, 41), device="cuda"))
    with pytest.raises(ValueError):
        S.W4Matrix(w.tiles, w.scales, 40, 200, 48)
    with pytest.raises(ValueError):
        S.W4Matrix(w.tiles, w.scales, 50, 200, 64)
    with pytest.raises(ValueError):
        S.W4Matrix.from_nibbles(torch.zeros((4, 100), dtype=torch.uint8, device="cuda"),
                                torch.zeros((4, 5), dtype=torch.bfloat16, device="cuda"), 200)
    with pytest.raises(ValueError):
        S.W4Matrix.quantize(x, 16)
