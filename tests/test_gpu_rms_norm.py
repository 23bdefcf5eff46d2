"""The root-mean-square norm with the residual's addition, its 8-bit output and its
gradients on the GPU against the 64-bit reference, within derived bounds."""
import numpy as np
import pytest
import torch

import sequence_reference as R
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)

EPS = 1e-5
SHAPES = [(1, 1), (3, 5), (7, 8), (1, 64), (16, 512), (5, 75), (33, 100), (9, 1000), (3, 1024), (2, 4099), (2, 8192),
          (1, 30001), (700, 24), (3000, 16)]


def _np(t):
    return t.double().cpu().numpy()


def _inputs(shape, dtype, seed, count=3):
    g = torch.Generator().manual_seed(seed)
    parts = [torch.randn(shape, generator=g) * torch.exp(torch.randn((*shape[:-1], 1), generator=g)) for _ in range(count)]
    w = 1.0 + 0.1 * torch.randn(shape[-1], generator=g)
    return [p.to(TORCH[dtype]).cuda() for p in parts], w.to(TORCH[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm(shape, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    print(f"[norm] {shape} {dtype}", flush=True)
    (x, res), w = _inputs(shape, dtype, 3, 2)
    y, r = S.rms_norm(x, w, eps=EPS)
    assert r is None
    _, want, bound = R.norm(_np(x), None, _np(w), EPS)
    R.assert_close(_np(y), want, bound, dtype, "y")
    y, r = S.rms_norm(x, w, residual=res, eps=EPS)
    rr, want, bound = R.norm(_np(x), _np(res), _np(w), EPS)
    # the sum's own rounding to fp32 is relative to the sum
    R.assert_close(_np(y), want, bound, dtype, "y with residual")
    R.assert_close(_np(r), rr, np.abs(rr) * 2.0 ** -24, dtype, "r")
    # in place: r over x
    x2 = x.clone()
    y2, r2 = S.rms_norm(x2, w, residual=res, eps=EPS, r=x2)
    assert r2 is x2 and torch.equal(y2, y) and torch.equal(x2, r)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("shape", [(1, 1), (3, 40), (16, 512), (5, 75), (7, 129), (2, 1000), (3, 8192), (300, 96)], ids=str)
def test_norm_fp8(shape, group, dtype):
    """Scales are those of the largest values; a code stands for a value within half
    a step of e4m3 of the norm's output: 2^-4 of it, or 2^-10 scales for the
    smallest, and for what an fp32 evaluation may be off."""
    from paper_1905_05233_amd import sequence_ops as S
    (x, res), w = _inputs(shape, dtype, 4, 2)
    for residual in (None, res):
        q, scales, r = S.rms_norm_fp8(x, w, residual=residual, eps=EPS, group=group)
        assert q.dtype == torch.float8_e4m3fn and (r is None) == (residual is None)
        _, want, bound = R.norm(_np(x), None if residual is None else _np(residual), _np(w), EPS)
        C = shape[1]
        size = group or C
        pad = -C % size
        tops = np.abs(np.pad(want, ((0, 0), (0, pad)))).reshape(shape[0], -1, size).max(2)
        assert scales.shape == tops.shape
        rel = (C / 2 + 16) * 2.0 ** -24
        assert (np.abs(_np(scales) - np.maximum(tops, 2.0 ** -100) / 448) <= rel * tops / 448 + 1e-38).all()
        s = np.repeat(_np(scales), size, 1)[:, :C]
        got = _np(q.float()) * s
        assert (np.abs(got - want) <= np.maximum(np.abs(want) * 2.0 ** -4, s * 2.0 ** -10) + 2 * bound).all()
        assert (np.abs(_np(q.float())) <= 448).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(70000, 16), (17000, 104), (9000, 520), (2600, 4100), (3, 20000), (2, 33000)], ids=str)
def test_norm_many_and_long_rows(shape, dtype):
    """More rows than workgroups walk at a time, and rows of a whole workgroup or
    more: outputs in both types and gradients."""
    from paper_1905_05233_amd import sequence_ops as S
    print(f"[norm] {shape} {dtype}", flush=True)
    (x, dy), w = _inputs(shape, dtype, 5, 2)
    y, r = S.rms_norm(x, w, residual=dy, eps=EPS)
    rr, want, bound = R.norm(_np(x), _np(dy), _np(w), EPS)
    R.assert_close(_np(y), want, bound, dtype, "y")
    R.assert_close(_np(r), rr, np.abs(rr) * 2.0 ** -24, dtype, "r")
    C = shape[1]
    for group in (0, 128):
        q, scales, _ = S.rms_norm_fp8(x, w, residual=dy, eps=EPS, group=group)
        s = np.repeat(_np(scales), group or C, 1)[:, :C]
        got = _np(q.float()) * s
        assert (np.abs(got - want) <= np.maximum(np.abs(want) * 2.0 ** -4, s * 2.0 ** -10) + 2 * bound).all()
        tops = np.abs(np.pad(want, ((0, 0), (0, -C % (group or C))))).reshape(shape[0], -1, group or C).max(2)
        assert (np.abs(_np(scales) - tops / 448) <= (C / 2 + 16) * 2.0 ** -24 * tops / 448).all()
    dx, dw = S.rms_norm_backward(dy, x, w, eps=EPS)
    want, bx, wantw, bw = R.norm_gradients(_np(dy), _np(x), _np(w), None, EPS)
    R.assert_close(_np(dx), want, bx, dtype, "dx")
    R.assert_close(_np(dw), wantw, bw, "f32", "dweight")


def test_norm_special_rows():
    """Rows of zeros; rows with NaN or infinity poison themselves alone."""
    from paper_1905_05233_amd import sequence_ops as S
    x = torch.randn((6, 200), device="cuda")
    x[1] = 0.0
    x[3, 7], x[4, 150] = float("nan"), float("inf")
    w = torch.ones(200, device="cuda")
    y, _ = S.rms_norm(x, w, eps=EPS)
    q, s, _ = S.rms_norm_fp8(x, w, eps=EPS, group=64)
    clean, _ = S.rms_norm(x[[0, 2, 5]], w, eps=EPS)
    assert torch.equal(y[[0, 2, 5]], clean) and not y[1].any()
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[4, 150])) and not y[4, :150].any()
    assert not q[1].float().any() and torch.equal(s[1], torch.full((4,), 2.0 ** -100 / 448, device="cuda"))
    assert bool(torch.isnan(q[3].float()).all()) and bool(torch.isnan(s[3]).all())
    y, _ = S.rms_norm(x[1:2], w, eps=0.0)
    assert bool(torch.isnan(y).all())      # 0 / 0, as the formula says


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm_gradients(shape, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    print(f"[norm] gradients {shape} {dtype}", flush=True)
    (r, dy, dr), w = _inputs(shape, dtype, 6)
    for extra in (None, dr):
        dx, dw = S.rms_norm_backward(dy, r, w, dr=extra, eps=EPS)
        want, bx, wantw, bw = R.norm_gradients(_np(dy), _np(r), _np(w), None if extra is None else _np(extra), EPS)
        R.assert_close(_np(dx), want, bx, dtype, "dx")
        R.assert_close(_np(dw), wantw, bw, "f32", "dweight")
    d2 = dy.clone()
    got, dw2 = S.rms_norm_backward(d2, r, w, dr=dr, eps=EPS, dx=d2)
    assert got is d2 and torch.equal(d2, dx) and torch.equal(dw2, dw)
    d2 = dr.clone()
    S.rms_norm_backward(dy, r, w, dr=d2, eps=EPS, dx=d2)
    assert torch.equal(d2, dx)


def test_norm_gradient_against_differences():
    """The directional derivative; step 2^-7 leaves a remainder below 1e-3 of the scale."""
    from paper_1905_05233_amd import sequence_ops as S
    r, dy, w = torch.randn((40, 96), device="cuda"), torch.randn((40, 96), device="cuda"), torch.rand(96, device="cuda") + 0.5
    dx, dw = S.rms_norm_backward(dy, r, w, eps=EPS)

    def loss(r, w):
        return float((S.rms_norm(r, w, eps=EPS)[0].double() * dy.double()).sum())

    for k, grad in ((0, dx), (1, dw)):
        args, step = [r, w], 2.0 ** -7
        d = torch.randn_like(args[k])
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + step * d, args[k] - step * d
        num = (loss(*up) - loss(*down)) / (2 * step)
        scale = float(torch.linalg.vector_norm(grad.double()))
        assert abs(num - float((grad.double() * d.double()).sum())) <= 2e-3 * scale + 1e-3


def test_norm_layouts_and_empty():
    from paper_1905_05233_amd import sequence_ops as S
    (x, res, dy), w = _inputs((3, 50, 72), "bf16", 8)
    y, r = S.rms_norm(x, w, residual=res, eps=EPS)
    q, s, _ = S.rms_norm_fp8(x, w, residual=res, eps=EPS, group=32)
    dx, dw = S.rms_norm_backward(dy, r, w, dr=res, eps=EPS)

    def wide(t, off):
        b = torch.zeros((3, 52, 80), dtype=t.dtype, device="cuda")
        b[:, 1:51, off:off + 72] = t
        return b[:, 1:51, off:off + 72]

    out = torch.full((3, 51, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    y2, r2 = S.rms_norm(wide(x, 1), w, residual=wide(res, 3), eps=EPS, y=out[:, 1:])
    assert torch.equal(y2, y) and torch.equal(r2, r) and bool((out[:, 0] == 5.0).all())
    q2, s2, _ = S.rms_norm_fp8(x.transpose(0, 1).contiguous().transpose(0, 1), w, residual=wide(res, 0), eps=EPS, group=32)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, s) and s.shape == (3, 50, 3)
    dx2, dw2 = S.rms_norm_backward(wide(dy, 1), wide(r, 2), w, dr=wide(res, 5), eps=EPS)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw)
    e = torch.empty((0, 72), dtype=torch.bfloat16, device="cuda")
    assert S.rms_norm(e, w)[0].shape == (0, 72)
    dx, dw = S.rms_norm_backward(e, e, w)
    assert dx.shape == (0, 72) and not dw.any()
    # one row for all sequences as the residual
    one = res[:1, :1].expand(3, 50, 72)
    assert torch.equal(S.rms_norm(x, w, residual=one, eps=EPS)[0], S.rms_norm(x, w, residual=one.contiguous(), eps=EPS)[0])


def test_norm_gradients_repeat_and_graph():
    """dweight is summed in a fixed order; a captured call replays."""
    from paper_1905_05233_amd import sequence_ops as S
    (r, dy), w = _inputs((5000, 200), "bf16", 9, 2)
    want = S.rms_norm_backward(dy, r, w, eps=EPS)
    for _ in range(3):
        got = S.rms_norm_backward(dy, r, w, eps=EPS)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = S.rms_norm_backward(dy, r, w, eps=EPS)
        q, s, _ = S.rms_norm_fp8(r, w, eps=EPS)
    for k in range(4):
        r.copy_(torch.randn(r.shape, device="cuda"))
        want = S.rms_norm_backward(dy, r, w, eps=EPS)
        q0, s0, _ = S.rms_norm_fp8(r, w, eps=EPS)
        for t in (*got, s):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), k
        assert torch.equal(s, s0) and torch.equal(q.view(torch.uint8), q0.view(torch.uint8)), k


def test_norm_refusals():
    from paper_1905_05233_amd import sequence_ops as S
    from paper_1905_05233_amd._native import WinogradError
    x, w = torch.zeros((4, 16), device="cuda"), torch.ones(16, device="cuda")
    with pytest.raises(TypeError):
        S.rms_norm(x, w.half())
    with pytest.raises(ValueError):
        S.rms_norm(x, w[:8])
    with pytest.raises(ValueError):
        S.rms_norm(x, w, r=x)
    with pytest.raises(ValueError):
        S.rms_norm(x[0], w)
    with pytest.raises(WinogradError, match="group"):
        S.rms_norm_fp8(x, w, group=48)
    with pytest.raises(WinogradError, match="eps"):
        S.rms_norm(x, w, eps=-1.0)
    with pytest.raises(WinogradError, match="eps"):
        S.rms_norm_backward(x, x, w, eps=float("nan"))
    with pytest.raises(TypeError):
        S.rms_norm_backward(x.half(), x, w)
