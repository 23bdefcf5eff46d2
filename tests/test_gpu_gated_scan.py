"""The gated linear recurrence, its gradients and its single step on the GPU
against the 64-bit reference, within the bounds that sequence_reference derives;
layouts, padding, special values, streams, graphs and refusals."""
import numpy as np
import pytest
import torch

import sequence_reference as R
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)

# sequences, steps, channels: one of everything, odd channels, steps around the
# kernels' blocks and tiles, few long rows, many short ones
SHAPES = [(1, 1, 1), (2, 3, 5), (1, 8, 8), (1, 31, 64), (2, 33, 75), (1, 64, 512), (3, 255, 24), (2, 257, 9),
          (1, 1025, 17), (5, 100, 200), (1, 4099, 40), (70, 40, 130), (300, 2, 33), (2, 513, 1024), (1, 20001, 3)]


def _np(t):
    return t.double().cpu().numpy()


def _inputs(shape, dtype, seed, out_gate=True, layout="dense"):
    N, L, C = shape
    g = torch.Generator().manual_seed(seed)
    parts = [torch.randn(shape, generator=g) * 1.5 + 2.0, torch.randn(shape, generator=g), torch.randn(shape, generator=g)]
    parts = [p.to(TORCH[dtype]).cuda() for p in parts[:3 if out_gate else 2]]
    if layout == "fused":      # slices of the rows of one projection, at odd offsets
        buf = torch.zeros((N, L, 3 * C + 1), dtype=TORCH[dtype], device="cuda")
        for k, p in enumerate(parts):
            buf[:, :, 1 + k * C:1 + (k + 1) * C] = p
        parts = [buf[:, :, 1 + k * C:1 + (k + 1) * C] for k in range(len(parts))]
    elif layout == "steps":    # steps outermost
        parts = [p.transpose(0, 1).contiguous().transpose(0, 1) for p in parts]
    return parts + [None] * (3 - len(parts))


def _call(shape, dtype, seed, out_gate=True, h0=False, lengths=None, layout="dense", grads=True):
    from paper_1905_05233_amd import sequence_ops as S
    N, L, C = shape
    z, v, o = _inputs(shape, dtype, seed, out_gate, layout)
    g = torch.Generator().manual_seed(seed + 1)
    h = torch.randn((N, C), generator=g).cuda() if h0 else None
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = dict(zip(("y", "h_last", "states"), S.gated_scan(z, v, o, h0=h, lengths=n, save_states=grads)))
    dy = dh = None
    if grads:
        dy = torch.randn(shape, generator=g).to(TORCH[dtype]).cuda()
        dh = torch.randn((N, C), generator=g).cuda() if h0 else None
        names = ("dgate", "dvalue", "dout_gate", "dh0")
        got |= dict(zip(names, S.gated_scan_backward(dy, z, v, got["states"], out_gate=o, dh_last=dh, lengths=n)))
    torch.cuda.synchronize()
    ref = R.scan(_np(z), _np(v), None if o is None else _np(o), None if h is None else _np(h),
                 None if n is None else np.array(lengths), None if dy is None else _np(dy),
                 None if dh is None else _np(dh))
    for name, (want, bound) in ref.items():
        R.assert_close(_np(got[name]), want, bound, "f32" if name in ("h_last", "dh0") else dtype, name)
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scan_and_gradients(shape, dtype):
    print(f"[scan] {shape} {dtype}", flush=True)
    _call(shape, dtype, seed=shape[1], out_gate=True, h0=shape[2] % 2 == 0)
    _call(shape, dtype, seed=shape[1] + 7, out_gate=False, h0=shape[2] % 2 == 1)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("shape", [(100, 600, 72), (200, 300, 64), (130, 270, 61), (2000, 20, 40), (3, 5000, 128)], ids=str)
def test_many_channels_over_several_tiles(shape, dtype):
    """Channels that fill the chip, in groups of 64 and of 128 bytes, over several
    tiles of steps; many short sequences; chunks of a tile."""
    print(f"[scan] {shape} {dtype}", flush=True)
    _call(shape, dtype, 17, out_gate=shape[0] != 200, h0=True, lengths=[(37 * k) % (shape[1] + 9) for k in range(shape[0])])


@pytest.mark.parametrize("layout", ["fused", "steps"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 70, 24), (2, 300, 37), (1, 9, 3), (2, 40, 130)], ids=str)
def test_layouts(shape, dtype, layout):
    print(f"[scan] {shape} {dtype} {layout}", flush=True)
    dense = _call(shape, dtype, 5, h0=True)
    got = _call(shape, dtype, 5, h0=True, layout=layout)
    for name in ("y", "h_last", "dgate", "dvalue", "dout_gate", "dh0"):
        assert torch.equal(dense[name], got[name]), name


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("C", [8, 75])
def test_lengths(C, dtype):
    # empty rows, full ones, ends inside and at the edges of blocks, and values out of range
    L = 600
    lengths = [0, 1, 31, 32, 33, 255, 256, 257, 599, 600, 512, 0]
    got = _call((len(lengths), L, C), dtype, 9, h0=True, lengths=lengths)
    h0 = torch.randn((len(lengths), C), generator=torch.Generator().manual_seed(10)).cuda()
    assert torch.equal(got["h_last"][0], h0[0]) and torch.equal(got["h_last"][-1], h0[-1])
    assert not got["y"][0].any() and not got["dgate"][0].any()
    a = _call((3, 40, C), dtype, 4, lengths=[-5, 41, 1 << 30])
    b = _call((3, 40, C), dtype, 4, lengths=[0, 40, 40])
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_padding_is_not_used(bad):
    from paper_1905_05233_amd import sequence_ops as S
    shape, lengths = (4, 300, 40), torch.tensor([0, 130, 299, 300], dtype=torch.int32, device="cuda")
    z, v, o = _inputs(shape, "bf16", 3)
    dy = torch.randn(shape, device="cuda").bfloat16()
    live = (torch.arange(300, device="cuda")[None] < lengths[:, None])[:, :, None]

    def run(*t):
        y, h, s = S.gated_scan(*t[:3], lengths=lengths, save_states=True)
        return (y, h, *S.gated_scan_backward(t[3], t[0], t[1], s, out_gate=t[2], lengths=lengths))

    want = run(z, v, o, dy)
    got = run(*[torch.where(live, t, bad) for t in (z, v, o, dy)])
    for a, b in zip(want, got):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


def test_saturated_gates():
    """Gates far out: f is 0 (the state is replaced) or 1 (it is kept) exactly."""
    from paper_1905_05233_amd import sequence_ops as S
    for big in (float("inf"), 200.0):
        z = torch.full((1, 40, 8), big, device="cuda")
        z[0, 20] = -big
        v = torch.randn((1, 40, 8), device="cuda")
        h0 = torch.randn((1, 8), device="cuda")
        y, h, s = S.gated_scan(z, v, h0=h0, save_states=True)
        assert torch.equal(y[0, :20], h0.expand(20, 8)) and torch.equal(y[0, 20:], v[0, 20].expand(20, 8))
        dz, dv, _, dh0 = S.gated_scan_backward(torch.ones_like(y), z, v, s)
        assert not dz.any() and torch.equal(dv[0, 20], torch.full((8,), 20.0, device="cuda"))
        assert torch.equal(dh0[0], torch.full((8,), 20.0, device="cuda")) and not dv[0, :20].any()


def test_no_steps_and_one_long_row():
    from paper_1905_05233_amd import sequence_ops as S
    e = torch.empty((3, 0, 16), dtype=torch.bfloat16, device="cuda")
    h0 = torch.randn((3, 16), device="cuda")
    y, h, s = S.gated_scan(e, e, h0=h0, save_states=True)
    assert y.shape == e.shape and torch.equal(h, h0) and s.shape == (3, 0, 16)
    dz, dv, do, dh0 = S.gated_scan_backward(e, e, e, s, out_gate=e, dh_last=h0)
    assert do.shape == e.shape and torch.equal(dh0, h0)
    assert torch.equal(S.gated_scan(e, e)[1], torch.zeros_like(h0))
    _call((1, 70001, 2), "f32", 2, h0=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(dtype):
    """The directional derivative of a weighted sum of the fp32 outputs.  With step
    2^-6 the second-order remainder of the central difference is below 1e-3 of the
    scale; the sums' rounding adds 1e-5 / 2^-6."""
    from paper_1905_05233_amd import sequence_ops as S
    shape = (2, 300, 20)
    z, v, o = [t.float() for t in _inputs(shape, dtype, 21)]
    h0, dh = torch.randn((2, 20), device="cuda"), torch.randn((2, 20), device="cuda")
    dy = torch.randn(shape, device="cuda")
    y, h, s = S.gated_scan(z, v, o, h0=h0, save_states=True)
    grads = S.gated_scan_backward(dy, z, v, s, out_gate=o, dh_last=dh)

    def loss(z, v, o, h0):
        y, h = S.gated_scan(z, v, o, h0=h0)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    args, step = [z, v, o, h0], 2.0 ** -6
    for k in range(4):
        d = torch.randn_like(args[k])
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + step * d, args[k] - step * d
        num = (loss(*up) - loss(*down)) / (2 * step)
        scale = float(torch.linalg.vector_norm(grads[k].double()))
        assert abs(num - float((grads[k].double() * d.double()).sum())) <= 2e-3 * scale + 1e-3


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 75), (16, 512), (257, 40)], ids=str)
def test_step_is_a_scan_of_one(shape, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    N, C = shape
    z, v, o = [t[:, 0] for t in _inputs((N, 1, C), dtype, 8, layout="fused")]
    h = torch.randn((N, C), generator=torch.Generator().manual_seed(1)).cuda()
    for og in (o, None):
        y, hn = S.gated_step(z, v, h, out_gate=og)
        ref = R.scan(_np(z)[:, None], _np(v)[:, None], None if og is None else _np(og)[:, None], _np(h), None)
        R.assert_close(_np(y)[:, None], *ref["y"], dtype, "y")
        R.assert_close(_np(hn), *ref["h_last"], "f32", "h")
        h2, y2 = h.clone(), torch.empty_like(y)
        assert S.gated_step(z, v, h2, out_gate=og, h_new=h2, y=y2)[1] is h2
        assert torch.equal(h2, hn) and torch.equal(y2, y)


def test_given_outputs_and_rows_that_leave_gaps():
    from paper_1905_05233_amd import sequence_ops as S
    shape = (2, 65, 20)
    z, v, o = _inputs(shape, "bf16", 12)
    y, h, s = S.gated_scan(z, v, o, save_states=True)
    buf = torch.full((2, 66, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    S.gated_scan(z, v, o, y=buf[:, 1:, 3:23])
    assert torch.equal(buf[:, 1:, 3:23], y)
    buf[:, 1:, 3:23] = 7.0
    assert bool((buf == 7.0).all())
    dy = torch.randn(shape, device="cuda").bfloat16()
    want = S.gated_scan_backward(dy, z, v, s, out_gate=o)
    buf = torch.full((2, 65, 61), 7.0, dtype=torch.bfloat16, device="cuda")
    got = S.gated_scan_backward(dy, z, v, s, out_gate=o, out=[buf[:, :, k * 20:(k + 1) * 20] for k in range(3)])
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert bool((buf[:, :, 60] == 7.0).all())


def test_other_stream_and_graph():
    from paper_1905_05233_amd import sequence_ops as S
    shape = (2, 900, 40)
    z, v, o = _inputs(shape, "bf16", 30)
    dy = torch.randn(shape, device="cuda").bfloat16()

    def run(stream=None):
        y, h, s = S.gated_scan(z, v, o, save_states=True, stream=stream)
        return (y, h, *S.gated_scan_backward(dy, z, v, s, out_gate=o, stream=stream))

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for k in range(4):
        z.copy_(torch.randn(shape, device="cuda") + 1.0)
        want = run()
        for t in got:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b), k


def test_refusals():
    from paper_1905_05233_amd import sequence_ops as S
    from paper_1905_05233_amd._native import WinogradError
    z = torch.zeros((2, 5, 8), device="cuda")
    h = torch.zeros((2, 8), device="cuda")
    with pytest.raises(TypeError):
        S.gated_scan(z, z.half())
    with pytest.raises(TypeError):
        S.gated_scan(z.double(), z.double())
    with pytest.raises(ValueError):
        S.gated_scan(z, z[:, :4])
    with pytest.raises(ValueError):
        S.gated_scan(z.cpu(), z)
    with pytest.raises(ValueError):
        S.gated_scan(z, z.transpose(1, 2).contiguous().transpose(1, 2))      # channels apart
    with pytest.raises(ValueError):
        S.gated_scan(z, z, h0=torch.zeros((8, 2), device="cuda").t())
    with pytest.raises(TypeError):
        S.gated_scan(z, z, lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(WinogradError, match="overlap"):
        S.gated_scan(z, z, y=torch.zeros((1, 5, 8), device="cuda").expand(2, 5, 8))
    y, _, s = S.gated_scan(z, z, save_states=True)
    with pytest.raises(ValueError):
        S.gated_scan_backward(z, z, z, s[:, :0])
    with pytest.raises(ValueError):
        S.gated_scan_backward(z, z, z, s, out=[z.clone()])
    with pytest.raises(ValueError):
        S.gated_step(h, h, h, h_new=torch.zeros((2, 9), device="cuda"))
    with pytest.raises(TypeError):
        S.gated_step(h, h, h.half())
