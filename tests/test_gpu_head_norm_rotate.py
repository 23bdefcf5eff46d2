"""The norm of heads with the rotation by position, and its gradients, on the GPU against
the 64-bit reference, within the bounds that attention_reference derives; pairs, layouts,
far positions, streams, graphs and refusals."""
import numpy as np
import pytest
import torch

import attention_reference as A
import sequence_reference as R
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)


# sequences, steps, heads of q and k, channels, turned channels: one of everything, halves
# that end inside 16 bytes, channels that are not turned, the widest heads, many rows
SHAPES = [(1, 1, 1, 1, 2, 2), (2, 3, 2, 1, 3, 2), (1, 5, 1, 1, 16, 16), (2, 7, 3, 1, 64, 64), (1, 9, 2, 2, 75, 74),
          (2, 4, 5, 1, 100, 50), (1, 3, 4, 4, 128, 128), (3, 2, 1, 2, 96, 32), (1, 2, 2, 2, 256, 256), (1, 4, 2, 1, 256, 2),
          (1, 3, 1, 1, 255, 6), (2, 300, 4, 2, 64, 48), (1, 2000, 2, 1, 40, 40), (1, 1, 64, 8, 128, 64), (5, 50, 1, 1, 17, 10),
          (7, 600, 8, 8, 64, 64)]


def _np(t):
    return t.double().cpu().numpy()


def _inputs(shape, dtype, seed, layout="dense"):
    N, L, Hq, Hk, D, _ = shape
    g = torch.Generator().manual_seed(seed)
    size = torch.exp(torch.randn((N, L, 1, 1), generator=g))
    q, k = [(torch.randn((N, L, h, D), generator=g) * size).to(TORCH[dtype]).cuda() for h in (Hq, Hk)]
    dq, dk = [torch.randn((N, L, h, D), generator=g).to(TORCH[dtype]).cuda() for h in (Hq, Hk)]
    w = [(1.0 + 0.3 * torch.randn(D, generator=g)).to(TORCH[dtype]).cuda() for _ in range(2)]
    if layout == "fused":
        rows = torch.cat((torch.zeros_like(q[:, :, 0, :1]), q.flatten(2), k.flatten(2)), 2)
        q, k = [t.unflatten(2, (h, D)) for t, h in zip(rows[:, :, 1:].split([Hq * D, Hk * D], 2), (Hq, Hk))]
    elif layout == "heads":
        q, k, dq, dk = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, dq, dk)]
    return q, k, dq, dk, w


def _frequencies(R_, base=10000.0):
    return [base ** (-2.0 * i / R_) for i in range(R_ // 2)]


def _call(shape, dtype, seed, adjacent, positions=None, start=0, layout="dense", eps=1e-6):
    from paper_1905_05233_amd import sequence_ops as S
    N, L, Hq, Hk, D, R_ = shape
    q, k, dq, dk, (wq, wk) = _inputs(shape, dtype, seed, layout)
    rot = S.Rotary(R_, adjacent=adjacent)
    p = None if positions is None else torch.tensor(positions, dtype=torch.int32, device="cuda").view(N, L)
    yq, yk = S.head_norm_rotate(q, k, wq, wk, rot, positions=p, start=start, eps=eps)
    gq, gk, gwq, gwk = S.head_norm_rotate_backward(dq, dk, q, k, wq, wk, rot, positions=p, start=start, eps=eps)
    torch.cuda.synchronize()
    where = np.array(positions).reshape(N, L) if positions is not None else np.tile(start + np.arange(L), (N, 1))
    for x, w, dy, y, gx, gw in ((q, wq, dq, yq, gq, gwq), (k, wk, dk, yk, gk, gwk)):
        want, bound = A.rotate(_np(x), _np(w), _frequencies(R_), where, eps, adjacent)
        R.assert_close(_np(y), want, bound, dtype, "y")
        (dx, bx), (dw, bw) = A.rotate(_np(x), _np(w), _frequencies(R_), where, eps, adjacent, _np(dy))
        R.assert_close(_np(gx), dx, bx, dtype, "dx")
        R.assert_close(_np(gw), dw, bw, "f32", "dw")
    return yq, yk, gq, gk, gwq, gwk


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm_rotation_and_gradients(shape, dtype):
    print(f"[rotate] {shape} {dtype}", flush=True)
    _call(shape, dtype, 3, adjacent=False)
    _call(shape, dtype, 4, adjacent=True, start=11)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_far_positions(adjacent, dtype):
    far = [0, 1, -1, 2 ** 20, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 12345678]
    _call((2, 4, 2, 1, 64, 64), dtype, 5, adjacent, positions=far)
    _call((1, 8, 2, 1, 64, 20), dtype, 5, adjacent, start=2 ** 31 - 4)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("layout", ["fused", "heads"])
@pytest.mark.parametrize("shape", [(2, 7, 3, 1, 64, 64), (1, 9, 2, 2, 75, 74), (3, 5, 2, 1, 36, 18)], ids=str)
def test_layouts(shape, layout, dtype):
    for adjacent in (False, True):
        dense = _call(shape, dtype, 6, adjacent)
        for a, b in zip(dense, _call(shape, dtype, 6, adjacent, layout=layout)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("adjacent", [False, True])
def test_tokens_and_outputs_in_place(adjacent):
    from paper_1905_05233_amd import sequence_ops as S
    shape = (5, 1, 3, 1, 50, 34)
    q, k, dq, dk, (wq, wk) = _inputs(shape, "bf16", 7)
    rot = S.Rotary(34, adjacent=adjacent)
    p = torch.tensor([[3], [900], [0], [7], [5]], dtype=torch.int32, device="cuda")
    want = S.head_norm_rotate(q, k, wq, wk, rot, positions=p)
    token = S.head_norm_rotate(q[:, 0], k[:, 0], wq, wk, rot, positions=p[:, 0])
    grads = S.head_norm_rotate_backward(dq, dk, q, k, wq, wk, rot, positions=p)
    at_tokens = S.head_norm_rotate_backward(dq[:, 0], dk[:, 0], q[:, 0], k[:, 0], wq, wk, rot, positions=p[:, 0])
    for a, b in zip(want + grads[:2], token + at_tokens[:2]):
        assert torch.equal(a[:, 0], b)
    S.head_norm_rotate_backward(dq, dk, q, k, wq, wk, rot, positions=p, out=(dq, dk))
    assert torch.equal(dq, grads[0]) and torch.equal(dk, grads[1])
    assert S.head_norm_rotate(q, k, wq, wk, rot, positions=p, q_out=q, k_out=k)[0] is q
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_frequencies_and_no_rows():
    from paper_1905_05233_amd import sequence_ops as S
    q, k, dq, dk, (wq, wk) = _inputs((2, 6, 2, 1, 8, 8), "f32", 8)
    f = [1.5, -0.25, 0.0, 7.0]
    y, _ = S.head_norm_rotate(q, k, wq, wk, S.Rotary(8, frequencies=f), start=3)
    want, bound = A.rotate(_np(q), _np(wq), f, np.tile(3 + np.arange(6), (2, 1)), 1e-6, False)
    R.assert_close(_np(y), want, bound, "f32", "y")
    e = torch.empty((2, 0, 2, 8), device="cuda")
    rot = S.Rotary(8)
    assert S.head_norm_rotate(e, e, wq, wk, rot)[0].shape == e.shape
    assert not any(t.any() for t in S.head_norm_rotate_backward(e, e, e, e, wq, wk, rot)[2:])
    z = torch.zeros_like(q)
    assert not S.head_norm_rotate(z, z, wq, wk, rot)[0].any()


def test_values_that_are_not_finite_stay_in_their_head():
    from paper_1905_05233_amd import sequence_ops as S
    q, k, dq, dk, (wq, wk) = _inputs((2, 6, 3, 1, 40, 30), "bf16", 9)
    rot = S.Rotary(30)
    want = S.head_norm_rotate(q, k, wq, wk, rot)
    bad = q.clone()
    bad[1, 2, 1, 5] = float("nan")
    bad[0, 4, 2, 39] = float("inf")
    got = S.head_norm_rotate(bad, k, wq, wk, rot)
    keep = torch.ones((2, 6, 3), dtype=torch.bool, device="cuda")
    keep[1, 2, 1] = keep[0, 4, 2] = False
    assert torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1], want[1])
    assert bool(torch.isnan(got[0][1, 2, 1]).all()) and bool(torch.isnan(got[0][0, 4, 2]).any())


def test_gradients_against_differences():
    """Central differences in fp32 with step 2^-7: off by the third derivative times
    step^2 and by the outputs' 1e-6 over the step."""
    from paper_1905_05233_amd import sequence_ops as S
    q, k, dq, dk, (wq, wk) = _inputs((2, 40, 3, 1, 24, 16), "f32", 10)
    q, k = q / q.norm(dim=-1, keepdim=True) * 5, k / k.norm(dim=-1, keepdim=True) * 5
    rot = S.Rotary(16)
    grads = S.head_norm_rotate_backward(dq, dk, q, k, wq, wk, rot, start=100)

    def loss(q, k, wq, wk):
        a, b = S.head_norm_rotate(q, k, wq, wk, rot, start=100)
        return float((a.double() * dq.double()).sum() + (b.double() * dk.double()).sum())

    args, step = [q, k, wq, wk], 2.0 ** -7
    for i in range(4):
        d = torch.randn_like(args[i])
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * d, args[i] - step * d
        num = (loss(*up) - loss(*down)) / (2 * step)
        size = float(torch.linalg.vector_norm(grads[i].double())) + 1.0
        assert abs(num - float((grads[i].double() * d.double()).sum())) <= 2e-3 * size, i


def test_other_stream_and_graph():
    from paper_1905_05233_amd import sequence_ops as S
    q, k, dq, dk, (wq, wk) = _inputs((2, 90, 3, 1, 64, 64), "bf16", 11)
    rot, p = S.Rotary(64), torch.arange(180, dtype=torch.int32, device="cuda").view(2, 90)

    def run(stream=None):
        return (*S.head_norm_rotate(q, k, wq, wk, rot, positions=p, stream=stream),
                *S.head_norm_rotate_backward(dq, dk, q, k, wq, wk, rot, positions=p, stream=stream))

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
    for i in range(4):
        q.copy_(torch.randn(q.shape, device="cuda"))
        p.add_(1000)
        want = run()
        for t in got:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b), i


def test_refusals():
    from paper_1905_05233_amd import sequence_ops as S
    from paper_1905_05233_amd._native import WinogradError
    q, w, rot = torch.zeros((2, 5, 2, 8), device="cuda"), torch.ones(8, device="cuda"), S.Rotary(8)
    for bad in (0, 7, -2):
        with pytest.raises(ValueError):
            S.Rotary(bad)
    with pytest.raises(ValueError):
        S.Rotary(8, frequencies=[1.0])
    with pytest.raises(ValueError):
        S.Rotary(4, frequencies=[1.0, float("inf")])
    with pytest.raises(ValueError):
        S.Rotary(4, base=0.0)
    with pytest.raises(TypeError):
        S.head_norm_rotate(q, q.half(), w, w, rot)
    with pytest.raises(TypeError):
        S.head_norm_rotate(q, q, w, w, rot.turns)
    with pytest.raises(TypeError):
        S.head_norm_rotate(q, q, w.half(), w, rot)
    with pytest.raises(ValueError):
        S.head_norm_rotate(q, q[:, :4], w, w, rot)
    with pytest.raises(ValueError):
        S.head_norm_rotate(q, q, w[:4], w, rot)
    with pytest.raises(TypeError):
        S.head_norm_rotate(q, q, w, w, rot, positions=torch.zeros((2, 5), dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        S.head_norm_rotate(q, q, w, w, rot, positions=torch.zeros((2, 4), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        S.head_norm_rotate(q, q, w, w, S.Rotary(8, device="cpu"))
    with pytest.raises(WinogradError, match="R must"):
        S.head_norm_rotate(q, q, w, w, S.Rotary(10))
    with pytest.raises(WinogradError, match="start"):
        S.head_norm_rotate(q, q, w, w, rot, start=2 ** 31)
    with pytest.raises(WinogradError, match="eps"):
        S.head_norm_rotate(q, q, w, w, rot, eps=-1.0)
    with pytest.raises(WinogradError, match="256"):
        x, one = torch.zeros((1, 1, 1, 258), device="cuda"), torch.ones(258, device="cuda")
        S.head_norm_rotate(x, x, one, one, rot)
    with pytest.raises(WinogradError, match="overlap"):
        S.head_norm_rotate(q, q, w, w, rot, q_out=torch.zeros((1, 5, 2, 8), device="cuda").expand(2, 5, 2, 8))
    with pytest.raises(ValueError):
        S.head_norm_rotate_backward(q, q, q, q, w, w, rot, out=[q.clone()])
