"""Linear attention at the ends of its numbers' ranges: decays down to the lowest finite
one, and infinities and NaN, which go on as the recurrence has them; for sequences, their
gradients and the single step.  And the norm of heads with rotation, where infinities stay
in the channels that the formula brings them to."""
import numpy as np
import pytest
import torch

import attention_reference as A
import sequence_reference as R
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu

NAMES = ("y", "s_last", "dq", "dk", "dv", "ds0")


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)


def _np(t):
    return t.double().cpu().numpy()


def _inputs(N, L, H, Dk, Dv, dtype):
    """q, k, v and dy of H heads each, s0 and the gradient at the last state."""
    rows = [torch.randn((N, L, H, d), device="cuda").to(TORCH[dtype]) for d in (Dk, Dk, Dv, Dv)]
    return (*rows, *[torch.randn((N, H, Dk, Dv), device="cuda") for _ in range(2)])


def _run(q, k, v, dy, s0, ds, g, lengths=None):
    from paper_1905_05233_amd import sequence_ops as S
    return dict(zip(NAMES, (*S.linear_attention(q, k, v, g, s0=s0, lengths=lengths),
                            *S.linear_attention_backward(dy, q, k, v, g, s0=s0, ds_last=ds, lengths=lengths))))


def _reference(q, k, v, dy, s0, ds, g, dtype, lengths=None):
    return A.attention(_np(q), _np(k), _np(v), _np(g), _np(s0), lengths, q.shape[-1] ** -0.5, dtype, _np(dy), _np(ds))


# -2.4e38 log2(e) and what is below it exceed fp32's range
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("decay", [-88.0, -104.0, -1e4, -1e30, -2.4e38, float(np.finfo(np.float32).min), -float("inf")], ids=str)
def test_decays_that_keep_nothing(decay, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    g = torch.tensor([decay, -0.01], device="cuda")
    for L in (1, 70, 700):     # a tile, and sequences that go in segments
        inputs = _inputs(1, L, 2, 24, 40, dtype)
        got, ref = _run(*inputs, g), _reference(*inputs, g, dtype)
        for name in NAMES:
            R.assert_close(_np(got[name]), *ref[name], "f32" if name in ("s_last", "ds0") else dtype, name)
    q, k, v, _, s0, _ = inputs
    y, s = S.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], g, s0)
    ref = A.attention(*[_np(t[:, :1]) for t in (q, k, v)], _np(g), _np(s0), None, 24 ** -0.5, dtype)
    R.assert_close(_np(y)[:, None], *ref["y"], dtype, "y")
    R.assert_close(_np(s), *ref["s_last"], "f32", "s")



@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 2, 3, 24, 40), (2, 5, 3, 64, 64), (1, 33, 3, 100, 128), (1, 70, 3, 130, 200), (1, 1500, 3, 64, 72)], ids=str)
def test_states_of_16_bits_are_fp32s(shape, dtype):
    """The last state and its gradient come in fp32, whatever the inputs: a term enters the
    products in three parts (2^-24 of it is left, and 2^-24 by a product of fp16's parts that is
    left out), and a run of 32 steps in five matrix instructions at most, whose sums may drop
    2^-23 each: 12 2^-24 of the terms' size, which is the bound of fp32 inputs.  (Two parts, with
    2^-16 left, would be up to 5 times beyond it here.)"""
    print(f"[states] {shape} {dtype}", flush=True)
    inputs, g = _inputs(*shape, dtype), torch.tensor([-0.02, -0.3, -1.0], device="cuda")
    got, ref = _run(*inputs, g), _reference(*inputs, g, "f32")
    for name in ("s_last", "ds0"):
        R.assert_close(_np(got[name]), *ref[name], "f32", name)


def _hold(got, ref, dtype, lengths=None):
    """Infinities and NaN where the reference has them, all else within its bound."""
    for name in got:
        (want, bound), t = ref[name], _np(got[name])
        if lengths is not None and name in ("y", "dq"):   # padding, of which the reference makes 0 times the state
            for n, e in enumerate(lengths):
                want[n, e:] = bound[n, e:] = 0.0
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(t), np.isnan(want)), (name, "NaN", np.argwhere(np.isnan(t) != np.isnan(want))[:4].tolist())
        assert np.array_equal(t[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), (name, "infinity")
        assert np.isfinite(bound[fine]).all()
        R.assert_close(t[fine], want[fine], bound[fine], "f32" if name in ("s_last", "ds0") else dtype, name)


# sequences, steps, heads, channels of q and k and of v: one for each width of a state and of
# its columns, the last ones long enough to go in segments
SHAPES = [(2, 70, 2, 24, 40), (1, 100, 1, 64, 64), (1, 130, 1, 100, 128), (1, 90, 1, 40, 100), (1, 70, 1, 200, 30),
          (1, 65, 1, 130, 256), (1, 3, 1, 5, 3), (1, 1500, 1, 32, 80), (2, 700, 2, 64, 64), (1, 900, 1, 130, 70)]
INPUTS = ("q", "k", "v", "dy", "s0", "ds")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("which", INPUTS)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_infinities_go_on_as_the_recurrence_has_them(shape, which, dtype):
    print(f"[infinities] {shape} {which} {dtype}", flush=True)
    N, L, H, Dk, Dv = shape
    g = torch.tensor([-0.01, -0.3][:H], device="cuda")
    for bad in ([float("inf")], [float("inf"), -float("inf"), float("nan")]):
        inputs = _inputs(*shape, dtype)
        t = inputs[INPUTS.index(which)]
        for i, b in enumerate(bad):
            if which in ("s0", "ds"):
                t[0, 0, (5 * i + 1) % Dk, (7 * i + 2) % Dv] = b
            else:
                t[0, (L // 3 + 19 * i) % L, 0, (5 * i + 1) % t.shape[-1]] = b
        got = _run(*inputs, g)
        with np.errstate(all="ignore"):
            _hold(got, _reference(*inputs, g, dtype), dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("L", [150, 1500])
def test_infinities_with_lengths_and_shared_heads(L, dtype):
    N, H, Dk, Dv, lengths = 4, 2, 48, 40, [L, 0, L - 70, 33]
    q, k, v, dy, s0, ds = _inputs(N, L, H, Dk, Dv, dtype)
    k, v = k[:, :, :1], v[:, :, 1:]
    g, n = torch.tensor([-0.02, -0.2], device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    v[0, L // 2, 0, 7] = k[2, 30, 0, 3] = dy[3, 20, 1, 0] = float("inf")
    q[2, 31, 0, 5] = s0[1, 0, 2, 2] = ds[1, 1, 3, 3] = -float("inf")
    for i, e in enumerate(lengths):
        for t in (q, k, v, dy):
            t[i, e:] = float("inf")      # padding is not used
    got = _run(q, k, v, dy, s0, ds, g, lengths=n)
    with np.errstate(all="ignore"):
        _hold(got, _reference(q, k, v, dy, s0, ds, g, dtype, np.array(lengths)), dtype, lengths)
    for name in ("y", "dq", "dk", "dv"):
        for i, e in enumerate(lengths):
            assert not got[name][i, e:].any(), name


def test_infinities_last_over_segments_whose_decay_is_zero():
    """The decay over a segment may be below fp32's range: an infinity stays all the same."""
    inputs = _inputs(1, 2000, 1, 24, 40, "bf16")
    inputs[2][0, 3, 0, 5], inputs[3][0, 1990, 0, 6] = float("inf"), -float("inf")
    g = torch.tensor([-0.9], device="cuda")
    got = _run(*inputs, g)
    with np.errstate(all="ignore"):
        _hold(got, _reference(*inputs, g, "bf16"), "bf16")
    assert bool(torch.isinf(got["s_last"][0, 0, :, 5]).all()) and bool(torch.isinf(got["ds0"][0, 0, :, 6]).all())


def test_products_beyond_fp32():
    """q.k of finite inputs may exceed fp32's range where the state and its product with q do not."""
    N, L, D = 1, 70, 32
    inputs = [t.clone() for t in _inputs(N, L, 1, D, D, "f32")]
    inputs[0][0, 20, 0] *= 2.0 ** 70
    inputs[1][0, 20, 0] *= 2.0 ** 70
    inputs[2][0, 20, 0] *= 2.0 ** -90
    g = torch.tensor([-0.1], device="cuda")
    got, ref = _run(*inputs, g), _reference(*inputs, g, "f32")
    for name in ("y", "s_last"):
        assert np.isfinite(ref[name][0]).all() and np.abs(ref[name][0]).max() < 2.0 ** 127
        R.assert_close(_np(got[name]), *ref[name], "f32", name)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("which", ("q", "k", "v", "s0"))
def test_infinities_in_a_step(which, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    inputs, g = _inputs(2, 1, 2, 24, 37, dtype), torch.tensor([-0.01, -0.3], device="cuda")
    inputs[INPUTS.index(which)][0, 0, 1, 3] = -float("inf")
    q, k, v, _, s0, _ = inputs
    y, s = S.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], g, s0)
    with np.errstate(all="ignore"):
        ref = A.attention(*[_np(t) for t in (q, k, v)], _np(g), _np(s0), None, 24 ** -0.5, dtype)
        _hold({"y": y[:, None], "s_last": s}, ref, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("D, R_", [(40, 30), (64, 32), (75, 10), (17, 16), (16, 16)])
def test_infinities_stay_in_channels_that_are_not_turned(D, R_, adjacent, dtype):
    """An infinite weight is in its channel's outputs alone, or in its pair's; an infinite
    dy in the gradients of its row, and of the weights of its channel or pair alone."""
    from paper_1905_05233_amd import sequence_ops as S
    half = R_ // 2
    x, dy = [torch.randn((2, 5, 2, D), device="cuda").to(TORCH[dtype]) for _ in range(2)]
    w, rot, f = torch.ones(D, dtype=TORCH[dtype], device="cuda"), S.Rotary(R_, adjacent=adjacent), [10000.0 ** (-i / half) for i in range(half)]
    where = np.tile(3 + np.arange(5), (2, 1))      # no angle whose sine or cosine is 0
    want, bound = A.rotate(_np(x), _np(w), f, where, 1e-6, adjacent)
    _, (want_w, bound_w) = A.rotate(_np(x), _np(w), f, where, 1e-6, adjacent, _np(dy))
    for c in range(D):
        pair = {c} if c >= R_ else {c, c ^ 1} if adjacent else {c, c + half if c < half else c - half}
        rest = [i for i in range(D) if i not in pair]
        bad = w.clone()
        bad[c] = float("inf")
        y, _ = S.head_norm_rotate(x, x, bad, w, rot, start=3)
        assert not np.isfinite(_np(y)[..., sorted(pair)]).any()
        R.assert_close(_np(y)[..., rest], want[..., rest], bound[..., rest], dtype, "y")
        bad = dy.clone()
        bad[1, 2, 0, c] = float("inf")
        dx, _, dw, _ = S.head_norm_rotate_backward(bad, dy, x, x, w, w, rot, start=3)
        assert not np.isfinite(_np(dw)[sorted(pair)]).any()
        R.assert_close(_np(dw)[rest], want_w[rest], bound_w[rest], "f32", "dw")
        keep = torch.ones((2, 5, 2), dtype=torch.bool, device="cuda")
        keep[1, 2, 0] = False
        assert bool(torch.isfinite(dx[keep]).all())


def test_heads_without_channels_are_refused():
    from paper_1905_05233_amd import sequence_ops as S
    from paper_1905_05233_amd._native import WinogradError
    q, v, g = torch.zeros((2, 5, 1, 0), device="cuda"), torch.zeros((2, 5, 1, 8), device="cuda"), torch.zeros(1, device="cuda")
    with pytest.raises(WinogradError, match="positive"):
        S.linear_attention(q, q, v, g)
    with pytest.raises(WinogradError, match="positive"):
        S.linear_attention_backward(v, q, q, v, g)
    with pytest.raises(WinogradError, match="positive"):
        S.linear_attention_step(q[:, 0], q[:, 0], v[:, 0], g, torch.zeros((2, 1, 0, 8), device="cuda"))
