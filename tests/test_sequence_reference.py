"""The 64-bit references of the sequence operators on the CPU: their gradients
against central differences of their own outputs, and their padding."""
import numpy as np
import pytest

import sequence_reference as R


def _case(seed, N=3, L=9, C=4):
    g = np.random.Generator(np.random.PCG64(seed))
    z, v, o = (g.standard_normal((N, L, C)) for _ in range(3))
    return g, z + 1.0, v, o, g.standard_normal((N, C)), np.array([L, 0, 5])


@pytest.mark.parametrize("out_gate", [False, True])
@pytest.mark.parametrize("padded", [False, True])
def test_scan_gradients_against_differences(out_gate, padded):
    g, z, v, o, h0, lengths = _case(3 + out_gate)
    o = o if out_gate else None
    lengths = lengths if padded else None
    dy, dh = g.standard_normal(z.shape), g.standard_normal(h0.shape)

    def loss(z, v, o, h0):
        r = R.scan(z, v, o, h0, lengths)
        return float((r["y"][0] * dy).sum() + (r["h_last"][0] * dh).sum())

    grads = R.scan(z, v, o, h0, lengths, dy, dh)
    at = {"dgate": 0, "dvalue": 1, "dout_gate": 2, "dh0": 3}
    for name, k in at.items():
        args = [z, v, o, h0]
        if args[k] is None:
            continue
        d = g.standard_normal(args[k].shape)
        step = 1e-5
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + step * d, args[k] - step * d
        num = (loss(*up) - loss(*down)) / (2 * step)
        # the difference is off by the third derivative times step^2, and by 1e-16 / step
        assert abs(num - float((grads[name][0] * d).sum())) <= 1e-8 * max(1.0, abs(num)), name


@pytest.mark.parametrize("residual", [False, True])
def test_norm_gradients_against_differences(residual):
    g = np.random.Generator(np.random.PCG64(5))
    r, dy, w = g.standard_normal((5, 7)), g.standard_normal((5, 7)), g.standard_normal(7)
    dr = g.standard_normal(r.shape) if residual else None

    def loss(r, w):
        return float((R.norm(r, None, w, 1e-3)[1] * dy).sum() + (0.0 if dr is None else (r * dr).sum()))

    dx, _, dw, _ = R.norm_gradients(dy, r, w, dr, 1e-3)
    step = 1e-5
    for k, grad in ((0, dx), (1, dw)):
        d = g.standard_normal(grad.shape)
        up, down = [r, w], [r, w]
        up[k], down[k] = up[k] + step * d, down[k] - step * d
        num = (loss(*up) - loss(*down)) / (2 * step)
        assert abs(num - float((grad * d).sum())) <= 1e-8 * max(1.0, abs(num))


def test_padding_is_not_used():
    g, z, v, o, h0, lengths = _case(11)
    dy = g.standard_normal(z.shape)
    want = R.scan(z, v, o, h0, lengths, dy)
    live = np.arange(z.shape[1])[None, :, None] < lengths[:, None, None]
    nan = [np.where(live, t, np.nan) for t in (z, v, o, dy)]
    got = R.scan(*nan[:3], h0, lengths, nan[3])
    for name in want:
        assert np.array_equal(want[name][0], got[name][0]), name
    assert np.array_equal(want["h_last"][0][1], h0[1]) and not want["y"][0][1].any()
