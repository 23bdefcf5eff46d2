"""The example layer's gradients for sequences as short as its convolution and
shorter, tap by tap against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

import sequence_reference as R

pytestmark = pytest.mark.gpu


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("L", [1, 2, 3, 4, 7])
def test_gradients_of_short_sequences(L):
    """fp32 with F(2, 3): its sums of 3 C products are off by some 1e-6 of their size,
    and gates, recurrence and norm keep that below 1e-4 of the largest gradient here."""
    from paper_1905_05233_amd.gated_conv import GatedConv
    N, C = 3, 32
    torch.manual_seed(L)
    layer = GatedConv(C, dtype="f32", seed=6)
    layer.norm_weight.copy_(torch.rand(C) + 0.5)
    x, dy, dr = (torch.randn((N, L, C), device="cuda") for _ in range(3))
    y, r, saved = layer.forward(x)
    dx, dweight, dnorm = layer.backward(dy, saved, dr=dr)

    w, weight = _np(layer.weight), _np(layer.norm_weight)
    _, n, _ = R.norm(_np(x), None, weight, layer.eps)
    pad = np.concatenate((np.zeros((N, 2, C)), n), 1)
    u = sum(pad[:, j:j + L] @ w[:, j].T for j in range(3))
    s = R.scan(u[..., :C], u[..., C:2 * C], u[..., 2 * C:], None, None, _np(dy))
    du = np.concatenate([s[k][0] for k in ("dgate", "dvalue", "dout_gate")], 2)
    dn = np.zeros((N, L, C))
    for j in range(3):
        back = 2 - j
        # tap j of step l meets the token l - back
        want = np.einsum("nlk,nlc->kc", du, pad[:, j:j + L])
        assert np.abs(_np(dweight[:, j]) - want).max() <= 1e-4 * max(1.0, np.abs(want).max()), (L, j)
        if back < L:
            dn[:, :L - back] += du[:, back:] @ w[:, j]
    want, _, wantw, _ = R.norm_gradients(dn, _np(x), weight, _np(dr), layer.eps)
    assert np.abs(_np(dx) - want).max() <= 1e-4 * max(1.0, np.abs(want).max())
    assert np.abs(_np(dnorm) - wantw).max() <= 1e-4 * max(1.0, np.abs(wantw).max())
