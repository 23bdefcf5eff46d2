"""Linear attention at the ends of its numbers' ranges: decays down to the lowest finite
one, for sequences, their gradients and the single step."""
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
