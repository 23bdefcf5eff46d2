"""The norm's eps is used in fp32: one that is infinite there is refused.  Nothing is launched."""
import pytest

from paper_1905_05233_amd import _native as N
from paper_1905_05233_amd import sequence_ops as S

P, ROWS, NONE, ARG = 1 << 20, (1 << 20, 640, 64), (0, 0, 0), 1


@pytest.mark.parametrize("eps", [1e39, 1e300, float("inf"), float("nan"), -1e-6])
def test_eps(eps):
    st = N.lib().winograd_rms_norm(S._pack_norm(2, 2, 10, 64, *ROWS, *NONE, *NONE, *ROWS, 0, 0, eps, 2, 0), None)
    assert st == ARG and "eps" in N.lib().winograd_last_error().decode()
    st = N.lib().winograd_rms_norm_backward(S._pack_norm_backward(2, 2, 10, 64, *ROWS, *ROWS, *NONE, *ROWS, 0, P, eps, 0, 0),
                                            None)
    assert st == ARG and "eps" in N.lib().winograd_last_error().decode()
