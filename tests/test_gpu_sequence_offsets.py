"""Rows further apart than 32 bits of bytes or elements: the same results as the
same rows close together."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)


@pytest.fixture(scope="module")
def far():
    """bf16 rows whose last one starts some 11 GiB behind the first."""
    buf = torch.empty(6 * 2 ** 30, dtype=torch.bfloat16, device="cuda")

    def place(t, at):   # [2][40][C]: sequences 2^32 + 64 elements apart, steps 2^25 + 8
        out = buf[at:].as_strided(t.shape, (2 ** 32 + 64, 2 ** 25 + 8, 1))
        out.copy_(t)
        return out
    yield place
    del buf
    torch.cuda.empty_cache()


def test_far_rows(far):
    from paper_1905_05233_amd import sequence_ops as S
    z, v, o, dy = (torch.randn((2, 40, 72), device="cuda").bfloat16() for _ in range(4))
    y, h, s = S.gated_scan(z, v, o, save_states=True)
    want = S.gated_scan_backward(dy, z, v, s, out_gate=o)
    fz, fv, fo, fd, fy = (far(t, 1024 * (1 + k)) for k, t in enumerate((z, v, o, dy, y)))
    fy.zero_()
    assert torch.equal(S.gated_scan(fz, fv, fo, y=fy)[1], h) and torch.equal(fy, y)
    got = S.gated_scan_backward(fd, fz, fv, s, out_gate=fo, out=[fy, far(y, 8192), far(y, 9216)])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    w = torch.rand(72, device="cuda").bfloat16()
    y, r = S.rms_norm(v, w, residual=dy)
    fy.zero_()
    assert torch.equal(S.rms_norm(fv, w, residual=fd, y=fy)[1], r) and torch.equal(fy, y)
    want = S.rms_norm_backward(dy, v, w)
    got = S.rms_norm_backward(fd, fv, w, dx=fy)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    m = S.W4Matrix.quantize(torch.randn((50, 72), device="cuda"), 32)
    assert torch.equal(S.matvec_w4(fv[0], m), S.matvec_w4(v[0], m))
