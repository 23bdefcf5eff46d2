"""More rows, channels or weights than one launch takes threads."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)
    yield
    torch.cuda.empty_cache()


def test_products_of_many_rows():
    """More than 2^20 rows of x."""
    from paper_1905_05233_amd import sequence_ops as S
    w = S.W4Matrix.quantize(torch.randn((5, 40), device="cuda"), 32)
    some = torch.randn((1000, 40), device="cuda").bfloat16()
    M = 2 ** 20 + 1003
    x = some.repeat(-(-M // 1000), 1)[:M]
    y, want = S.matvec_w4(x, w), S.matvec_w4(some, w)
    assert torch.equal(y, want.repeat(-(-M // 1000), 1)[:M])
    scales = torch.rand((M, 1), device="cuda") + 0.5
    q = x.to(torch.float8_e4m3fn)
    y = S.matvec_w4(q, w, x_scales=scales)
    for at in (0, 2 ** 20 - 20, M - 100):
        assert torch.equal(y[at:at + 100], S.matvec_w4(q[at:at + 100], w, x_scales=scales[at:at + 100]))


def test_products_with_many_outputs():
    """2^30 rows of the matrix and some more: one column, as its tiles are 64 bytes a row."""
    from paper_1905_05233_amd import sequence_ops as S
    rows = 2 ** 30 + 40
    w = S.W4Matrix._empty(rows, 1, 32, "cuda")
    small = S.W4Matrix.quantize(torch.randn((1600, 1), device="cuda"), 32)
    tiles = w.tiles.shape[0]
    for at in range(0, tiles, 100):
        if at >= 3200 and at + 3200 < tiles and at % 1000000:
            continue                        # the rest holds whatever it holds
        n = min(100, tiles - at)
        w.tiles[at:at + n] = small.tiles[:n]
        w.scales[at:at + n] = small.scales[:n]
    x = torch.randn((3, 1), device="cuda").bfloat16()
    y, want = S.matvec_w4(x, w), S.matvec_w4(x, small)
    for at in (0, 1000000, tiles // 100 * 100 - 1000, tiles // 100 * 100):
        n = min(100, tiles - at) * 16
        n = min(n, rows - at * 16)
        assert torch.equal(y[:, at * 16:at * 16 + n], want[:, :n]), at


def test_step_of_many_channels():
    """More than 2^32 states."""
    from paper_1905_05233_amd import sequence_ops as S
    N, C = 4099, 2 ** 20
    z, v, o = (torch.randn((1, C), device="cuda").bfloat16() for _ in range(3))
    h = torch.randn((1, C), device="cuda")
    wy, wh = S.gated_step(z, v, h, out_gate=o)
    big = h.repeat(N, 1)
    y, new = S.gated_step(z.expand(N, C), v.expand(N, C), big, out_gate=o.expand(N, C), h_new=big)
    for at in range(0, N, 500):
        assert bool((new[at:at + 500] == wh).all()) and bool((y[at:at + 500] == wy).all()), at


def test_making_large_matrices():
    """Matrices of more groups, words or runs of columns than 2^32."""
    from paper_1905_05233_amd import sequence_ops as S
    rows = 2 ** 30 + 48
    some = torch.randn((1600, 1), device="cuda").bfloat16()
    small = S.W4Matrix.quantize(some, 32)
    w = S.W4Matrix.quantize(some.repeat(-(-rows // 1600), 1)[:rows], 32)
    for at in (0, 10 ** 7, rows // 1600 * 100 - 100):
        assert torch.equal(w.tiles[at:at + 100], small.tiles) and torch.equal(w.scales[at:at + 100], small.scales)
    n = w.tiles.shape[0] % 100
    assert torch.equal(w.tiles[-n:], small.tiles[:n]) and torch.equal(w.scales[-n:], small.scales[:n])
    del w
    torch.cuda.empty_cache()

    rows = 2 ** 28 + 48
    codes = torch.randint(0, 256, (1600, 1), device="cuda").to(torch.uint8)
    scales = torch.rand((1600, 1), device="cuda").bfloat16()
    small = S.W4Matrix.from_nibbles(codes, scales, 1)
    w = S.W4Matrix.from_nibbles(codes.repeat(-(-rows // 1600), 1)[:rows], scales.repeat(-(-rows // 1600), 1)[:rows], 1)
    for at in (0, 10 ** 7, rows // 1600 * 100 - 100):
        assert torch.equal(w.tiles[at:at + 100], small.tiles) and torch.equal(w.scales[at:at + 100], small.scales)
    del w
    torch.cuda.empty_cache()

    rows, cols = 2 ** 22 + 16, 8192
    small = S.W4Matrix.quantize(torch.randn((16, cols), device="cuda"), 128)
    w = S.W4Matrix._empty(rows, cols, 128, "cuda")
    w.tiles.copy_(small.tiles.expand_as(w.tiles))
    w.scales.copy_(small.scales.expand_as(w.scales))
    m, want = w.dequantize().view(-1, 16, cols), small.dequantize()
    for at in range(0, rows // 16, 2 ** 14):
        assert bool((m[at:at + 2 ** 14] == want).all()), at


@pytest.mark.parametrize("shape", [(2 ** 21 + 3, 1, 1024), (1, 35, 2 ** 29 + 64)], ids=str)
def test_scan_of_many_channels(shape):
    """More channels than one launch has threads: many sequences of a step, and one
    wide one."""
    from paper_1905_05233_amd import sequence_ops as S
    N, L, C = shape
    some = 1024
    parts = [torch.randn((1, L, some), device="cuda").bfloat16() for _ in range(3)]
    want = S.gated_scan(*parts[:2], save_states=True)
    grads = S.gated_scan_backward(parts[2], *parts[:2], want[2])
    if N > 1:
        wide = [p.expand(N, L, some) for p in parts]
    else:   # every input row is the same memory, with the channels repeated
        parts = [p[:, :1].expand(1, L, some) for p in parts]
        want = S.gated_scan(*parts[:2], save_states=True)
        grads = S.gated_scan_backward(parts[2], *parts[:2], want[2])
        wide = [p[:, :1].repeat(1, 1, -(-C // some))[:, :, :C].expand(1, L, C) for p in parts]
    y, h, s = S.gated_scan(*wide[:2], save_states=True)

    def same(got, ref):   # [N or 1][..][C] against [1][..][some]
        if N > 1:
            return all(bool((got[at:at + 2 ** 18] == ref).all()) for at in range(0, N, 2 ** 18))
        whole = C // some * some
        ok = torch.equal(got[..., whole:], ref[..., :C - whole])
        for l in range(0, whole, 2 ** 24):
            part = got[..., l:min(l + 2 ** 24, whole)]
            ok = ok and bool((part.unflatten(-1, (-1, some)) == ref.unsqueeze(-2)).all())
        return ok

    assert same(y, want[0]) and same(h, want[1]) and same(s, want[2])
    del y, h
    dz, dv, _, dh = S.gated_scan_backward(wide[2], *wide[:2], s)
    assert same(dz, grads[0]) and same(dv, grads[1]) and same(dh, grads[3])


def test_no_sequences():
    from paper_1905_05233_amd import sequence_ops as S
    e = torch.empty((0, 5, 8), device="cuda").bfloat16()
    h = torch.empty((0, 8), device="cuda")
    lengths = torch.empty(0, dtype=torch.int32, device="cuda")
    y, last, states = S.gated_scan(e, e, e, h0=h, lengths=lengths, save_states=True)
    assert y.shape == e.shape and last.shape == (0, 8) and states.shape == (0, 1, 8)
    dz, dv, do, dh = S.gated_scan_backward(e, e, e, states, out_gate=e, dh_last=h, lengths=lengths)
    assert dz.shape == dv.shape == do.shape == e.shape and dh.shape == (0, 8)
    with pytest.raises(ValueError):
        S.gated_scan(e, e, h0=torch.empty((1, 8), device="cuda"))
