"""The sequence operators' C ABI on the CPU: argument checks and workspace sizes.
No kernel is launched: every call here is refused, or asks for a size."""
import ctypes

import pytest

from paper_1905_05233_amd import _native as N
from paper_1905_05233_amd import sequence_ops as S

P = 1 << 20      # a pointer that nothing follows
ROWS = (P, 640, 64)
NONE = (0, 0, 0)
ARG, UNSUPPORTED, WORKSPACE = 1, 5, 7


def _scan(dtype=2, n=2, l=10, c=64, gate=ROWS, value=ROWS, out_gate=NONE, y=ROWS, h0=0, lengths=0, h_last=P, states=0,
          ws=0, nbytes=0):
    return N.lib().winograd_gated_scan(S._pack_scan(dtype, n, l, c, *gate, *value, *out_gate, *y, h0, lengths, h_last,
                                                    states, ws, nbytes), None)


def _message():
    return N.lib().winograd_last_error().decode()


@pytest.mark.parametrize("status,words,args", [
    (UNSUPPORTED, "dtype", dict(dtype=3)),
    (ARG, "sizes", dict(n=0)),
    (ARG, "sizes", dict(c=0)),
    (ARG, "sizes", dict(l=-1)),
    (ARG, "sizes", dict(n=1 << 31)),
    (UNSUPPORTED, "large", dict(n=1 << 20, l=1 << 21)),
    (UNSUPPORTED, "steps", dict(n=1, l=(1 << 31) - 1, c=8)),
    (UNSUPPORTED, "channels", dict(n=1, l=8, c=(1 << 30) + 1)),
    (ARG, "null tensor gate", dict(gate=NONE)),
    (ARG, "aligned", dict(value=(P + 1, 640, 64))),
    (ARG, "strides", dict(value=(P, -1, 64))),
    (ARG, "strides", dict(value=(P, 640, 1 << 60))),
    (ARG, "rows of y overlap", dict(y=(P, 640, 63))),
    (ARG, "rows of y overlap", dict(y=(P, 639, 64))),
    (ARG, "rows of y overlap", dict(y=(P, 0, 64))),
    (ARG, "rows of y overlap", dict(y=(P, 64, 127))),
    (ARG, "h_last", dict(h_last=0)),
    (ARG, "h0", dict(h0=P + 2)),
    (ARG, "lengths", dict(lengths=P + 2)),
    (WORKSPACE, "workspace", dict(n=1, l=100000, gate=ROWS, value=ROWS, y=ROWS)),
    (WORKSPACE, "workspace", dict(n=1, l=100000, ws=P, nbytes=16)),
    (ARG, "workspace", dict(n=1, l=100000, ws=P + 4, nbytes=1 << 30)),
], ids=lambda v: str(v)[:40])
def test_scan_refusals(status, words, args):
    assert _scan(**args) == status and words in _message()


def test_scan_backward_refusals():
    def call(**a):
        a = {**dict(dy=ROWS, out_gate=NONE, dout=NONE, states=P, dgate=ROWS), **a}
        return N.lib().winograd_gated_scan_backward(S._pack_scan_backward(
            2, 2, 10, 64, *a["dy"], *ROWS, *ROWS, *a["out_gate"], *a["dgate"], *ROWS, *a["dout"], a["states"], 0, 0, P, 0, 0),
            None)
    assert call(dy=NONE) == ARG and "dy" in _message()
    assert call(out_gate=ROWS) == ARG and "dout_gate" in _message()
    assert call(states=0) == ARG and "states" in _message()
    assert call(dgate=(P, 64, 64)) == ARG and "overlap" in _message()
    assert N.lib().winograd_gated_scan(None, None) == ARG
    assert N.lib().winograd_gated_step(None, None) == ARG


def test_workspaces():
    size = ctypes.c_size_t(7)
    lib = N.lib()

    def scan(dtype, n, l, c, backward=0):
        assert lib.winograd_gated_scan_workspace(dtype, n, l, c, backward, ctypes.byref(size)) == 0
        return size.value

    assert scan(2, 1, 1, 512) == 0 and scan(2, 1, 0, 512) == 0
    assert scan(2, 1 << 16, 4096, 64) == 0                 # channels fill the chip: no cut
    long = scan(2, 1, 1 << 20, 64)
    assert 0 < long <= 256 * 64 * 8 and long % 16 == 0     # a map a channel of at most 256 chunks
    assert scan(2, 1, 1 << 20, 64, 1) > 0
    assert lib.winograd_gated_scan_workspace(2, 0, 5, 5, 0, ctypes.byref(size)) == ARG
    assert lib.winograd_gated_scan_workspace(2, 1, 5, 5, 0, None) == ARG
    assert lib.winograd_rms_norm_workspace(0, 0, 5, 5, ctypes.byref(size)) == 0
    assert lib.winograd_rms_norm_workspace(0, 1, 5, 1 << 26, ctypes.byref(size)) == UNSUPPORTED
    assert lib.winograd_rms_norm_workspace(2, 1, 16, 512, ctypes.byref(size)) == 0 and size.value == 0   # one part
    assert lib.winograd_rms_norm_workspace(2, 1, 17, 512, ctypes.byref(size)) == 0 and size.value == 5 * 512 * 4


@pytest.mark.parametrize("status,words,args", [
    (UNSUPPORTED, "y_dtype", dict(y_dtype=0)),
    (UNSUPPORTED, "group", dict(group=64)),
    (UNSUPPORTED, "group", dict(y_dtype=3, group=16, scales=P)),
    (ARG, "scales", dict(y_dtype=3)),
    (ARG, "eps", dict(eps=-1.0)),
    (ARG, "eps", dict(eps=float("inf"))),
    (ARG, "weight", dict(weight=0)),
    (ARG, "overlap", dict(r=(P, 0, 64))),
    (UNSUPPORTED, "channels", dict(c=1 << 26)),
], ids=lambda v: str(v)[:40])
def test_norm_refusals(status, words, args):
    a = {**dict(dtype=2, n=2, l=10, c=64, r=NONE, weight=P, scales=0, eps=1e-6, y_dtype=2, group=0), **args}
    st = N.lib().winograd_rms_norm(S._pack_norm(a["dtype"], a["n"], a["l"], a["c"], *ROWS, *NONE, *a["r"], *ROWS,
                                                a["weight"], a["scales"], a["eps"], a["y_dtype"], a["group"]), None)
    assert st == status and words in _message()


def test_norm_backward_refusals():
    def call(weight=P, dweight=P, ws=P, nbytes=1 << 20, dx=(P, 64000, 64)):
        return N.lib().winograd_rms_norm_backward(S._pack_norm_backward(2, 2, 1000, 64, *ROWS, *ROWS, *NONE, *dx, weight,
                                                                        dweight, 1e-6, ws, nbytes), None)
    assert call(weight=P + 1) == ARG and "weight" in _message()
    assert call(dweight=0) == ARG and "dweight" in _message()
    assert call(nbytes=8) == WORKSPACE and "need" in _message()
    assert call(ws=0) == WORKSPACE
    assert call(dx=(P, 640, 8)) == ARG and "overlap" in _message()


@pytest.mark.parametrize("status,words,args", [
    (ARG, "codes", dict(codes=0)),
    (ARG, "16-byte", dict(codes=P + 8)),
    (ARG, "rows and cols", dict(rows=0)),
    (UNSUPPORTED, "group", dict(group=16)),
    (UNSUPPORTED, "large", dict(rows=(1 << 31) - 1, cols=(1 << 31) - 1)),
    (UNSUPPORTED, "x_dtype", dict(xd=4)),
    (UNSUPPORTED, "y_dtype", dict(yd=3)),
    (ARG, "null tensor x", dict(x=0)),
    (ARG, "overlap", dict(ldy=31)),
    (ARG, "x_scales", dict(xd=3)),
    (ARG, "x_scales", dict(xd=3, xs=P, xg=2)),
    (ARG, "x_scales", dict(xs=P, xg=1)),
    (ARG, "M must", dict(m=-1)),
], ids=lambda v: str(v)[:40])
def test_matvec_refusals(status, words, args):
    a = {**dict(codes=P, scales=P, rows=32, cols=256, group=64, m=2, xd=2, yd=2, x=P, ldx=256, xs=0, xg=0, y=P, ldy=32), **args}
    st = N.lib().winograd_matvec_w4(S._pack_matvec(a["codes"], a["scales"], a["rows"], a["cols"], a["group"], a["m"], a["xd"],
                                                   a["yd"], a["x"], a["ldx"], a["xs"], a["xg"], a["y"], a["ldy"]), None)
    assert st == status and words in _message()
    w = S._pack_w4(0, P, 32, 256, 64)
    assert N.lib().winograd_quantize_w4(w, 2, P, 256, None) == ARG
    assert N.lib().winograd_dequantize_w4(S._pack_w4(P, P, 32, 256, 64), 3, P, 256, None) == UNSUPPORTED
    assert N.lib().winograd_pack_w4(S._pack_w4(P, P, 32, 256, 64), 0, P, None) == ARG


def test_nothing_to_do_is_no_error():
    empty = S._pack_norm(2, 0, 10, 64, *NONE, *NONE, *NONE, *NONE, P, 0, 1e-6, 2, 0)
    assert N.lib().winograd_rms_norm(empty, None) == 0
    assert N.lib().winograd_matvec_w4(S._pack_matvec(P, P, 32, 256, 64, 0, 2, 2, 0, 256, 0, 0, 0, 32), None) == 0
    assert N.lib().winograd_gated_step(S._pack_step(2, 0, 64, *NONE, *NONE, *NONE, *NONE, 0, 0), None) == 0
