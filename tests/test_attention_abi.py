"""The C ABI of linear attention and of the norm of heads with rotation on the CPU:
argument checks and workspace sizes.  No kernel is launched: every call here is refused,
has nothing to do, or asks for a size."""
import ctypes

import pytest

import paper_1905_05233_amd._native as N
from paper_1905_05233_amd import sequence_ops as S

P = 1 << 20      # a pointer that nothing follows
HEADS = (P, 6400, 640, 64)
NONE = (0, 0, 0, 0)
ARG, UNSUPPORTED, WORKSPACE = 1, 5, 7


def _message():
    return N.lib().winograd_last_error().decode()


def _attention(dtype=2, n=2, l=10, hq=8, hk=8, hv=8, h=8, dk=64, dv=64, q=HEADS, k=HEADS, v=HEADS, y=HEADS, g=P, s0=0,
               lengths=0, s_last=P, scale=1.0, ws=0, nbytes=0):
    return N.lib().winograd_linear_attention(S._pack_attention(dtype, n, l, hq, hk, hv, h, dk, dv, *q, *k, *v, *y, g, s0,
                                                               lengths, s_last, scale, ws, nbytes), None)


@pytest.mark.parametrize("status,words,args", [
    (UNSUPPORTED, "dtype", dict(dtype=3)),
    (ARG, "sizes", dict(n=-1)),
    (ARG, "sizes", dict(l=-1)),
    (ARG, "sizes", dict(n=1 << 31)),
    (ARG, "heads", dict(h=0)),
    (ARG, "heads", dict(h=1 << 17)),
    (ARG, "divide", dict(hq=3)),
    (ARG, "divide", dict(hk=0)),
    (ARG, "divide", dict(hv=16)),
    (ARG, "Dk and Dv", dict(dk=0)),
    (UNSUPPORTED, "256", dict(dv=257)),
    (UNSUPPORTED, "large", dict(n=1 << 20, l=1 << 20)),
    (UNSUPPORTED, "large", dict(n=(1 << 31) - 1, l=1)),
    (UNSUPPORTED, "steps", dict(n=1, l=(1 << 31) - 1, hq=1, hk=1, hv=1, h=1, dk=1, dv=1)),
    (ARG, "null tensor q", dict(q=NONE)),
    (ARG, "null tensor y", dict(y=NONE)),
    (ARG, "aligned", dict(k=(P + 1, 6400, 640, 64))),
    (ARG, "strides", dict(v=(P, -1, 640, 64))),
    (ARG, "strides", dict(v=(P, 6400, 640, 1 << 60))),
    (ARG, "rows of y overlap", dict(y=(P, 6400, 640, 63))),
    (ARG, "rows of y overlap", dict(y=(P, 6400, 500, 64))),
    (ARG, "rows of y overlap", dict(y=(P, 6000, 640, 64))),
    (ARG, "rows of y overlap", dict(y=(P, 0, 640, 64))),
    (ARG, "log_decay", dict(g=0)),
    (ARG, "log_decay", dict(g=P + 2)),
    (ARG, "s0", dict(s0=P + 2)),
    (ARG, "lengths", dict(lengths=P + 2)),
    (ARG, "s_last", dict(s_last=P + 1)),
    (ARG, "scale", dict(scale=float("nan"))),
    (ARG, "scale", dict(scale=1e39)),
], ids=lambda v: str(v)[:40])
def test_attention_refusals(status, words, args):
    assert _attention(**args) == status and words in _message()


def test_attention_backward_refusals():
    def call(hq=8, ws=0, nbytes=0, **a):
        a = {**dict(dy=HEADS, dq=HEADS, dk=HEADS, dv=HEADS, ds=0, ds0=P), **a}
        return N.lib().winograd_linear_attention_backward(S._pack_attention_backward(
            2, 2, 10, hq, 8, 8, 8, 64, 64, *a["dy"], *HEADS, *HEADS, *HEADS, *a["dq"], *a["dk"], *a["dv"], P, 0, a["ds"], 0,
            a["ds0"], 1.0, ws, nbytes), None)
    assert call(dy=NONE) == ARG and "null tensor dy" in _message()
    for name in ("dq", "dk", "dv"):
        assert call(**{name: (P, 0, 640, 64)}) == ARG and f"rows of {name} overlap" in _message()
    assert call(ds=P + 2) == ARG and "ds_last" in _message()
    assert call(ds0=P + 2) == ARG and "ds0" in _message()
    assert call(hq=2) == WORKSPACE and "need" in _message()          # sums over the heads that share q
    assert call(hq=2, ws=P, nbytes=16) == WORKSPACE
    assert call(hq=2, ws=P + 4, nbytes=1 << 30) == ARG and "workspace" in _message()
    assert N.lib().winograd_linear_attention(None, None) == ARG
    assert N.lib().winograd_linear_attention_backward(None, None) == ARG
    assert N.lib().winograd_linear_attention_step(None, None) == ARG


def test_attention_step_refusals():
    def call(n=2, h=8, y=HEADS, s=P, s_new=P, scale=1.0):
        return N.lib().winograd_linear_attention_step(S._pack_attention_step(
            2, n, 8, 8, 8, h, 64, 64, *HEADS, *HEADS, *HEADS, *y, P, s, s_new, scale), None)
    assert call(h=4) == ARG and "divide" in _message()
    assert call(y=(P, 64, 0, 64)) == ARG and "overlap" in _message()
    assert call(s=0) == ARG and "s" in _message()
    assert call(s_new=0) == ARG and "s_new" in _message()
    assert call(scale=float("inf")) == ARG and "scale" in _message()
    assert call(n=0) == 0


def _rotate(n=2, l=10, hq=8, hk=2, d=64, r=64, dtype=2, q=HEADS, q_out=HEADS, qw=P, kw=P, turns=P, positions=0, start=0, eps=1e-6):
    return N.lib().winograd_head_norm_rotate(S._pack_rotate(dtype, n, l, hq, hk, d, r, 0, *q, *HEADS, *q_out, *HEADS, qw, kw,
                                                            turns, positions, start, eps), None)


@pytest.mark.parametrize("status,words,args", [
    (UNSUPPORTED, "dtype", dict(dtype=3)),
    (ARG, "heads", dict(hq=0)),
    (ARG, "heads", dict(hk=0)),
    (ARG, "heads", dict(hq=1 << 17)),
    (UNSUPPORTED, "256", dict(d=257)),
    (ARG, "R must", dict(r=0)),
    (ARG, "R must", dict(r=7)),
    (ARG, "R must", dict(r=66)),
    (ARG, "sizes", dict(n=-1)),
    (UNSUPPORTED, "large", dict(n=1 << 20, l=1 << 20)),
    (ARG, "start", dict(start=1 << 31)),
    (ARG, "eps", dict(eps=-1.0)),
    (ARG, "eps", dict(eps=float("nan"))),
    (ARG, "eps", dict(eps=1e39)),
    (ARG, "null tensor q", dict(q=NONE)),
    (ARG, "aligned", dict(q=(P + 1, 6400, 640, 64))),
    (ARG, "rows of q_out overlap", dict(q_out=(P, 6400, 640, 32))),
    (ARG, "weight", dict(qw=0)),
    (ARG, "weight", dict(kw=P + 1)),
    (ARG, "turns", dict(turns=0)),
    (ARG, "turns", dict(turns=P + 4)),
    (ARG, "positions", dict(positions=P + 2)),
], ids=lambda v: str(v)[:40])
def test_rotate_refusals(status, words, args):
    assert _rotate(**args) == status and words in _message()


def test_rotate_backward_refusals():
    def call(dq=HEADS, dqw=P, ws=P, nbytes=1 << 30):
        return N.lib().winograd_head_norm_rotate_backward(S._pack_rotate_backward(
            2, 2, 10, 8, 2, 64, 64, 0, *HEADS, *HEADS, *HEADS, *HEADS, *dq, *HEADS, P, P, P, 0, 0, 1e-6, dqw, P, ws, nbytes), None)
    assert call(dq=(P, 0, 640, 64)) == ARG and "rows of dq overlap" in _message()
    assert call(dqw=0) == ARG and "dq_weight" in _message()
    assert call(ws=0) == WORKSPACE and "need" in _message()
    assert call(nbytes=16) == WORKSPACE
    assert N.lib().winograd_head_norm_rotate(None, None) == ARG
    assert N.lib().winograd_head_norm_rotate_backward(None, None) == ARG


def test_nothing_to_do_is_no_error():
    assert _rotate(n=0, q=NONE, q_out=NONE, qw=0) == 0
    assert _rotate(l=0, q=NONE, q_out=NONE, qw=0) == 0
    assert _attention(n=0, q=NONE, y=NONE, g=0) == 0


def test_workspaces():
    size = ctypes.c_size_t(7)
    lib = N.lib()

    def attention(backward, n, l, hq, hk, hv, h, dk=64, dv=32):
        args = S._pack_attention(2, n, l, hq, hk, hv, h, dk, dv, *(0,) * 20, 0.0, 0, 0)
        assert lib.winograd_linear_attention_workspace(args, backward, ctypes.byref(size)) == 0
        return size.value

    assert attention(0, 1, 1, 2, 2, 2, 2) == 0 and attention(0, 0, 5, 1, 1, 1, 1) == 0
    assert attention(1, 1, 10, 2, 2, 2, 2) == 0
    # the parts in fp32 of the gradients of shared inputs
    assert attention(1, 300, 10, 2, 2, 1, 2) - attention(1, 300, 10, 2, 2, 2, 2) == 300 * 10 * 2 * 32 * 4
    assert lib.winograd_linear_attention_workspace(None, 0, ctypes.byref(size)) == ARG
    assert lib.winograd_head_norm_rotate_workspace(2, 1, 1, 2, 64, 64, 0, ctypes.byref(size)) == 0
    assert size.value > 0 and size.value % (2 * 64 * 4) == 0
    assert lib.winograd_head_norm_rotate_workspace(2, 1, 1, 2, 64, 65, 0, ctypes.byref(size)) == ARG
    assert lib.winograd_head_norm_rotate_workspace(2, 1, 1, 2, 64, 64, 0, None) == ARG


def test_rotary_words():
    """Frequencies as fractions of a turn modulo 1, to the last bit of 64."""
    half_turn = 3.141592653589793          # fp64's pi, 1.2246e-16 below it
    words = S.Rotary(6, frequencies=[half_turn, -half_turn, 0.0], device="cpu").turns.tolist()
    off = round(1.2246467991473532e-16 / 6.283185307179586 * 2 ** 64)
    assert (words[0] - 2 ** 63) % 2 ** 64 in (2 ** 64 - off, 2 ** 64 - off - 1, 2 ** 64 - off + 1)
    assert (words[0] + words[1]) % 2 ** 64 == 0 and words[2] == 0
