"""Linear attention and the norm of heads with rotation in 64 bits, written step by
step with numpy, and the bounds on how far the kernels' arithmetic may be off.

Bounds of the attention.  A term of a sum is a product of inputs, decays and the
scale.  Relative to the term's size, an fp32 operation adds at most 2^-24, and so
does each addition to the size of the sum's terms together; decays over n steps are
exp2 of a rounded n log2(lambda), whose error goes with n |log lambda|.  With A the
state of the absolute values, a state's bound is therefore the recurrence
E[l] = lambda (E[l-1] + 4 u |log lambda| A[l-1]) + 4 u A[l], u = 2^-24: a rounding or two
a step for the sums, one for the decays' products.
Values made in fp32 enter the matrix products in bf16 parts.  A bf16 rounding is off by
2^-8 of its value at most, so two parts leave 2^-16 and three 2^-24; of fp16 inputs the
product of the two lower parts is left out (2^-16), of fp32 ones those from 2^-24 on (two
of 2^-24, one of 2^-32).  A term passes three such products (the weights, the state or
v, the output): PART covers them.  The dot products over D channels add D roundings.
"""
import numpy as np

from sequence_reference import TINY, U

u = U["f32"]
PART = {"f32": 3 * 4 * 2.0 ** -24, "f16": 3 * 2 * 2.0 ** -16, "bf16": 3 * 2.0 ** -16}


def _shared(x, h):
    """[N][L][H][D] summed over the heads that share an input."""
    N, L, H, D = x.shape
    return x.reshape(N, L, h, H // h, D).sum(3)


def attention(q, k, v, g, s0, lengths, scale, dtype, dy=None, ds=None):
    """Outputs and, with dy, gradients: a dict of (value, bound before its rounding)."""
    N, L, Hq, Dk = q.shape
    Hk, (Hv, Dv), H = k.shape[2], v.shape[2:], len(g)
    lengths = np.full(N, L) if lengths is None else np.clip(lengths, 0, L)
    live = np.arange(L)[None] < lengths[:, None]

    def heads(x):
        return np.where(live[:, :, None, None], x, 0.0).repeat(H // x.shape[2], axis=2)

    q, k, v = heads(q), heads(k), heads(v)
    lam = np.exp(g)[None, :, None, None]
    slope = 4 * u * np.minimum(np.abs(g), 1e3)[None, :, None, None]
    S = np.zeros((N, H, Dk, Dv)) if s0 is None else s0.copy()
    A, E = np.abs(S), np.zeros_like(S)
    part, near = PART[dtype], (2 * max(Dk, Dv) + 96) * u
    y, by = np.zeros((N, L, H, Dv)), np.zeros((N, L, H, Dv))
    dq, bq = np.zeros((N, L, H, Dk)), np.zeros((N, L, H, Dk))
    if dy is not None:
        dy = np.where(live[:, :, None, None], dy, 0.0)

    def times(M, x):   # M x over the last axis
        return np.einsum("nhij,nhj->nhi", M, x)

    def back(M, x):
        return np.einsum("nhij,nhi->nhj", M, x)

    for l in range(L):
        up = live[:, l, None, None, None]
        kv = k[:, l, :, :, None] * v[:, l, :, None, :]
        An = lam * A + np.abs(kv)
        En = lam * (E + slope * A) + 4 * u * An
        S, A, E = np.where(up, lam * S + kv, S), np.where(up, An, A), np.where(up, En, E)
        y[:, l] = scale * back(S, q[:, l])
        by[:, l] = abs(scale) * back(E + (part + near) * A, np.abs(q[:, l]))
        if dy is not None:
            dq[:, l] = scale * times(S, dy[:, l])
            bq[:, l] = abs(scale) * times(E + (part + near) * A, np.abs(dy[:, l]))
    out = {"y": (y, by), "s_last": (S, E + part * A)}
    if dy is None:
        return out
    G = np.zeros((N, H, Dk, Dv)) if ds is None else ds.copy()
    A, E = np.abs(G), np.zeros_like(G)
    dk, bk, dv, bv = np.zeros_like(dq), np.zeros_like(dq), np.zeros_like(y), np.zeros_like(y)
    for l in range(L - 1, -1, -1):
        up = live[:, l, None, None, None]
        qd = scale * q[:, l, :, :, None] * dy[:, l, :, None, :]
        G, A = G + np.where(up, qd, 0.0), A + np.where(up, np.abs(qd), 0.0)
        E = E + np.where(up, 4 * u * A, 0.0)
        at = live[:, l, None, None]
        dk[:, l], dv[:, l] = np.where(at, times(G, v[:, l]), 0.0), np.where(at, back(G, k[:, l]), 0.0)
        B = E + (part + near) * A
        bk[:, l], bv[:, l] = np.where(at, times(B, np.abs(v[:, l])), 0.0), np.where(at, back(B, np.abs(k[:, l])), 0.0)
        G, E, A = np.where(up, lam * G, G), np.where(up, lam * (E + slope * A), E), np.where(up, lam * A, A)
    share = 1 + H * u   # the sums over heads that share an input
    return out | {"dq": (_shared(dq, Hq), _shared(bq, Hq) * share), "dk": (_shared(dk, Hk), _shared(bk, Hk) * share),
                  "dv": (_shared(dv, Hv), _shared(bv, Hv) * share), "ds0": (G, E + part * A)}


def _turned(x, c, s, R, adjacent):
    a, b = (slice(0, R, 2), slice(1, R, 2)) if adjacent else (slice(0, R // 2), slice(R // 2, R))
    y, size = x.copy(), np.abs(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def rotate(x, w, frequencies, positions, eps, adjacent, dy=None):
    """(y, bound), or with dy ((dx, bound), (dw, bound)).  Angles in 80 bits: the product
    of a far position and a frequency exceeds 64.  The norm is off as in
    sequence_reference; a turn adds an angle's error below 2^-30, the sine's and
    cosine's own of 2 units, and three roundings, relative to the pair's size."""
    R, D = 2 * len(frequencies), x.shape[-1]
    angle = positions.astype(np.longdouble)[..., None, None] * np.array(frequencies, dtype=np.longdouble)
    c, s = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)
    rstd = 1.0 / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    k = (D / 2 + 20) * u
    if dy is None:
        y, size = _turned(x * rstd * w, c, s, R, adjacent)
        return y, size * k
    du, size = _turned(dy, c, -s, R, adjacent)
    g, ga = du * w, size * np.abs(w)
    k = (D + 32) * u
    mean = np.mean(g * x, axis=-1, keepdims=True) * rstd * rstd
    mabs = np.mean(ga * np.abs(x), axis=-1, keepdims=True) * rstd * rstd
    rows = x.size // D
    dw = (du * x * rstd).reshape(rows, D)
    bw = (size * np.abs(x) * rstd).reshape(rows, D).sum(0) * (rows + D / 2 + 32) * u
    return (rstd * (g - x * mean), rstd * (ga + 3 * np.abs(x) * mabs) * k), (dw.sum(0), bw)


__all__ = ["attention", "rotate", "TINY", "U"]
