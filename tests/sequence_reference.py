"""The sequence operators in 64 bits, written step by step with numpy, and the
bounds on how far an evaluation in fp32, rounded once to its type, may be off.

Bounds.  Every fp32 operation adds a relative error of at most 2^-24; the
hardware's exp2, reciprocal and square root are good to one or two units in the last place.
sigmoid(z) is exp, a sum and a reciprocal, and the exponent's own rounding enters
as |z| 2^-24: within (|z| + 8) 2^-24.  KAPPA = 64 2^-24 covers, for |z| up to 40, a
step's gate, its products and its sum.  The recurrence then gives the bound of a
state: E[l] = f E[l-1] + KAPPA H[l], with H the recurrence of the absolute
values, whatever the grouping of the steps, since a product of gates over a run
of steps is off by KAPPA a step too.
"""
import numpy as np

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}   # where rounding turns absolute
KAPPA = 64 * 2.0 ** -24


def sigmoid(z):
    t = np.exp(-np.abs(z))
    return np.where(z < 0, t, 1.0) / (1.0 + t)


def scan(z, v, o, h0, lengths, dy=None, dh_last=None):
    """Outputs, gradients (with dy) and the bounds of all of them: a dict of
    (value, bound of the fp32 evaluation before its rounding)."""
    N, L, C = z.shape
    h0 = np.zeros((N, C)) if h0 is None else h0
    lengths = np.full(N, L) if lengths is None else np.clip(lengths, 0, L)
    live = np.arange(L)[None, :, None] < lengths[:, None, None]
    z, v = np.where(live, z, 0.0), np.where(live, v, 0.0)
    f, i = sigmoid(z), sigmoid(-z)
    s = ds = np.ones_like(z)
    if o is not None:
        o = np.where(live, o, 0.0)
        sg = sigmoid(o)
        s, ds = o * sg, sg * (1.0 + o * sigmoid(-o))
    h, H, E = h0.copy(), np.abs(h0), np.zeros((N, C))
    hs, Hs, Es, before, Hb, Eb = (np.zeros((N, L, C)) for _ in range(6))
    for l in range(L):
        before[:, l], Hb[:, l], Eb[:, l] = h, H, E
        up = live[:, l]
        hn = f[:, l] * h + i[:, l] * v[:, l]
        Hn = f[:, l] * H + i[:, l] * np.abs(v[:, l])
        En = f[:, l] * E + KAPPA * Hn
        h, H, E = np.where(up, hn, h), np.where(up, Hn, H), np.where(up, En, E)
        hs[:, l], Hs[:, l], Es[:, l] = h, H, E
    zero = np.zeros_like(z)
    out = {"y": (np.where(live, hs * s, 0.0), np.where(live, np.abs(s) * (Es + KAPPA * Hs), 0.0)),
           "h_last": (h, E)}
    if dy is None:
        return out
    dy = np.where(live, dy, 0.0)
    G = np.zeros((N, C)) if dh_last is None else dh_last.copy()
    A, EG = np.abs(G), np.zeros((N, C))
    dz, dv, bz, bv = zero.copy(), zero.copy(), zero.copy(), zero.copy()
    for l in range(L - 1, -1, -1):
        up = live[:, l]
        Gn, An = G + dy[:, l] * s[:, l], A + np.abs(dy[:, l] * s[:, l])
        En = EG + KAPPA * An
        dv[:, l] = np.where(up, i[:, l] * Gn, 0.0)
        bv[:, l] = np.where(up, i[:, l] * (En + KAPPA * An), 0.0)
        fi = f[:, l] * i[:, l]
        dz[:, l] = np.where(up, fi * (before[:, l] - v[:, l]) * Gn, 0.0)
        spread = Hb[:, l] + np.abs(v[:, l])
        bz[:, l] = np.where(up, fi * (spread * (En + 2 * KAPPA * An) + (Eb[:, l] + KAPPA * spread) * An), 0.0)
        G, A = np.where(up, f[:, l] * Gn, G), np.where(up, f[:, l] * An, A)
        EG = np.where(up, f[:, l] * En + KAPPA * A, EG)
    out |= {"dgate": (dz, bz), "dvalue": (dv, bv), "dh0": (G, EG)}
    if o is not None:
        # silu' = s (1 + o (1 - s)) may cancel: its terms' absolute values
        mag = sg * (1.0 + np.abs(o) * sigmoid(-o))
        out["dout_gate"] = (dy * hs * ds, np.abs(dy) * (np.abs(ds) * Es + 3 * KAPPA * mag * Hs))
    return out


def norm(x, res, w, eps):
    """(r, y, bound of y before its rounding): the root of a sum of C squares is
    off by at most (C / 2 + 4) 2^-24, whatever the order of the sum; fp32 adds a few
    units for the products."""
    r = x if res is None else x + res
    C = r.shape[-1]
    y = r / np.sqrt(np.mean(r * r, axis=-1, keepdims=True) + eps) * w
    # the sum x + res itself is rounded to fp32
    return r, y, np.abs(y) * (C / 2 + 12) * U["f32"]


def norm_gradients(dy, r, w, dr, eps):
    C = r.shape[-1]
    rstd = 1.0 / np.sqrt(np.mean(r * r, axis=-1, keepdims=True) + eps)
    g = dy * w
    m = np.mean(g * r, axis=-1, keepdims=True) * rstd * rstd
    dx = rstd * (g - r * m) + (0.0 if dr is None else dr)
    k = (C + 24) * U["f32"]
    mabs = np.mean(np.abs(g * r), axis=-1, keepdims=True) * rstd * rstd
    bx = rstd * (np.abs(g) + 3 * np.abs(r) * mabs) * k + (0.0 if dr is None else np.abs(dr) * 2 * U["f32"])
    rows = int(np.prod(r.shape[:-1]))
    flat = (dy * r * rstd).reshape(-1, C)
    bw = np.abs(flat).sum(0) * (rows + C / 2 + 16) * U["f32"]
    return dx, bx, flat.sum(0), bw


def assert_close(got, ref, bound, dtype, what):
    """got is the rounding to dtype of a value within bound of ref."""
    got = np.asarray(got, dtype=np.float64)
    allowed = bound + U[dtype] * (np.abs(ref) + bound) + TINY[dtype]
    off = np.abs(got - ref)
    bad = ~(off <= allowed)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(off / allowed)), np.argwhere(bad)[:4].tolist())
