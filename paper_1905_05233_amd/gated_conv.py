"""A gated recurrent layer around the 1D convolution, as an example of the
sequence operators together: training, reading a prompt, and single tokens.

    r = x + residual
    n = rms_norm(r)
    gate, value, out_gate = causal convolution of width 3 of n, C -> 3 C channels
    y = gated_scan(gate, value, out_gate)

The convolution is ``Plan.conv1d`` with one leading row of zeros, which makes it
look back only: the norm writes behind that row and the scan reads its three
inputs as slices of the convolution's rows, so nothing is copied between them.
For single tokens it is a product of the matrix w [3 C][3 C] with the last three
tokens' norms, in 4 bits with the norms in 8 (or 16).

    layer = GatedConv(512, dtype="bf16")
    y, r, state = layer.prompt(x)                 # x [N][L][C]
    w4 = layer.quantize(group=64)
    y, r = layer.step(token, state, w4)           # token [N][C], state updated in place
"""
import math

import torch

from . import sequence_ops as S
from .winograd import Plan, TORCH_DTYPES
from .workloads import F2_LINEAR


class State:
    """What a layer keeps of N sequences: the norms of the last three tokens
    [N][3][C] (the oldest first), in 8 bits with their scales or in the layer's
    dtype, and the recurrence's state h fp32 [N][C]."""

    def __init__(self, window, scales, h):
        self.window, self.scales, self.h = window, scales, h


def _live(lengths, L):
    """Which steps [N][L][1] are none of the padding."""
    return (torch.arange(L, device=lengths.device)[None] < lengths[:, None])[:, :, None]


class GatedConv:
    def __init__(self, C, dtype="bf16", moduli=F2_LINEAR, m=2, eps=1e-6, seed=0, device="cuda"):
        self.C, self.eps, self.tdt = C, eps, TORCH_DTYPES[dtype]
        self.plan = Plan(moduli, m=m, dtype=dtype)
        g = torch.Generator().manual_seed(seed)
        w = torch.randn((3 * C, 3, C), generator=g) / math.sqrt(3 * C)
        self.weight = w.to(self.tdt).to(device)                      # [3C][3][C], taps from the oldest token on
        self.norm_weight = torch.ones(C, dtype=self.tdt, device=device)

    def _forward(self, x, residual, lengths, h0, save):
        N, L, C = x.shape
        if lengths is not None:
            # the convolution's tiles of steps mix live ones with padding behind them, where
            # a product with zero would not remove NaN or infinities
            S._dense(lengths, "lengths", (N,), torch.int32, x.get_device())
            live = _live(lengths, L)
            x = torch.where(live, x, 0)
            residual = None if residual is None else torch.where(live, residual, 0)
        rows = x.new_empty((N, L + 1, C))
        rows[:, 0].zero_()
        n, r = S.rms_norm(x, self.norm_weight, residual=residual, eps=self.eps, y=rows[:, 1:])
        u = self.plan.conv1d(rows, self.weight)[:, :L]
        gate, value, out_gate = u.split(C, dim=2)
        out = S.gated_scan(gate, value, out_gate, h0=h0, lengths=lengths, save_states=save)
        return n, (x if r is None else r), (gate, value, out_gate), out

    def forward(self, x, residual=None, lengths=None):
        """y [N][L][C] and r, which the next layer takes as its residual, and what
        ``backward`` needs.  lengths int32 [N]: steps from there on are padding; nothing
        there is used, and y and r are 0."""
        n, r, gates, (y, _, states) = self._forward(x, residual, lengths, None, True)
        return y, r, (n, r, gates, states, lengths)

    def backward(self, dy, saved, dr=None):
        """Gradients from dy (and dr, what reaches r from later layers): (dx, of x and
        of the residual, 0 at padding; dweight fp32 [3C][3][C]; dnorm_weight fp32 [C])."""
        n, r, (gate, value, out_gate), states, lengths = saved
        N, L, C = dy.shape
        # the convolution's gradient by its input is a convolution with the taps in
        # reverse, looking ahead: the scan's gradients stand ahead of a row of zeros
        rows = dy.new_empty((N, L + 1, 3 * C))
        rows[:, L].zero_()
        du = rows[:, :L]
        S.gated_scan_backward(dy, gate, value, states, out_gate=out_gate, lengths=lengths, out=du.split(C, dim=2))
        flipped = self.weight.flip(1).permute(2, 1, 0).contiguous()   # [C][3][3C]
        dn = self.plan.conv1d(rows, flipped)[:, 1:]
        if lengths is not None:
            live = _live(lengths, L)
            dn = torch.where(live, dn, 0)
            dr = None if dr is None else torch.where(live, dr, 0)
        dx, dnorm = S.rms_norm_backward(dn, r, self.norm_weight, dr=dr, eps=self.eps)
        dweight = torch.zeros((3 * C, 3, C), dtype=torch.float32, device=dy.device)
        for j in range(3):   # tap j meets the token 2 - j steps back
            back = 2 - j
            if back >= L:
                continue
            a = du[:, back:].reshape(-1, 3 * C).float()
            dweight[:, j] = a.t().contiguous() @ n[:, :L - back].reshape(-1, C).float()
        return dx, dweight, dnorm

    def prompt(self, x, residual=None, eight_bit=True, group=64):
        """y and r as ``forward``, and the sequences' state behind the last token."""
        n, r, _, (y, h) = self._forward(x, residual, None, None, False)
        N, L, C = x.shape
        state = self.new_state(N, eight_bit, group, device=x.device)
        keep = min(3, L)
        if eight_bit:
            q, scales, _ = S.rms_norm_fp8(r[:, L - keep:], self.norm_weight, eps=self.eps, group=group)
            state.window.view(torch.uint8)[:, 3 - keep:] = q.view(torch.uint8)
            state.scales[:, 3 - keep:] = scales
        else:
            state.window[:, 3 - keep:] = n[:, L - keep:]
        state.h = h
        return y, r, state

    def new_state(self, N, eight_bit=True, group=64, device="cuda"):
        if eight_bit and self.C % group:
            raise ValueError("C must be a multiple of the group")
        dt = torch.float8_e4m3fn if eight_bit else self.tdt
        window = torch.zeros((N, 3, self.C), dtype=torch.float32, device=device).to(dt)
        scales = torch.ones((N, 3, self.C // group), dtype=torch.float32, device=device) if eight_bit else None
        return State(window, scales, torch.zeros((N, self.C), dtype=torch.float32, device=device))

    def quantize(self, group=64):
        """The convolution's weights in 4 bits, as the matrix of the last three tokens."""
        return S.W4Matrix.quantize(self.weight.view(3 * self.C, 3 * self.C), group)

    def _check_step(self, x, state, w4, residual):
        """What the calls of a step would refuse, before any of them changes the state."""
        dev, shape = S._first(x, "x", (2,)), state.h.shape
        S._rows(x, "x", shape, self.tdt, dev)
        if residual is not None:
            S._rows(residual, "residual", shape, self.tdt, dev)
        if (w4.rows, w4.cols) != (3 * self.C, 3 * self.C) or w4.tiles.get_device() != dev:
            raise ValueError("w4 must be the layer's matrix, on the GPU of the tokens")
        if state.scales is not None and state.scales.shape[2] * w4.group != self.C:
            raise ValueError("the state's scales must go by the groups of w4")

    def step(self, x, state, w4, residual=None):
        """One token x [N][C] of each sequence; the state is updated in its own memory,
        so that a captured step can be replayed."""
        self._check_step(x, state, w4, residual)
        N, C = x.shape
        if state.scales is not None:
            bits = state.window.view(torch.uint8)
            bits[:, :2] = bits[:, 1:].clone()
            _, scales, r = S.rms_norm_fp8(x, self.norm_weight, residual=residual, eps=self.eps, group=w4.group,
                                          y=state.window[:, 2])
            state.scales[:, :2] = state.scales[:, 1:].clone()
            state.scales[:, 2] = scales
            u = S.matvec_w4(state.window.view(N, 3 * C), w4, x_scales=state.scales.view(N, -1), dtype=self.tdt)
        else:
            state.window[:, :2] = state.window[:, 1:].clone()
            _, r = S.rms_norm(x, self.norm_weight, residual=residual, eps=self.eps, y=state.window[:, 2])
            u = S.matvec_w4(state.window.view(N, 3 * C), w4)
        gate, value, out_gate = u.split(C, dim=1)
        y, _ = S.gated_step(gate, value, state.h, out_gate=out_gate, h_new=state.h)
        return y, (x if r is None else r)
