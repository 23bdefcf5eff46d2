"""Python binding of the sequence operators (argument marshalling only; the work
runs in the gfx950 kernels of gated_scan.hip, rms_norm.hip and matvec_w4.hip):
what stands around ``Plan.conv1d`` in a sequence model.

  * ``gated_scan``, ``gated_scan_backward``, ``gated_step``: the recurrence
    h = f h_before + (1 - f) value with f = sigmoid(gate), y = h or h silu(out_gate);
  * ``rms_norm``, ``rms_norm_fp8``, ``rms_norm_backward``: the root-mean-square
    norm of rows with the residual's addition, into the storage type or 8 bits;
  * ``W4Matrix``, ``matvec_w4``: products with 4-bit weights with group scales.

Tensors are f32, f16 or bf16 on the current GPU.  Rows [N][L][C] may have any
strides as long as the channels are contiguous (slices of a projection's rows,
a buffer with a leading row); states, scales and weights are contiguous.  Calls
are asynchronous on ``stream`` or the current stream; work that another stream
has still to do on the inputs is the caller's to wait for.  Outputs must not overlap
inputs, unless said otherwise.

Autograd sees nothing of these calls: results carry no graph, also where inputs
require gradients.  Gradients come from the ``_backward`` calls (the 4-bit products have
none), from within a ``torch.autograd.Function`` where a graph is wanted.
"""
import ctypes
import struct

import torch

from . import _native as N
from .winograd import _raw_stream

SCAN_BLOCK = 32      # WG_SCAN_BLOCK
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_E4M3 = 3
_NO_ROWS = (0, 0, 0)
_DENSE = torch.contiguous_format
_pack_scan = struct.Struct("4q" + "Pqq" * 4 + "4PPq").pack
_pack_scan_backward = struct.Struct("4q" + "Pqq" * 7 + "4PPq").pack
_pack_step = struct.Struct("3q" + "Pqq" * 4 + "2P").pack
_pack_norm = struct.Struct("4q" + "Pqq" * 4 + "2Pd2q").pack
_pack_norm_backward = struct.Struct("4q" + "Pqq" * 4 + "2PdPq").pack
_pack_w4 = struct.Struct("2P3q").pack
_pack_matvec = struct.Struct("2P3q" + "3q" + "PqPqPq").pack
_SIZES_KEPT = 256
_sizes = {}


def _first(t, name, dims):
    """(dtype code, device index) of the tensor that the others are held against."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU device")
    if t.dim() not in dims:
        raise ValueError(f"{name} must have {' or '.join(map(str, dims))} dimensions, got {t.dim()}")
    dev = t.get_device()
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on GPU {dev}, the current one is {torch._C._cuda_getDevice()}")
    return dev


def _code(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    return code


def _check(t, name, shape, dtype, dev):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_cuda or t.get_device() != dev:
        raise ValueError(f"{name} must be on the GPU of the other tensors")


def _rows(t, name, shape, dtype, dev):
    """(address, stride_n, stride_l) of [N][L][C], or of [L][C] as one sequence."""
    try:
        s = t.stride()
        if t.dtype is dtype and t.shape == shape and t.get_device() == dev and (s[-1] == 1 or shape[-1] <= 1):
            return (t.data_ptr(), s[0], s[1]) if len(s) == 3 else (t.data_ptr(), 0, s[0])
    except AttributeError:
        pass
    _check(t, name, shape, dtype, dev)   # raises, or the strides are at fault
    raise ValueError(f"{name}: the channels of a row must be contiguous")


def _dense(t, name, shape, dtype, dev):
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _check(t, name, shape, dtype, dev)
    raise ValueError(f"{name} must be contiguous")


def _out(t, name, like, dtype, dev):
    """(tensor, its rows): t, or if it is None a new contiguous one of like's shape."""
    if t is not None:
        return t, _rows(t, name, like.shape, dtype, dev)
    # the quickest way that torch has (1.3 us; new_empty takes 1.8, and is checked again)
    t = torch.empty_like(like, dtype=dtype, memory_format=_DENSE)
    shape = like.shape
    if len(shape) == 3:
        return t, (t.data_ptr(), shape[1] * shape[2], shape[2])
    return t, (t.data_ptr(), 0, shape[1])


def _new_f32(like, *shape):
    """A contiguous fp32 tensor of two or three dimensions on like's GPU."""
    strides = (shape[1], 1) if len(shape) == 2 else (shape[1] * shape[2], shape[2], 1)
    return torch.empty_strided(shape, strides, dtype=torch.float32, device=like.device)


def _size(query, dev, *args):
    """Bytes of workspace on the current device, dev, asked of the library once for given
    sizes: they go by the device's compute units too."""
    key = (query, dev, args)
    need = _sizes.get(key)
    if need is None:
        out = ctypes.c_size_t()
        N.check(getattr(N.lib(), query)(*args, ctypes.byref(out)))
        need = out.value
        if len(_sizes) >= _SIZES_KEPT:
            _sizes.clear()
        _sizes[key] = need
    return need


def _workspace(need, like):
    return torch.empty_strided((need,), (1,), dtype=torch.uint8, device=like.device) if need else None


def _tensors(values):
    for v in values:
        if isinstance(v, torch.Tensor):
            yield v
        elif isinstance(v, W4Matrix):
            yield from (v.tiles, v.scales)
        elif isinstance(v, (tuple, list)):
            yield from _tensors(v)


def _on(stream, call, *args):
    """call(*args) with ``stream`` as the current one.  What is allocated within belongs
    to that stream, so that no other stream's work is still to be done on it; the
    caching allocator is told which other tensors the stream uses, and that the
    caller's stream uses the results."""
    caller = torch.cuda.current_stream()
    if stream == caller:
        return call(*args)
    with torch.cuda.stream(stream):
        out = call(*args)
    for t in _tensors(args):
        t.record_stream(stream)
    for t in _tensors((out,)):
        t.record_stream(caller)
    return out


def gated_scan(gate, value, out_gate=None, h0=None, lengths=None, y=None, save_states=False, stream=None):
    """The recurrence over sequences: gate, value and out_gate [N][L][C] (one
    dtype), h0 fp32 [N][C] (zeros if absent), lengths int32 [N] (steps from there on
    are padding: y is 0 and the state stays).  Returns (y, h_last), h_last fp32
    [N][C] the last state; with ``save_states`` also the fp32 states ahead of every
    SCAN_BLOCK steps, for ``gated_scan_backward``."""
    if stream is not None:
        return _on(stream, gated_scan, gate, value, out_gate, h0, lengths, y, save_states)
    dev = _first(gate, "gate", (3,))
    dt, shape = gate.dtype, gate.shape
    code = _code(gate, "gate")
    Nn, L, C = shape
    g = _rows(gate, "gate", shape, dt, dev)
    v = _rows(value, "value", shape, dt, dev)
    o = _NO_ROWS if out_gate is None else _rows(out_gate, "out_gate", shape, dt, dev)
    y, yr = _out(y, "y", gate, dt, dev)
    h0p = 0 if h0 is None else _dense(h0, "h0", (Nn, C), torch.float32, dev)
    lp = 0 if lengths is None else _dense(lengths, "lengths", (Nn,), torch.int32, dev)
    h_last = _new_f32(gate, Nn, C)
    states = None
    if save_states:
        states = _new_f32(gate, Nn, -(-L // SCAN_BLOCK), C)
    if Nn == 0:   # the library takes one sequence and more
        return (y, h_last, states) if save_states else (y, h_last)
    need = _size("winograd_gated_scan_workspace", dev, code, Nn, L, C, 0)
    ws = _workspace(need, gate)
    st = N.lib().winograd_gated_scan(
        _pack_scan(code, Nn, L, C, *g, *v, *o, *yr, h0p, lp, h_last.data_ptr(),
                   0 if states is None else states.data_ptr(), 0 if ws is None else ws.data_ptr(), need),
        _raw_stream(None))
    if st != N.WG_OK:
        N.check(st)
    return (y, h_last, states) if save_states else (y, h_last)


def gated_scan_backward(dy, gate, value, states, out_gate=None, dh_last=None, lengths=None, out=None, stream=None):
    """Gradients of ``gated_scan`` from dy [N][L][C] and dh_last (fp32 [N][C], zeros
    if absent); gate, value, out_gate and lengths as in the forward call, states as
    it kept them.  Returns (dgate, dvalue, dout_gate, dh0), dout_gate None without
    out_gate.  ``out``: tensors [N][L][C] for the first two or three, as slices of
    the gradient of one projection."""
    if stream is not None:
        return _on(stream, gated_scan_backward, dy, gate, value, states, out_gate, dh_last, lengths, out)
    dev = _first(gate, "gate", (3,))
    dt, shape = gate.dtype, gate.shape
    code = _code(gate, "gate")
    Nn, L, C = shape
    d = _rows(dy, "dy", shape, dt, dev)
    g = _rows(gate, "gate", shape, dt, dev)
    v = _rows(value, "value", shape, dt, dev)
    o = _NO_ROWS if out_gate is None else _rows(out_gate, "out_gate", shape, dt, dev)
    sp = _dense(states, "states", (Nn, -(-L // SCAN_BLOCK), C), torch.float32, dev)
    dhp = 0 if dh_last is None else _dense(dh_last, "dh_last", (Nn, C), torch.float32, dev)
    lp = 0 if lengths is None else _dense(lengths, "lengths", (Nn,), torch.int32, dev)
    if out is None:
        out = (None, None) if out_gate is None else (None, None, None)
    elif len(out) != (2 if out_gate is None else 3):
        raise ValueError("out must hold dgate, dvalue and, with out_gate, dout_gate")
    dgate, zr = _out(out[0], "dgate", gate, dt, dev)
    dvalue, vr = _out(out[1], "dvalue", gate, dt, dev)
    dout_gate, outr = (None, _NO_ROWS) if out_gate is None else _out(out[2], "dout_gate", gate, dt, dev)
    dh0 = _new_f32(gate, Nn, C)
    if Nn == 0:
        return dgate, dvalue, dout_gate, dh0
    need = _size("winograd_gated_scan_workspace", dev, code, Nn, L, C, 1)
    ws = _workspace(need, gate)
    st = N.lib().winograd_gated_scan_backward(
        _pack_scan_backward(code, Nn, L, C, *d, *g, *v, *o, *zr, *vr, *outr, sp, dhp, lp, dh0.data_ptr(),
                            0 if ws is None else ws.data_ptr(), need), _raw_stream(None))
    if st != N.WG_OK:
        N.check(st)
    return dgate, dvalue, dout_gate, dh0


def gated_step(gate, value, h, out_gate=None, h_new=None, y=None, stream=None):
    """One step for N sequences: gate, value and out_gate [N][C], h fp32 [N][C] the
    states.  Returns (y, h_new); ``h_new=h`` updates the states in place."""
    if stream is not None:
        return _on(stream, gated_step, gate, value, h, out_gate, h_new, y)
    dev = _first(gate, "gate", (2,))
    dt, shape = gate.dtype, gate.shape
    code = _code(gate, "gate")
    Nn, C = shape
    # [N][C]: N sequences of one step
    g = _rows(gate, "gate", shape, dt, dev)
    v = _rows(value, "value", shape, dt, dev)
    o = _NO_ROWS if out_gate is None else _rows(out_gate, "out_gate", shape, dt, dev)
    hp = _dense(h, "h", shape, torch.float32, dev)
    y, yr = _out(y, "y", gate, dt, dev)
    if h_new is None:
        h_new = torch.empty_like(h)
        hnp = h_new.data_ptr()
    else:
        hnp = _dense(h_new, "h_new", shape, torch.float32, dev)
    st = N.lib().winograd_gated_step(
        _pack_step(code, Nn, C, g[0], g[2], 0, v[0], v[2], 0, o[0], o[2], 0, yr[0], yr[2], 0, hp, hnp),
        _raw_stream(None))
    if st != N.WG_OK:
        N.check(st)
    return y, h_new


def _norm(x, weight, residual, eps, out, r, quant, group):
    dev = _first(x, "x", (2, 3))
    dt, shape = x.dtype, x.shape
    code = _code(x, "x")
    C = shape[-1]
    Nn, L = (1, shape[0]) if len(shape) == 2 else (shape[0], shape[1])
    xr = _rows(x, "x", shape, dt, dev)
    rr = sr = _NO_ROWS
    if residual is not None:
        rr = _rows(residual, "residual", shape, dt, dev)
        r, sr = _out(r, "r", x, dt, dev)
    elif r is not None:
        raise ValueError("r is the sum with the residual: there is none")
    wp = _dense(weight, "weight", (C,), dt, dev)
    odt = torch.float8_e4m3fn if quant else dt
    out, yr = _out(out, "y", x, odt, dev)
    scales = None
    if quant:
        scales = _new_f32(x, *shape[:-1], -(-C // group) if group > 0 else 1)
    st = N.lib().winograd_rms_norm(
        _pack_norm(code, Nn, L, C, *xr, *rr, *sr, *yr, wp, 0 if scales is None else scales.data_ptr(), eps,
                   _E4M3 if quant else code, group), _raw_stream(None))
    if st != N.WG_OK:
        N.check(st)
    return out, scales, r


def rms_norm(x, weight, residual=None, eps=1e-6, y=None, r=None, stream=None):
    """The norm of the rows of x + residual ([N][L][C] or [L][C]), times weight [C].
    Returns (y, r): r is the sum in the storage type (None without a residual); it
    may be given, and be x or the residual itself."""
    if stream is not None:
        return _on(stream, rms_norm, x, weight, residual, eps, y, r)
    out, _, r = _norm(x, weight, residual, eps, y, r, False, 0)
    return out, r


def rms_norm_fp8(x, weight, residual=None, eps=1e-6, group=0, y=None, r=None, stream=None):
    """``rms_norm`` into 8 bits.  Returns (q, scales, r): q float8_e4m3fn shaped as
    x, scales fp32 [..., G], one for every ``group`` channels (32, 64 or 128) or for
    the row (0); q times its scale is the norm's output."""
    if stream is not None:
        return _on(stream, rms_norm_fp8, x, weight, residual, eps, group, y, r)
    return _norm(x, weight, residual, eps, y, r, True, group)


def rms_norm_backward(dy, r, weight, dr=None, eps=1e-6, dx=None, stream=None):
    """Gradients of ``rms_norm`` at the rows r that were normalised, with dr the
    gradient that reaches r from elsewhere.  Returns (dx, dweight): dx is the
    gradient of r, and so of x and of the residual; dweight is fp32 [C].  dx may be
    given, and be dy or dr itself."""
    if stream is not None:
        return _on(stream, rms_norm_backward, dy, r, weight, dr, eps, dx)
    dev = _first(r, "r", (2, 3))
    dt, shape = r.dtype, r.shape
    code = _code(r, "r")
    C = shape[-1]
    Nn, L = (1, shape[0]) if len(shape) == 2 else (shape[0], shape[1])
    d = _rows(dy, "dy", shape, dt, dev)
    rr = _rows(r, "r", shape, dt, dev)
    dd = _NO_ROWS if dr is None else _rows(dr, "dr", shape, dt, dev)
    wp = _dense(weight, "weight", (C,), dt, dev)
    dx, xr = _out(dx, "dx", r, dt, dev)
    dweight = torch.empty_like(weight, dtype=torch.float32)
    need = _size("winograd_rms_norm_workspace", dev, code, Nn, L, C)
    ws = _workspace(need, r)
    st = N.lib().winograd_rms_norm_backward(
        _pack_norm_backward(code, Nn, L, C, *d, *rr, *dd, *xr, wp, dweight.data_ptr(), eps,
                            0 if ws is None else ws.data_ptr(), need), _raw_stream(None))
    if st != N.WG_OK:
        N.check(st)
    return dx, dweight


class W4Matrix:
    """A matrix [rows][cols] in 4 bits with a bf16 scale for every ``group`` (32, 64
    or 128) columns of a row: tiles int32 [ceil(rows/16)][ceil(cols/128)][4][16][4]
    and scales bf16 [ceil(rows/16)][ceil(cols/group)][16] in the library's layout.
    Its attributes are what it was made of and cannot be set."""
    __slots__ = ("_tiles", "_scales", "_rows", "_cols", "_group", "_dev", "_packed")
    tiles = property(lambda self: self._tiles)
    scales = property(lambda self: self._scales)
    rows = property(lambda self: self._rows)
    cols = property(lambda self: self._cols)
    group = property(lambda self: self._group)

    def __init__(self, tiles, scales, rows, cols, group):
        if group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        if rows < 1 or cols < 1:
            raise ValueError("rows and cols must be positive")
        dev = _first(tiles, "tiles", (5,))
        self._tiles, self._scales, self._rows, self._cols, self._group = tiles, scales, rows, cols, group
        self._check(dev)

    def _check(self, dev):
        rt = -(-self._rows // 16)
        tp = _dense(self._tiles, "tiles", (rt, -(-self._cols // 128), 4, 16, 4), torch.int32, dev)
        sp = _dense(self._scales, "scales", (rt, -(-self._cols // self._group), 16), torch.bfloat16, dev)
        self._dev, self._packed = dev, (tp, sp, self._rows, self._cols, self._group)

    def _words(self, dev):
        """The argument's words for a call on dev.  Tensors that were given other memory
        since they were last checked are checked again."""
        packed = self._packed
        if self._tiles.data_ptr() != packed[0] or self._scales.data_ptr() != packed[1]:
            self._check(dev)
        elif self._dev != dev:
            raise ValueError("w must be on the GPU of the other tensors")
        return self._packed

    @classmethod
    def _empty(cls, rows, cols, group, device):
        if group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        rt = -(-rows // 16)
        return cls(torch.empty((rt, -(-cols // 128), 4, 16, 4), dtype=torch.int32, device=device),
                   torch.empty((rt, -(-cols // group), 16), dtype=torch.bfloat16, device=device), rows, cols, group)

    @classmethod
    def quantize(cls, m, group=128, stream=None):
        """m [rows][cols] rounded to the nearest multiples -7 .. 7 of each group's
        scale, bf16(max |m| / 7).  A group with NaN or an infinity becomes NaN."""
        if stream is not None:
            return _on(stream, cls.quantize, m, group)
        dev = _first(m, "m", (2,))
        mp, _, ld = _rows(m, "m", m.shape, m.dtype, dev)
        code = _code(m, "m")
        w = cls._empty(m.shape[0], m.shape[1], group, m.device)
        N.check(N.lib().winograd_quantize_w4(_pack_w4(*w._words(dev)), code, mp, ld, _raw_stream(None)))
        return w

    @classmethod
    def from_nibbles(cls, nibbles, scales, cols, stream=None):
        """From codes 0 .. 15 (value code - 8) as checkpoints hold them: uint8
        [rows][ceil(cols/2)], the even column in the lower half, and scales bf16
        [rows][ceil(cols/group)]; the group follows from their number."""
        if stream is not None:
            return _on(stream, cls.from_nibbles, nibbles, scales, cols)
        dev = _first(nibbles, "nibbles", (2,))
        rows = nibbles.shape[0]
        np_ = _dense(nibbles, "nibbles", (rows, -(-cols // 2)), torch.uint8, dev)
        if not isinstance(scales, torch.Tensor) or scales.dim() != 2:
            raise ValueError("scales must be [rows][groups]")
        fits = [g for g in (128, 64, 32) if -(-cols // g) == scales.shape[1]]
        if not fits:
            raise ValueError("scales must be [rows][ceil(cols/group)] for a group of 32, 64 or 128")
        sp = _dense(scales, "scales", (rows, scales.shape[1]), torch.bfloat16, dev)
        w = cls._empty(rows, cols, fits[0], nibbles.device)
        N.check(N.lib().winograd_pack_w4(_pack_w4(*w._words(dev)), np_, sp, _raw_stream(None)))
        return w

    def dequantize(self, dtype=torch.bfloat16, stream=None):
        """The matrix [rows][cols] that the codes and scales stand for."""
        if stream is not None:
            return _on(stream, W4Matrix.dequantize, self, dtype)
        m = torch.empty((self.rows, self.cols), dtype=dtype, device=self.tiles.device)
        code = _code(m, "m")
        dev = _first(self.tiles, "tiles", (5,))
        N.check(N.lib().winograd_dequantize_w4(_pack_w4(*self._words(dev)), code, m.data_ptr(), self.cols,
                                               _raw_stream(None)))
        return m


def matvec_w4(x, w, x_scales=None, y=None, dtype=None, stream=None):
    """y [M][rows] = x [M][cols] times the transpose of the ``W4Matrix`` w, for a few
    rows x in f32, f16, bf16 or, with x_scales fp32 [M][1] or [M][groups of w],
    float8_e4m3fn.  y has ``dtype``, by default x's (bf16 for 8 bits)."""
    if stream is not None:
        return _on(stream, matvec_w4, x, w, x_scales, y, dtype)
    dev = _first(x, "x", (2,))
    xdt = x.dtype
    x8 = xdt == torch.float8_e4m3fn
    M, rows = x.shape[0], w._rows
    xp, _, ldx = _rows(x, "x", (M, w._cols), xdt, dev)
    xcode = _E4M3 if x8 else _code(x, "x")
    words = w._words(dev)
    sp, groups = 0, 0
    if x8:
        if not isinstance(x_scales, torch.Tensor) or x_scales.dim() != 2:
            raise ValueError("rows in 8 bits need x_scales [M][1] or [M][groups]")
        groups = x_scales.shape[1]
        sp = _dense(x_scales, "x_scales", (M, groups), torch.float32, dev)
    elif x_scales is not None:
        raise ValueError("x_scales are for rows in 8 bits")
    if y is None:
        if dtype is None:
            dtype = torch.bfloat16 if x8 else xdt
        y = torch.empty_strided((M, rows), (rows, 1), dtype=dtype, device=x.device)
        yp, ldy = y.data_ptr(), rows
    else:
        if dtype is not None and dtype != y.dtype:
            raise TypeError("dtype is that of y")
        yp, _, ldy = _rows(y, "y", (M, rows), y.dtype, dev)
    st = N.lib().winograd_matvec_w4(
        _pack_matvec(*words, M, xcode, _code(y, "y"), xp, ldx, sp, groups, yp, ldy), _raw_stream(None))
    if st != N.WG_OK:
        N.check(st)
    return y
