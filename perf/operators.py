"""The operators that a sequence model built around the 1D convolution needs, and the cases by which their speed is judged.

  * the gated linear recurrence over [N][L][C] with its backward pass, and its form for single tokens;
  * the root-mean-square norm of rows with the residual's addition, its output in the storage type or in 8 bits with
    scales, and its backward pass;
  * products of a few rows with a matrix of 4-bit weights with group scales: a convolution of width three for a new token,
    the classifier behind a VGG-16 stack for one image.

``run`` with ``own`` false computes them in elementary torch operations in 32 bits; with ``own`` true it calls
``paper_1905_05233_amd.sequence_ops``.  ``exact`` is their definition in 64 bits.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FP8_MAX = 448.0        # largest value of e4m3
FP8_LEAST = 2.0 ** -100  # absolute maxima below this count as this
EPS = 1e-6


def listed():
    return [
        # serving, one new token for each of sixteen sequences: a call's latency
        {"name": "step_bf16", "op": "step", "dtype": "bf16", "N": 16, "C": 512, "out_gate": True, "fused": True},
        # serving, the prompt of one sequence: few rows, a long axis, gates as slices of one projection, a state carried in
        {"name": "prefill_long_bf16", "op": "scan", "dtype": "bf16", "N": 1, "L": 16381, "C": 512, "out_gate": True,
         "h0": True, "lengths": False, "fused": True},
        # serving, prompts of different lengths in one batch, sizes that fill no vector
        {"name": "scan_ragged_f16", "op": "scan", "dtype": "f16", "N": 13, "L": 1021, "C": 75, "out_gate": False,
         "h0": True, "lengths": True, "fused": False},
        # training, a batch of long sequences: outputs, then gradients
        {"name": "scan_train_bf16", "op": "scan_train", "dtype": "bf16", "N": 16, "L": 4096, "C": 512, "out_gate": True,
         "h0": False, "lengths": False, "fused": False},
        # training in 32 bits, as an error study does: a small batch with an initial state and padding
        {"name": "scan_train_f32", "op": "scan_train", "dtype": "f32", "N": 4, "L": 1000, "C": 96, "out_gate": True,
         "h0": True, "lengths": True, "fused": False},
        # serving, the norm ahead of 4-bit products for single tokens
        {"name": "norm_fp8_token_bf16", "op": "norm", "dtype": "bf16", "rows": 16, "C": 512, "residual": True, "fp8": True,
         "group": 0},
        # a whole batch through the norm into 8 bits, scales by groups
        {"name": "norm_fp8_bf16", "op": "norm", "dtype": "bf16", "rows": 65536, "C": 512, "residual": True, "fp8": True,
         "group": 128},
        # rows that are no power of two
        {"name": "norm_f16", "op": "norm", "dtype": "f16", "rows": 3001, "C": 1000, "residual": True, "fp8": False, "group": 0},
        # training, the norm's gradients over the same batch as the scan's
        {"name": "norm_grad_bf16", "op": "norm_grad", "dtype": "bf16", "rows": 65536, "C": 512, "residual": True},
        # the widest layer behind a VGG-16 stack, one image: 7 x 7 x 512 activations to 4096
        {"name": "matvec_head_bf16", "op": "matvec", "dtype": "bf16", "M": 1, "K": 25088, "R": 4096, "group": 128},
        # its last layer for a few images, in 32 bits
        {"name": "matvec_classes_f32", "op": "matvec", "dtype": "f32", "M": 5, "K": 4096, "R": 1000, "group": 64},
        # a convolution of width three, 512 channels to three times 512, for one new token of sixteen sequences, from 8 bits
        {"name": "matvec_window_fp8", "op": "matvec", "dtype": "fp8", "M": 16, "K": 1536, "R": 1536, "group": 32},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def channels(lo, hi):
        return 2 ** rng.randint(math.ceil(math.log2(lo)), int(math.log2(hi))) if rng.random() < 0.5 else log(lo, hi)

    while True:
        op = rng.choices(("step", "scan", "scan_train", "norm", "norm_grad", "matvec"), (1, 3, 3, 3, 2, 4))[0]
        case = {"op": op, "dtype": rng.choice(("f32", "f16", "bf16", "bf16"))}
        if op == "step":
            return {**case, "N": log(1, 256), "C": channels(32, 4096), "out_gate": rng.random() < 0.6,
                    "fused": rng.random() < 0.5}
        if op in ("scan", "scan_train"):
            case |= {"N": log(1, 64), "L": log(1, 32768), "C": channels(24, 2048), "out_gate": rng.random() < 0.6,
                     "h0": rng.random() < 0.5, "lengths": rng.random() < 0.4, "fused": rng.random() < 0.4}
            size = case["N"] * case["L"] * case["C"]
        elif op == "norm":
            case |= {"rows": log(1, 131072), "C": channels(24, 8192), "residual": rng.random() < 0.7,
                     "fp8": rng.random() < 0.5}
            case["group"] = rng.choice((0, 0, 32, 64, 128)) if case["fp8"] else 0
            size = case["rows"] * case["C"]
        elif op == "norm_grad":
            case |= {"rows": log(1, 131072), "C": channels(24, 8192), "residual": rng.random() < 0.7}
            size = case["rows"] * case["C"]
        else:
            case |= {"dtype": rng.choice(("f32", "f16", "bf16", "bf16", "fp8")), "M": log(1, 16), "K": log(64, 25088),
                     "R": log(64, 8192), "group": rng.choice((32, 64, 128))}
            if rng.random() < 0.7:
                case["K"] -= case["K"] % 64
            if case["K"] * case["R"] <= 25088 * 4096:
                return case
            continue
        if size <= 2 ** 25 // (2 if case["dtype"] == "f32" else 1):
            return case


# ---------------------------------------------------------------- inputs

def _generator(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 41)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _gates(case, g, shape):
    """Pre-activations of the forget gate (memories from a few steps to some hundreds), values and output gates."""
    parts = [_randn(g, *shape) * 1.5 + 2.0, _randn(g, *shape)] + ([_randn(g, *shape)] if case["out_gate"] else [])
    parts = [p.to(TORCH[case["dtype"]]) for p in parts]
    if case["fused"]:  # slices of the rows of one projection
        parts = list(torch.cat(parts, dim=-1).split(shape[-1], dim=-1))
    return parts + [None] * (3 - len(parts))


def _tiles(codes, rows, cols):
    """Codes 0 .. 15 of a matrix [rows][cols] in the order in which the products read them: tiles of 16 rows and 128
    columns; of a tile, for each quarter q, row, and s = 0 .. 3 the eight codes of columns 32 s + 8 q + j in a 32-bit word,
    the even j in its lower half and the odd ones in its upper half, rotated left by 3 bits.  Padding is code 8, a zero."""
    rt, kt = -(-rows // 16), -(-cols // 128)
    full = torch.full((rt * 16, kt * 128), 8, dtype=torch.int32, device=codes.device)
    full[:rows, :cols] = codes
    c = full.view(rt, 16, kt, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)  # [row tile][column tile][q][row][s][j]
    at = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], dtype=torch.int64, device=codes.device)
    w = (c.to(torch.int64) << at).sum(-1)
    w = ((w << 3) | (w >> 29)) & 0xFFFFFFFF
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32).contiguous()


def prepare(case, seed):
    g = _generator(case, seed)
    op, s = case["op"], {"case": case}
    if op == "step":
        s["gate"], s["value"], s["out_gate"] = _gates(case, g, (case["N"], case["C"]))
        s["h"] = _randn(g, case["N"], case["C"])
    elif op in ("scan", "scan_train"):
        N, L, C = case["N"], case["L"], case["C"]
        s["gate"], s["value"], s["out_gate"] = _gates(case, g, (N, L, C))
        s["h0"] = _randn(g, N, C) if case["h0"] else None
        s["lengths"] = None
        if case["lengths"]:  # one of them empty, one full
            n = torch.randint(0, L + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
            n[-1], n[0] = 0, L
            s["lengths"] = n
        if op == "scan_train":
            s["dy"] = _randn(g, N, L, C).to(TORCH[case["dtype"]])
            s["dh"] = _randn(g, N, C) if case["h0"] else None
    elif op in ("norm", "norm_grad"):
        R, C, t = case["rows"], case["C"], TORCH[case["dtype"]]
        size = torch.exp(_randn(g, R, 1))  # rows of different magnitude
        s["x"] = (_randn(g, R, C) * size).to(t)
        s["weight"] = (1.0 + 0.1 * _randn(g, C)).to(t)
        s["other"] = (_randn(g, R, C) * (size if op == "norm" else 1.0)).to(t) if case["residual"] else None
        if op == "norm_grad":
            s["dy"] = _randn(g, R, C).to(t)
    else:
        M, K, R, group = case["M"], case["K"], case["R"], case["group"]
        codes = (_randn(g, R, K) * 2.5).round_().clamp_(-8, 7).to(torch.int32) + 8
        groups = -(-K // group)
        scales = (torch.rand((R, groups), generator=g, device="cuda") + 0.5).mul_(0.02).to(torch.bfloat16)
        even = torch.cat((codes, torch.full((R, 1), 8, dtype=torch.int32, device="cuda")), 1) if K % 2 else codes
        s["nibbles"] = (even[:, 0::2] | (even[:, 1::2] << 4)).to(torch.uint8)  # as a checkpoint holds them
        s["scales"] = scales
        s["tiles"] = _tiles(codes, R, K)
        rt = -(-R // 16)
        padded = torch.zeros((rt * 16, groups), dtype=torch.bfloat16, device="cuda")
        padded[:R] = scales
        s["tile_scales"] = padded.view(rt, 16, groups).transpose(1, 2).contiguous()
        x = _randn(g, M, K)
        s["x_scales"] = None
        if case["dtype"] == "fp8":  # a scale for each row, as the norm gives them
            top = x.abs().amax(1, keepdim=True) / FP8_MAX
            s["x_scales"] = top
            x = (x / top).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)
        else:
            x = x.to(TORCH[case["dtype"]])
        s["x"] = x
    return s


# ---------------------------------------------------------------- plain forms, in 32 bits

def _linear_scan(f, b):
    """h_t = f_t h_(t-1) + b_t along dimension 1 from h = 0: pairs of steps are joined, the half as long sequence is
    solved, and the steps between are filled in."""
    T = f.shape[1]
    if T <= 1:
        return b
    half = T // 2
    f0, f1, b0, b1 = f[:, 0:2 * half:2], f[:, 1::2], b[:, 0:2 * half:2], b[:, 1::2]
    odd = _linear_scan(f1 * f0, f1 * b0 + b1)
    h = torch.empty_like(b)
    h[:, 1::2] = odd
    h[:, 0] = b[:, 0]
    h[:, 2::2] = f[:, 2::2] * odd[:, :(T - 1) // 2] + b[:, 2::2]
    return h


def _alive(s, L):
    if s["lengths"] is None:
        return None
    return (torch.arange(L, device="cuda")[None, :] < s["lengths"][:, None])[:, :, None]


def _plain_scan(s):
    """(states, f, i, value) in 32 bits; padding has f = 1, i = 0."""
    z, v = s["gate"].float(), s["value"].float()
    f, i = 1.0 / (1.0 + torch.exp(-z)), 1.0 / (1.0 + torch.exp(z))
    alive = _alive(s, z.shape[1])
    if alive is not None:
        f, i, v = torch.where(alive, f, 1.0), torch.where(alive, i, 0.0), torch.where(alive, v, 0.0)
    b = i * v
    if s["h0"] is not None:
        b[:, 0] += f[:, 0] * s["h0"]
    return _linear_scan(f, b), f, i, v


def _plain_outputs(s, h):
    y = h
    if s["out_gate"] is not None:
        o = s["out_gate"].float()
        y = h * (o / (1.0 + torch.exp(-o)))
    alive = _alive(s, h.shape[1])
    if alive is not None:
        y = torch.where(alive, y, 0.0)
    return {"y": y.to(s["gate"].dtype), "h_last": h[:, -1].contiguous()}


def _plain_gradients(s, h, f, i, v):
    dt, dy = s["gate"].dtype, s["dy"].float()
    alive = _alive(s, h.shape[1])
    if alive is not None:
        dy = torch.where(alive, dy, 0.0)
    do, g = None, dy
    if s["out_gate"] is not None:
        o = s["out_gate"].float()
        if alive is not None:
            o = torch.where(alive, o, 0.0)
        sig = 1.0 / (1.0 + torch.exp(-o))
        g = dy * (o * sig)
        do = (dy * h * (sig * (1.0 + o * (1.0 - sig)))).to(dt)
    if s["dh"] is not None:
        g = torch.cat((g[:, :-1], g[:, -1:] + s["dh"][:, None]), 1)
    later = torch.cat((f[:, 1:], torch.zeros_like(f[:, :1])), 1)
    G = _linear_scan(later.flip(1), g.flip(1)).flip(1)
    first = torch.zeros_like(h[:, :1]) if s["h0"] is None else s["h0"][:, None]
    before = torch.cat((first, h[:, :-1]), 1)
    return {"dgate": (f * i * (before - v) * G).to(dt), "dvalue": (i * G).to(dt), "dout_gate": do,
            "dh0": f[:, 0] * G[:, 0]}


def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    r = x if s["other"] is None else x + s["other"].float()
    y = r * (1.0 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS)) * s["weight"].float()
    out = {"r": r.to(s["x"].dtype) if s["other"] is not None else None}
    if not case["fp8"]:
        return {**out, "y": y.to(s["x"].dtype)}
    C = y.shape[1]
    group = case["group"] or C
    groups = -(-C // group)
    full = torch.nn.functional.pad(y, (0, groups * group - C)).view(-1, groups, group)
    scales = full.abs().amax(2, keepdim=True).clamp(min=FP8_LEAST) / FP8_MAX
    q = (full / scales).clamp(-FP8_MAX, FP8_MAX).view(-1, groups * group)[:, :C].to(torch.float8_e4m3fn)
    return {**out, "q": q, "scales": scales[:, :, 0]}


def _plain_norm_gradients(s):
    r, dy, w = s["x"].float(), s["dy"].float(), s["weight"].float()
    rstd = 1.0 / torch.sqrt((r * r).mean(1, keepdim=True) + EPS)
    g = dy * w
    dx = rstd * (g - r * (rstd * rstd * (g * r).mean(1, keepdim=True)))
    if s["other"] is not None:
        dx = dx + s["other"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * (r * rstd)).sum(0)}


def _plain_matvec(s):
    case = s["case"]
    K, group = case["K"], case["group"]
    b = s["nibbles"]
    w = torch.stack((b & 15, b >> 4), 2).view(b.shape[0], -1)[:, :K].float() - 8.0
    w = w * s["scales"].float().repeat_interleave(group, 1)[:, :K]
    x = s["x"].float()
    if s["x_scales"] is not None:
        x = x * s["x_scales"]
    y = x @ w.t()
    return y.to(torch.bfloat16 if case["dtype"] == "fp8" else s["x"].dtype)


def _plain(s):
    op = s["case"]["op"]
    if op == "step":
        z, v = s["gate"].float(), s["value"].float()
        h = s["h"] / (1.0 + torch.exp(-z)) + v / (1.0 + torch.exp(z))
        y = h
        if s["out_gate"] is not None:
            o = s["out_gate"].float()
            y = h * (o / (1.0 + torch.exp(-o)))
        return {"y": y.to(s["gate"].dtype), "h": h}
    if op == "scan":
        return _plain_outputs(s, _plain_scan(s)[0])
    if op == "scan_train":
        h, f, i, v = _plain_scan(s)
        return {**_plain_outputs(s, h), **_plain_gradients(s, h, f, i, v)}
    if op == "norm":
        return _plain_norm(s)
    if op == "norm_grad":
        return _plain_norm_gradients(s)
    return _plain_matvec(s)


# ---------------------------------------------------------------- the framework's operators

def _framework(s):
    from paper_1905_05233_amd import sequence_ops as S
    case = s["case"]
    op = case["op"]
    if op == "step":
        y, h = S.gated_step(s["gate"], s["value"], s["h"], out_gate=s["out_gate"])
        return {"y": y, "h": h}
    if op == "scan":
        y, h_last = S.gated_scan(s["gate"], s["value"], out_gate=s["out_gate"], h0=s["h0"], lengths=s["lengths"])
        return {"y": y, "h_last": h_last}
    if op == "scan_train":
        y, h_last, states = S.gated_scan(s["gate"], s["value"], out_gate=s["out_gate"], h0=s["h0"],
                                         lengths=s["lengths"], save_states=True)
        dgate, dvalue, dout_gate, dh0 = S.gated_scan_backward(s["dy"], s["gate"], s["value"], states,
                                                              out_gate=s["out_gate"], dh_last=s["dh"],
                                                              lengths=s["lengths"])
        return {"y": y, "h_last": h_last, "dgate": dgate, "dvalue": dvalue, "dout_gate": dout_gate, "dh0": dh0}
    if op == "norm":
        if case["fp8"]:
            q, scales, r = S.rms_norm_fp8(s["x"], s["weight"], residual=s["other"], eps=EPS, group=case["group"])
            return {"r": r, "q": q, "scales": scales}
        y, r = S.rms_norm(s["x"], s["weight"], residual=s["other"], eps=EPS)
        return {"r": r, "y": y}
    if op == "norm_grad":
        dx, dweight = S.rms_norm_backward(s["dy"], s["x"], s["weight"], dr=s["other"], eps=EPS)
        return {"dx": dx, "dweight": dweight}
    w = S.W4Matrix(s["tiles"], s["tile_scales"], case["R"], case["K"], case["group"])
    return S.matvec_w4(s["x"], w, x_scales=s["x_scales"])


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------- what cannot be done without

def work(case):
    op = case["op"]
    es = {"f32": 4, "f16": 2, "bf16": 2, "fp8": 1}[case["dtype"]]
    if op == "matvec":
        M, K, R, groups = case["M"], case["K"], case["R"], -(-case["K"] // case["group"])
        es_y = 2 if case["dtype"] == "fp8" else es
        return {"bytes": R * K / 2 + 2 * R * groups + es * M * K + es_y * M * R, "flops": 2.0 * M * R * K}
    if op in ("norm", "norm_grad"):
        n = case["rows"] * case["C"]
        if op == "norm_grad":
            return {"bytes": es * n * (4 if case["residual"] else 3) + (es + 4) * case["C"], "flops": 11.0 * n}
        b = es * n * (3 if case["residual"] else 1) + es * case["C"]  # x, and the residual's sum in and out
        if case["fp8"]:
            return {"bytes": b + n + 4 * case["rows"] * -(-case["C"] // (case["group"] or case["C"])), "flops": 8.0 * n}
        return {"bytes": b + es * n, "flops": 5.0 * n}
    gates = 3 if case["out_gate"] else 2
    n = case["N"] * case["C"]
    if op == "step":
        return {"bytes": es * n * (gates + 1) + 8 * n, "flops": 12.0 * n}
    ends = 4 * n * (2 if case["h0"] else 1)
    n *= case["L"]
    if op == "scan":
        return {"bytes": es * n * (gates + 1) + ends, "flops": 12.0 * n}
    # forward, then the gates and dy in and a gradient for each gate out
    return {"bytes": es * n * (gates + 1 + gates + 1 + gates) + 2 * ends, "flops": 40.0 * n}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "matvec":
        b = s["nibbles"].to(torch.int64)
        w = torch.empty((case["R"], 2 * b.shape[1]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (b % 16 - 8).double(), (b // 16 - 8).double()
        x = s["x"].double() if s["x_scales"] is None else s["x"].double() * s["x_scales"].double()
        y = torch.zeros((case["M"], case["R"]), dtype=torch.float64, device="cuda")
        for g in range(s["scales"].shape[1]):
            a, e = g * case["group"], min((g + 1) * case["group"], case["K"])
            y += (x[:, a:e] @ w[:, a:e].t().contiguous()) * s["scales"][:, g].double()
        return y
    if op == "norm":
        r = s["x"].double() + (0.0 if s["other"] is None else s["other"].double())
        y = r / torch.sqrt(r.square().sum(1, keepdim=True) / case["C"] + EPS) * s["weight"].double()
        out = {"r": None if s["other"] is None else r}
        if not case["fp8"]:
            return {**out, "y": y}
        group = case["group"] or case["C"]
        cut = y.split(group, dim=1)
        tops = [c.abs().amax(1, keepdim=True).clamp(min=FP8_LEAST) / FP8_MAX for c in cut]
        q = [(c / t).float().to(torch.float8_e4m3fn).double() for c, t in zip(cut, tops)]
        return {**out, "q": torch.cat(q, 1), "scales": torch.cat(tops, 1)}
    if op == "norm_grad":
        r, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
        unit = r / torch.sqrt(r.square().sum(1, keepdim=True) / case["C"] + EPS)
        dunit = dy * w
        # d unit / d r is (1 - unit unit^T / C) times the inverse root
        dx = (dunit - unit * (dunit * unit).sum(1, keepdim=True) / case["C"])
        dx = dx / torch.sqrt(r.square().sum(1, keepdim=True) / case["C"] + EPS)
        return {"dx": dx if s["other"] is None else dx + s["other"].double(), "dweight": (dy * unit).sum(0)}
    f = torch.sigmoid(s["gate"].double())
    i, v = torch.sigmoid(-s["gate"].double()), s["value"].double()
    silu = None if s["out_gate"] is None else s["out_gate"].double() * torch.sigmoid(s["out_gate"].double())
    if op == "step":
        h = f * s["h"].double() + i * v
        return {"y": h if silu is None else h * silu, "h": h}
    N, L, C = v.shape
    start = torch.zeros((N, C), dtype=torch.float64, device="cuda") if s["h0"] is None else s["h0"].double()
    ends = torch.full((N, 1), L, device="cuda") if s["lengths"] is None else s["lengths"][:, None].long()
    h, before, hs = start, [], []
    for t in range(L):  # one step after the other
        before.append(h)
        h = torch.where(t < ends, torch.addcmul(i[:, t] * v[:, t], f[:, t], h), h)
        hs.append(h)
    hs = torch.stack(hs, 1)
    alive = (torch.arange(L, device="cuda")[None] < ends)[:, :, None]
    y = hs if silu is None else hs * silu
    out = {"y": torch.where(alive, y, 0.0), "h_last": h}
    if op == "scan":
        return out
    before = torch.stack(before, 1)
    dy = torch.where(alive, s["dy"].double(), 0.0)
    dout = None
    if silu is not None:
        sig = torch.sigmoid(s["out_gate"].double())
        dout = torch.where(alive, dy * hs * (sig + silu * (1.0 - sig)), 0.0)
        dy = dy * silu
    G = torch.zeros((N, C), dtype=torch.float64, device="cuda") if s["dh"] is None else s["dh"].double()
    Gs = [None] * L
    for t in range(L - 1, -1, -1):  # G: the gradient at the state after step t
        live = t < ends
        Gs[t] = torch.where(live, G + dy[:, t], 0.0)
        G = torch.where(live, Gs[t] * f[:, t], G)
    Gs = torch.stack(Gs, 1)
    return {**out, "dgate": f * i * (before - v) * Gs, "dvalue": i * Gs, "dout_gate": dout, "dh0": G}
