"""Linear attention and the norm of heads with rotation where calls are long, far apart in
memory or many: sequences cut into segments, offsets and launches past 2^32, memory given
up after a call, graphs that live side by side, and the operators run together."""
import numpy as np
import pytest
import torch

import attention_reference as A
import sequence_reference as R
from gpu_helpers import TORCH

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)


def _np(t):
    return t.double().cpu().numpy()


def _randn(*shape, dtype="bf16"):
    return torch.randn(shape, device="cuda").to(TORCH[dtype])


def _inputs(N, L, Hq, Hk, Hv, H, Dk, Dv, dtype):
    return (_randn(N, L, Hq, Dk, dtype=dtype), _randn(N, L, Hk, Dk, dtype=dtype), _randn(N, L, Hv, Dv, dtype=dtype),
            _randn(N, L, H, Dv, dtype=dtype))


NAMES = ("y", "s_last", "dq", "dk", "dv", "ds0")


def _run(q, k, v, g, dy, stream=None, out=None, y=None, **kw):
    from paper_1905_05233_amd import sequence_ops as S
    ds = kw.pop("ds_last", None)
    return (*S.linear_attention(q, k, v, g, y=y, stream=stream, **kw),
            *S.linear_attention_backward(dy, q, k, v, g, ds_last=ds, out=out, stream=stream, **kw))


# few heads and many steps: the sequences go in segments, of one tile to many, the last of
# them short, from either end
LONG = [(1, 4000, 1, 1, 1, 1, 128, 128, "bf16"), (5, 1999, 1, 1, 1, 1, 40, 72, "bf16"), (2, 3001, 2, 1, 1, 2, 64, 64, "bf16"),
        (1, 2500, 1, 1, 1, 1, 200, 130, "bf16"), (3, 1500, 1, 3, 3, 3, 17, 100, "f16"), (1, 2049, 1, 1, 1, 1, 128, 64, "f16"),
        (2, 1700, 2, 2, 1, 2, 48, 48, "f32"), (1, 1025, 1, 1, 1, 1, 256, 33, "f32")]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("case", LONG, ids=str)
def test_segments(case, ragged):
    *shape, dtype = case
    N, L, *_, H, Dk, Dv = shape
    print(f"[segments] {case} {ragged}", flush=True)
    q, k, v, dy = _inputs(*shape, dtype)
    g = torch.tensor([-0.003, -0.2, -1.0][:H], device="cuda")
    s0, ds = [torch.randn((N, H, Dk, Dv), device="cuda") for _ in range(2)]
    lengths = np.array([L - 1, 70, 0, 1, L // 2 + 3][-N:] if ragged else [L] * N)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda") if ragged else None
    got = _run(q, k, v, g, dy, s0=s0, ds_last=ds, lengths=n)
    ref = A.attention(_np(q), _np(k), _np(v), _np(g), _np(s0), lengths, Dk ** -0.5, dtype, _np(dy), _np(ds))
    for name, t in zip(NAMES, got):
        R.assert_close(_np(t), *ref[name], "f32" if name in ("s_last", "ds0") else dtype, name)
    for name, t in zip(NAMES, got):
        for i in range(N):
            if name not in ("s_last", "ds0"):
                assert not t[i, lengths[i]:].any(), name


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [1, 63, 64, 1000, 1498])
def test_segments_keep_the_order_of_steps(bad, at):
    """With segments too a value that is not finite is in nothing ahead of it."""
    from paper_1905_05233_amd import sequence_ops as S
    q, k, v, dy = _inputs(1, 1500, 1, 1, 1, 1, 32, 80, "bf16")
    g = torch.tensor([-0.01], device="cuda")
    ref = A.attention(_np(q), _np(k), _np(v), _np(g), None, None, 32 ** -0.5, "bf16", _np(dy))

    def held(name, got, part):
        want, bound = ref[name]
        R.assert_close(_np(got)[:, part], want[:, part], bound[:, part], "bf16", name)

    for i in range(3):
        t = [q.clone(), k.clone(), v.clone()]
        t[i][0, at, 0, 3] = bad
        y, s = S.linear_attention(*t, g)
        assert not bool(torch.isfinite(y[0, at]).all()) and bool(torch.isfinite(s).all()) == (i == 0)
        held("y", y, slice(0, at))
        if i > 0:
            held("dq", S.linear_attention_backward(dy, *t, g)[0], slice(0, at))
    dy[0, at, 0, 3] = bad
    _, dk, dv, _ = S.linear_attention_backward(dy, q, k, v, g)
    held("dk", dk, slice(at + 1, None))
    held("dv", dv, slice(at + 1, None))


# (sequences, steps, heads) and strides of them, one past 2^32 elements in all
FAR = {"sequences": ((2, 70, 3), (2 ** 32 + 40, 1000, 150)), "steps": ((1, 70, 3), (0, 2 ** 26 + 8, 150)),
       "heads": ((1, 70, 3), (0, 150, 2 ** 31 + 56))}


@pytest.mark.parametrize("axis", FAR)
def test_offsets_past_32_bits(axis):
    from paper_1905_05233_amd import sequence_ops as S
    (N, L, H), strides = FAR[axis]
    D, width = 48, 150
    span = sum((n - 1) * s for n, s in zip((N, L, H), strides)) + width
    assert span > 2 ** 32
    buf = torch.empty(span + 16, dtype=torch.bfloat16, device="cuda")
    if axis != "heads":      # the rows of a step hold all heads
        strides = (strides[0], max(strides[1], H * width), width)

    def far(i):              # three tensors in a row's 150 channels
        return buf.as_strided((N, L, H, D), (*strides, 1), i * 50)

    q, k, v, dy = _inputs(N, L, H, H, H, H, D, D, "bf16")
    g = torch.tensor([-0.01, -0.1, -1.0], device="cuda")
    want = _run(q, k, v, g, dy)
    for i, t in enumerate((q, k, v)):
        far(i).copy_(t)
    for name, a, b in zip(NAMES, want, _run(far(0), far(1), far(2), g, dy)):
        assert torch.equal(a, b), name
    y, _ = S.linear_attention(q, k, v, g, y=far(0))
    assert torch.equal(y, want[0])
    got = S.linear_attention_backward(y.copy_(dy), q, k, v, g)      # dy far away
    assert all(torch.equal(a, b) for a, b in zip(want[2:], got))
    S.linear_attention_backward(dy, q, k, v, g, out=[far(i) for i in range(3)])
    assert all(torch.equal(a, far(i)) for i, a in enumerate(want[2:5]))
    dq, dk, dv, ds0 = S.linear_attention_backward(dy, q[:, :, :1], k, v, g, out=[far(0)[:, :, :1], far(1), far(2)])
    assert torch.equal(dq, S.linear_attention_backward(dy, q[:, :, :1], k, v, g)[0])
    w, rot = [_randn(D) for _ in range(2)], S.Rotary(32)
    plain = (*S.head_norm_rotate(q, k, *w, rot), *S.head_norm_rotate_backward(dy, v, q, k, *w, rot))
    far(0).copy_(q), far(1).copy_(k)
    got = (*S.head_norm_rotate(far(0), far(1), *w, rot), *S.head_norm_rotate_backward(dy, v, far(0), far(1), *w, rot))
    assert all(torch.equal(a, b) for a, b in zip(plain, got))
    S.head_norm_rotate(far(0), far(1), *w, rot, q_out=far(0), k_out=far(1))
    assert torch.equal(far(0), plain[0]) and torch.equal(far(1), plain[1])


def test_states_past_32_bits():
    """65540 states of 256 x 256 channels, 17 GB of them, written by a call of one step and
    updated in place by a single step."""
    from paper_1905_05233_amd import sequence_ops as S
    N, D = 65540, 256
    q, k, v = [_randn(N, 1, 1, D) for _ in range(3)]
    g = torch.tensor([-0.5], device="cuda")
    y, s = S.linear_attention(q, k, v, g, scale=1.0)
    at = [0, 1, 32767, 32768, 65535, 65536, 65539]
    for n in at:
        kv = k[n, 0, 0].double()[:, None] * v[n, 0, 0].double()
        assert torch.equal(s[n, 0].double(), kv)
    before = s[at].double()
    k2, v2 = [_randn(N, 1, D) for _ in range(2)]
    y, same = S.linear_attention_step(q[:, 0], k2, v2, g, s, scale=1.0, s_new=s)
    assert same is s
    for i, n in enumerate(at):
        want = float(np.exp(-0.5)) * before[i, 0] + k2[n, 0].double()[:, None] * v2[n, 0].double()
        off = (s[n, 0].double() - want).abs() - 8 * 2.0 ** -24 * (want.abs() + before[i, 0].abs())
        assert float(off.max()) <= 0.0
        out = q[n, 0, 0].double() @ want
        size = q[n, 0, 0].double().abs() @ want.abs()
        assert bool(((y[n, 0].double() - out).abs() <= 2.0 ** -8 * out.abs() + (2 * D + 100) * 2.0 ** -24 * size).all())


def test_more_sequences_than_a_launch_takes():
    """A launch takes fewer than 2^32 threads, 2^22 workgroups of 1024."""
    from paper_1905_05233_amd import sequence_ops as S
    N, Dv = 2 ** 22 + 5, 65
    q, k, v = _randn(N, 1, 1, 1), _randn(N, 1, 1, 1), _randn(N, 1, 1, Dv)
    y, s = S.linear_attention(q, k, v, torch.tensor([-1.0], device="cuda"), scale=2.0)
    kv = k.float() * v.float()
    assert torch.equal(s.view(N, 1, 1, Dv), kv)      # products of 16 bits are exact
    want = 2.0 * q.float() * kv
    assert bool(((y.float() - want).abs() <= (2.0 ** -8 + 3 * 2.0 ** -16 + 100 * 2.0 ** -24) * want.abs()).all())


def test_rows_past_a_launch():
    """More rows of heads than workgroups have groups for, one row in many."""
    from paper_1905_05233_amd import sequence_ops as S
    N, D = 2 ** 21 + 3, 8
    q, k = _randn(1, N, 2, D), _randn(1, N, 1, D)
    w, rot = [_randn(D) for _ in range(2)], S.Rotary(D)
    yq, yk = S.head_norm_rotate(q, k, *w, rot)
    for a in (0, 2 ** 20 + 1, N - 7):
        part = S.head_norm_rotate(q[:, a:a + 7], k[:, a:a + 7], *w, rot, start=a)
        assert torch.equal(part[0], yq[:, a:a + 7]) and torch.equal(part[1], yk[:, a:a + 7])


def _calls():
    from paper_1905_05233_amd import sequence_ops as S
    g = torch.tensor([-0.02, -0.3], device="cuda")
    rot, w = S.Rotary(64), [_randn(64) for _ in range(2)]
    n = torch.tensor([700, 650], dtype=torch.int32, device="cuda")
    state = torch.randn((2, 2, 64, 64), device="cuda")

    def rotated(q, k, dy, stream):
        return (*S.head_norm_rotate(q, k, *w, rot, stream=stream),
                *S.head_norm_rotate_backward(dy, dy, q, k, *w, rot, stream=stream))

    return {
        "attention": lambda q, k, v, dy, stream: _run(q, k, v, g, dy, stream, lengths=n),
        "shared": lambda q, k, v, dy, stream: _run(q[:, :, :1], k[:, :, 1:], v, g, dy, stream),
        "step": lambda q, k, v, dy, stream: S.linear_attention_step(q[:, 3], k[:, 3], v[:, 3], g, state, stream=stream),
        "rotate": lambda q, k, v, dy, stream: rotated(q, k, dy, stream),
    }


@pytest.mark.parametrize("name", ["attention", "shared", "step", "rotate"])
def test_memory_given_up_after_the_call(name):
    call = _calls()[name]
    parts = _inputs(2, 700, 2, 2, 2, 2, 64, 64, "bf16")
    want = [t.clone() for t in call(*parts, None)]
    side = torch.cuda.Stream()
    for _ in range(3):
        inputs = [p.clone() for p in parts]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)        # some ms of work ahead of the call
        got = call(*inputs, side)
        del inputs
        junk = [torch.full(parts[0].shape, 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(16)]
        states = [torch.full((2, 2, 12, 64, 64), 9.0, device="cuda") for _ in range(4)]   # or a workspace's place
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(want, got):
            assert torch.equal(a, b), name
        del junk, states, got


@pytest.mark.parametrize("name", ["attention", "shared", "rotate"])
def test_graphs_side_by_side(name):
    """Two graphs, captured one after the other and replayed at the same time on two
    streams with eager calls between: each has a workspace of its own."""
    call = _calls()[name]
    sets = [list(_inputs(2, 700, 2, 2, 2, 2, 64, 64, "bf16")) for _ in range(2)]
    for s in sets:
        call(*s, None)
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in sets], []
    for graph, s in zip(graphs, sets):
        with torch.cuda.graph(graph):
            outs.append(call(*s, None))
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(4):
        for s in sets:
            for t in s:
                t.copy_(torch.randn(t.shape, device="cuda"))
        want = [call(*s, None) for s in sets]
        for o in outs:
            for t in o:
                t.fill_(3.0)
        torch.cuda.synchronize()
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
        extra = call(*sets[0], None)
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            assert all(torch.equal(a, b) for a, b in zip(w, o)), name
        assert all(torch.equal(a, b) for a, b in zip(want[0], extra)), name


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_operators_together(dtype):
    """Queries, keys and values from one projection's rows; the norm and rotation in
    place, attention over a prompt and single tokens behind it, against the 64-bit
    formulas at what each operator was given."""
    from paper_1905_05233_amd import sequence_ops as S
    N, L, more, Hq, Hk, D, Dv = 2, 130, 5, 4, 2, 32, 48
    widths = [Hq * D, Hk * D, Hq * Dv]
    rows = _randn(N, L + more, sum(widths), dtype=dtype)
    q, k, v = [t.unflatten(2, (h, -1)) for t, h in zip(rows.split(widths, 2), (Hq, Hk, Hq))]
    x, w, rot = (q.clone(), k.clone()), [1.0 + 0.1 * _randn(D, dtype=dtype) for _ in range(2)], S.Rotary(16)
    g = torch.tensor([-0.01, -0.1, -0.5, -2.0], device="cuda")
    S.head_norm_rotate(q[:, :L], k[:, :L], *w, rot, q_out=q[:, :L], k_out=k[:, :L])
    y, s = S.linear_attention(q[:, :L], k[:, :L], v[:, :L], g)
    outs = [y]
    for l in range(L, L + more):
        at = torch.full((N,), l, dtype=torch.int32, device="cuda")
        S.head_norm_rotate(q[:, l], k[:, l], *w, rot, positions=at, q_out=q[:, l], k_out=k[:, l])
        y, s = S.linear_attention_step(q[:, l], k[:, l], v[:, l], g, s, s_new=s)
        outs.append(y[:, None])
    where = np.tile(np.arange(L + more), (N, 1))
    for before, now, weight in zip(x, (q, k), w):
        want, bound = A.rotate(_np(before), _np(weight), [10000.0 ** (-i / 8) for i in range(8)], where, 1e-6, False)
        R.assert_close(_np(now), want, bound, dtype, "rotated")
    ref = A.attention(_np(q), _np(k), _np(v), _np(g), None, None, D ** -0.5, dtype)
    R.assert_close(_np(torch.cat(outs, 1)), *ref["y"], dtype, "y")
    R.assert_close(_np(s), *ref["s_last"], "f32", "s")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradients_together(dtype):
    """A training pass of both: the gradients of queries, keys and values go in the slices
    of one projection's gradient, and those through the norm and rotation in place; each
    operator against the 64-bit formulas at what it was given."""
    from paper_1905_05233_amd import sequence_ops as S
    N, L, Hq, Hk, H, D, Dv = 3, 90, 4, 2, 4, 32, 24
    widths, lengths = [Hq * D, Hk * D, Hk * Dv], np.array([90, 0, 61])
    rows = _randn(N, L, sum(widths), dtype=dtype)
    x, k0, v = [t.unflatten(2, (h, -1)) for t, h in zip(rows.split(widths, 2), (Hq, Hk, Hk))]
    w, rot = [1.0 + 0.1 * _randn(D, dtype=dtype) for _ in range(2)], S.Rotary(32, adjacent=True)
    g, n = torch.tensor([-0.01, -0.1, -0.5, -2.0], device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q, k = S.head_norm_rotate(x, k0, *w, rot)
    y, _ = S.linear_attention(q, k, v, g, lengths=n)
    dy, drows = torch.randn_like(y), torch.full_like(rows, 7.0)
    out = [t.unflatten(2, (h, -1)) for t, h in zip(drows.split(widths, 2), (Hq, Hk, Hk))]
    S.linear_attention_backward(dy, q, k, v, g, lengths=n, out=out)
    ref = A.attention(_np(q), _np(k), _np(v), _np(g), None, lengths, D ** -0.5, dtype, _np(dy))
    R.assert_close(_np(y), *ref["y"], dtype, "y")
    for name, t in zip(("dq", "dk", "dv"), out):
        R.assert_close(_np(t), *ref[name], dtype, name)
    before = [t.clone() for t in out[:2]]
    dq, dk, dwq, dwk = S.head_norm_rotate_backward(*out[:2], x, k0, *w, rot, out=out[:2])
    assert dq is out[0] and dk is out[1]
    where, f = np.tile(np.arange(L), (N, 1)), [10000.0 ** (-i / 16) for i in range(16)]
    for at, weight, d, dx, dw in ((x, w[0], before[0], dq, dwq), (k0, w[1], before[1], dk, dwk)):
        (want, bound), (want_w, bound_w) = A.rotate(_np(at), _np(weight), f, where, 1e-6, True, _np(d))
        R.assert_close(_np(dx), want, bound, dtype, "dx")
        R.assert_close(_np(dw), want_w, bound_w, "f32", "dw")
    for i in range(N):
        assert not drows[i, lengths[i]:].any()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads", [(2, 2), (1, 2)], ids=str)
@pytest.mark.parametrize("Dv", [3, 20, 72, 150])
def test_padding_is_cleared_and_nothing_beside_it(Dv, heads, dtype):
    from paper_1905_05233_amd import sequence_ops as S
    N, L, Dk, lengths = 4, 700, 24, [0, 1, 650, 699]
    q, k, v, dy = _inputs(N, L, *heads, 2, 2, Dk, Dv, dtype)
    g, n = torch.tensor([-0.1, -0.01], device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    width = 2 * Dv + (heads[0] + heads[1]) * Dk
    buf = torch.full((N, L, width + 1), 7.0, dtype=TORCH[dtype], device="cuda")
    parts = buf[:, :, 1:].split([2 * Dv, heads[0] * Dk, heads[1] * Dk], 2)
    dv, dq, dk = [t.unflatten(2, (h, -1)) for t, h in zip(parts, (2, *heads))]
    want = _run(q, k, v, g, dy, lengths=n)
    S.linear_attention(q, k, v, g, lengths=n, y=dv)
    assert torch.equal(dv, want[0])
    S.linear_attention_backward(dy, q, k, v, g, lengths=n, out=(dq, dk, dv))
    for a, b in zip((dq, dk, dv), want[2:5]):
        assert torch.equal(a, b)
        for i, e in enumerate(lengths):
            assert not a[i, e:].any() and (e == 0 or bool(a[i, :e].any()))
    assert bool((buf[:, :, 0] == 7.0).all())


def test_work_on_both_streams_at_once():
    """A call on the current stream and one on another, in flight together."""
    call = _calls()["attention"]
    sets = [_inputs(2, 700, 2, 2, 2, 2, 64, 64, "bf16") for _ in range(2)]
    want = [call(*s, None) for s in sets]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a, b = call(*sets[0], None), call(*sets[1], side)
        torch.cuda.current_stream().wait_stream(side)
        for w, got in zip(want, (a, b)):
            assert all(torch.equal(x, y) for x, y in zip(w, got))
