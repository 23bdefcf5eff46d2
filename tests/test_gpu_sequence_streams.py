"""The sequence operators on a stream that is not the tensors' own: memory that the
caller gives up right after the call is not used again before that stream has
read it, and what the call allocates is free of the caller's unfinished work."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(1)


def _calls():
    from paper_1905_05233_amd import sequence_ops as S
    w4 = S.W4Matrix.quantize(torch.randn((600, 512), device="cuda"), 64)
    weight = torch.rand(512, device="cuda").bfloat16()
    lengths = torch.tensor([300, 17], dtype=torch.int32, device="cuda")

    def train(z, v, o, dy, stream):
        y, h, s = S.gated_scan(z, v, o, lengths=lengths, save_states=True, stream=stream)
        return (y, h, *S.gated_scan_backward(dy, z, v, s, out_gate=o, lengths=lengths, stream=stream))

    return {
        "scan": train,
        "step": lambda z, v, o, dy, stream: S.gated_step(z[:, 0], v[:, 0], o[:, 0].float(), out_gate=dy[:, 0], stream=stream),
        "norm": lambda z, v, o, dy, stream: S.rms_norm(z, weight, residual=v, stream=stream),
        "fp8": lambda z, v, o, dy, stream: [t.float() for t in S.rms_norm_fp8(z, weight, residual=v, group=64, stream=stream)],
        "norm_gradients": lambda z, v, o, dy, stream: S.rms_norm_backward(dy, z, weight, dr=o, stream=stream),
        "matvec": lambda z, v, o, dy, stream: (S.matvec_w4(z[0], w4, stream=stream),),
    }


@pytest.mark.parametrize("name", ["scan", "step", "norm", "norm_gradients", "matvec"])
def test_memory_given_up_after_the_call(name):
    call = _calls()[name]
    parts = [torch.randn((2, 300, 512), device="cuda").bfloat16() for _ in range(4)]
    want = [t.clone() for t in call(*parts, None)]
    side = torch.cuda.Stream()
    for _ in range(3):
        inputs = [p.clone() for p in parts]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)        # some ms of work ahead of the call
        got = call(*inputs, side)
        del inputs
        junk = [torch.full((2, 300, 512), 9.0, device="cuda").bfloat16() for _ in range(16)]   # would take their place
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(want, got):
            assert torch.equal(a, b), name
        del junk, got


def test_outputs_begin_free_of_the_callers_work():
    """A block that the caller's stream gave back, with work on it still to be done, is
    not handed to the other stream."""
    call = _calls()["norm"]
    parts = [torch.randn((2, 300, 512), device="cuda").bfloat16() for _ in range(4)]
    want = [t.clone() for t in call(*parts, None)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    late = [torch.empty((2, 300, 512), dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    torch.cuda._sleep(20_000_000)
    for t in late:
        t.fill_(5.0)                             # behind the wait, on the caller's stream
    del late, t
    got = call(*parts, side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_quantized_matrices_on_another_stream():
    from paper_1905_05233_amd import sequence_ops as S
    m = torch.randn((64, 256), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w = S.W4Matrix.quantize(m, 64, stream=side)
    back = w.dequantize(torch.float32, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(back, S.W4Matrix.quantize(m, 64).dequantize(torch.float32))
