"""The conveniences of the output layer's operators on a stream that is not torch's current one: what they
allocate is that stream's, so that the current stream's next tensors do not take its memory while it is in use."""

from __future__ import annotations

import pytest

import paper_2609_14991_amd as F

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

T, S, B, V, K = 6, 40, 4, 1001, 320
H = S * B


def _inputs():
    g = torch.Generator(device="cuda").manual_seed(5)
    A = torch.randn((T, H, K), generator=g, device="cuda").bfloat16()
    W = (torch.randn((V, K), generator=g, device="cuda") / 9).bfloat16()
    tok = torch.randint(0, V, (T, H), generator=g, device="cuda", dtype=torch.int32)
    par = torch.randint(0, B, (T, H), generator=g, device="cuda", dtype=torch.int32)
    gl = torch.randn((T, H), generator=g, device="cuda")
    return A, W, tok, par, gl


def _calls(A, W, tok, par, gl):
    """name -> call(stream), each giving a list of tensors."""
    x = F.project(A.view(T * H, K), W).view(T, H, V)
    scored = F.score(x, tok, par, B)
    wq, aq = F.quantize(W), F.quantize(A.view(T * H, K))
    return dict(
        score=lambda s: list(F.score(x, tok, par, B, 4, stream=s).values()),
        score_backward=lambda s: [F.score_backward(x, scored, tok, par, B, gl, gl, stream=s)],
        score_projected=lambda s: list(F.score_projected(A, W, None, tok, par, B, stream=s).values()),
        quantize=lambda s: list(F.quantize(A.view(T * H, K), stream=s)),
        dequantize=lambda s: [F.dequantize(*aq, stream=s)],
        project_mx=lambda s: [F.project_mx(A.view(T * H, K), wq, stream=s)])


@pytest.mark.parametrize("name", ["score", "score_backward", "score_projected", "quantize", "dequantize", "project_mx"])
def test_memory_of_a_busy_stream_is_not_handed_out(name, monkeypatch):
    call = _calls(*_inputs())[name]
    want = call(None)
    big = torch.randn((4096, 4096), device="cuda")
    big @ big
    torch.cuda.synchronize()
    # where everything that the call allocates lies
    held, empty = [], torch.empty

    def watched(*a, **kw):
        t = empty(*a, **kw)
        held.append((t.data_ptr(), t.numel() * t.element_size()))
        return t

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):
            big @ big  # the call's work waits behind it
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", watched)
        got = call(side.cuda_stream)
    # the same sizes, allocated and overwritten on the current stream while the side stream is at work
    for at, size in held:
        t = empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF)
        assert not any(a < t.data_ptr() + size and t.data_ptr() < a + n for a, n in held)
    torch.cuda.synchronize()
    assert len(held) >= len(want)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_the_default_stream_by_its_address():
    """Address 0 is the default stream, also from under another one."""
    call = _calls(*_inputs())["score_projected"]
    want = call(None)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = call(0)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
