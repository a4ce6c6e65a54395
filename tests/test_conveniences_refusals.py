"""What the conveniences of the output layer refuse before anything is launched (CPU)."""

from __future__ import annotations

import pytest

import paper_2609_14991_amd as F

torch = pytest.importorskip("torch")


class OnDevice:
    """A tensor as the checks see it, on a device that need not exist."""

    is_cuda = True

    def __init__(self, t, device):
        self.t, self.device_index, self.shape, self.dtype = t, device, t.shape, t.dtype
        self.device = torch.device("cpu")

    def get_device(self):
        return self.device_index

    def __getattr__(self, name):
        return getattr(self.t, name)

    def unsqueeze(self, d):
        return OnDevice(self.t.unsqueeze(d), self.device_index)


@pytest.fixture
def on(monkeypatch):
    """Tensors on a device of choice while device 0 is the current one; no call reaches the library."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def reached(*_):
        raise AssertionError("launched")

    for name in ("token_logprobs", "token_logprobs_backward", "joint_logprobs", "mx_quantize", "mx_dequantize", "joint_project_mx"):
        monkeypatch.setattr(F, name, reached)
    return OnDevice


def _calls(on, d, odd=None):
    """Every convenience with its tensors on device d, the one named `odd` on device 1."""
    t = lambda n, x: on(x, 1 if n == odd else d)  # noqa: E731
    x, f = torch.zeros((2, 4, 8)), torch.zeros((2, 4))
    i = torch.zeros((2, 4), dtype=torch.int32)
    A, W = torch.zeros((2, 4, 64)).bfloat16(), torch.zeros((8, 64)).bfloat16()
    q, s = torch.zeros((8, 32), dtype=torch.uint8), torch.zeros((8, 8), dtype=torch.uint8)
    scored = lambda: dict(logp=t("logp", f), entropy=t("entropy", f), lse=t("lse", f))  # noqa: E731
    return [("logits tokens parents", lambda: F.score(t("logits", x), t("tokens", i), t("parents", i), 2)),
            ("logits tokens parents logp entropy lse grad_logp grad_entropy",
             lambda: F.score_backward(t("logits", x), scored(), t("tokens", i), t("parents", i), 2, t("grad_logp", f),
                                      t("grad_entropy", f), in_place=True)),
            ("A W bias tokens parents",
             lambda: F.score_projected(t("A", A), t("W", W), t("bias", torch.zeros(8)), t("tokens", i), t("parents", i), 2)),
            ("x", lambda: F.quantize(t("x", torch.zeros((4, 64))))), ("q scales", lambda: F.dequantize(t("q", q), t("scales", s))),
            ("q scales W Ws bias", lambda: F.project_mx((t("q", q), t("scales", s)), (t("W", q), t("Ws", s)), t("bias", torch.zeros(8))))]


def test_tensors_of_another_device_than_the_current_one(on):
    for names, call in _calls(on, 0):
        with pytest.raises(AssertionError, match="launched"):
            call()
    for names, _ in _calls(on, 0):
        for name in names.split():
            for has, call in _calls(on, 0, odd=name):
                if has == names:
                    with pytest.raises(ValueError, match="current CUDA device"):
                        call()
    for _, call in _calls(on, 1):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()


@pytest.mark.parametrize("B", [0, -1, 3, 5])
def test_slots_that_the_rows_are_no_multiple_of(on, B):
    x, f, i = (on(t, 0) for t in (torch.zeros((2, 4, 8)), torch.zeros((2, 4)), torch.zeros((2, 4), dtype=torch.int32)))
    A, W = on(torch.zeros((2, 4, 64)).bfloat16(), 0), on(torch.zeros((8, 64)).bfloat16(), 0)
    for call in (lambda: F.score(x, i, None, B), lambda: F.score_projected(A, W, None, i, None, B),
                 lambda: F.score_backward(x, dict(logp=f, entropy=f, lse=f), i, None, B, f)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16, torch.float32, torch.float64])
def test_a_workspace_counts_by_its_bytes(dtype):
    """joint_logprobs takes the workspace's size from its tensor: one of another type holds as many floats as its
    bytes.  (Refused for its size before anything is launched.)"""
    need = 4 * F.joint_logprobs_workspace(8, 50, 64)
    size = torch.empty(0, dtype=dtype).element_size()
    with pytest.raises(F.FusionError, match="workspace too small"):
        F.joint_logprobs(Address(), Address(), None, 64, 1, 8, 1, 50, None, None, None, Address(), None,
                         torch.zeros((need - 1) // size, dtype=dtype), stream=0)


class Address:
    def data_ptr(self):
        return 4096
