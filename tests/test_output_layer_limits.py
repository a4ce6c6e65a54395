"""The output layer's operators at the largest sizes that they take: rows, vocabularies, operands of nearly 2 GiB, and
offsets past 32 bits."""

from __future__ import annotations

import numpy as np
import pytest

import paper_2609_14991_amd as F
from oracle import mx, projection
from oracle import scores as O
from test_logprobs import _near

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _bits(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def test_the_most_rows():
    """2^24 - 1 rows of 2 logits: log p = -log(1 + e^-d), by float64 on the device."""
    M = (1 << 24) - 1
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((1, M, 2), generator=g, device="cuda") * 3
    tok = torch.randint(-1, 2, (1, M), generator=g, device="cuda", dtype=torch.int32)
    o = F.score(x, tok, k=1)
    lp = torch.log_softmax(x.double(), 2)
    want = torch.where(tok >= 0, lp.gather(2, tok.clamp(min=0).long()[:, :, None])[:, :, 0], 0.0)
    # x - max and log s: a few roundings of each, and the exponential's of |d| under 40
    d = (x[:, :, 0] - x[:, :, 1]).double().abs()
    assert ((o["logp"].double() - want).abs() <= O.U32 * (8 + 4 * d + 2 * want.abs())).all()
    assert torch.equal(o["top"][:, :, 0].long(), (x[:, :, 1] > x[:, :, 0]).long())
    gl = torch.ones((1, M), device="cuda")
    grad = F.score_backward(x, o, tok, None, 1, gl)
    one = torch.where(tok[:, :, None] >= 0, torch.nn.functional.one_hot(tok.clamp(min=0).long(), 2).double() - lp.exp(), 0.0)
    assert ((grad.double() - one).abs() <= O.U32 * (16 + 8 * d)[:, :, None]).all()
    with pytest.raises(F.FusionError):
        F.score(torch.empty((1, M + 1, 1), device="cuda"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_widest_vocabulary(dtype):
    V = 1 << 24
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((1, 3, V), generator=g, device="cuda").to(dtype)
    x[0, 1] = torch.finfo(dtype).min                       # masked as a whole
    x[0, 2] += (torch.arange(V, device="cuda") * (8.0 / V)).to(dtype)
    tok = torch.tensor([[V - 1, V // 2, 12345]], dtype=torch.int32, device="cuda")
    o = F.score(x, tok, k=8)
    ref = O.scores(x.double().cpu().numpy(), tok.cpu().numpy(), None, 3, 1, 8)
    for n, tol in (("logp", "tol_logp"), ("entropy", "tol_entropy"), ("lse", "tol_lse"), ("top_logp", "tol_top")):
        _near(o[n].cpu().double().numpy(), ref[n], ref[tol], n)
    assert np.array_equal(o["top"].cpu().numpy(), ref["top"])
    ge = torch.ones((1, 3), device="cuda")
    grad = F.score_backward(x, o, tok, None, 1, ge, ge)
    got = grad.double()
    # the columns sum to 0, each off by its rounding and p's; a row masked as a whole: (1[y] - 1 / V)
    assert (got.sum(2).abs() <= got.abs().sum(2) * 2.0 ** (-8 if dtype == torch.bfloat16 else -16)).all()
    p = -got[0, 1, 0].item() * V
    assert abs(p - 1) <= 2.0 ** -8 + ref["tol_logp"][0, 1]
    assert (got[0, 1] < 0).sum() == V - 1 and abs(got[0, 1, V // 2].item() - 1) <= 2.0 ** -8


def test_hidden_states_of_nearly_2_gib():
    K, V = 640, 40
    M = 0x7FFFFFF0 // 2 // K
    A = torch.randn((1, M, K), device="cuda", dtype=torch.bfloat16)
    W = torch.randn((V, K), device="cuda").mul_(0.08).bfloat16()
    tok = torch.randint(0, V, (1, M), device="cuda", dtype=torch.int32)
    o = F.score_projected(A, W, None, tok)
    pick = np.concatenate([np.arange(70), M // 2 + np.arange(70), M - 1 - np.arange(140)])
    a, w, t = _bits(A[0, torch.tensor(pick)]), _bits(W), tok[:, torch.tensor(pick)].cpu().numpy()
    ref = O.scores(projection.joint_project(a, w)[None], t, None, pick.size, 1, 0)
    d = projection.fp32_error_bound(a, w).max(axis=1)
    for n, grow in (("logp", 2.0), ("lse", 1.0), ("entropy", 2.0 * ref["entropy"] + 0.01)):
        _near(o[n][:, torch.tensor(pick)].cpu().double().numpy(), ref[n], 2 * ref["tol_" + n] + 64 * O.U32 * (1 + ref["entropy"]) + grow * d * 1.01, n)
    assert torch.isfinite(o["lse"]).all() and (o["logp"] <= 0).all()
    with pytest.raises(F.FusionError):
        F.joint_logprobs_workspace(M + 1, V, K)


@pytest.mark.parametrize("K", [640, 1056])
def test_4_bit_states_of_nearly_2_gib(K):
    N = 40
    M = 0x7FFFFFF0 // (K // 2)
    q = torch.randint(0, 256, (M, K // 2), device="cuda", dtype=torch.uint8)
    s = torch.randint(125, 130, (M, F.mx_scale_stride(K)), device="cuda", dtype=torch.uint8)
    qw = torch.randint(0, 256, (N, K // 2), device="cuda", dtype=torch.uint8)
    sw = torch.randint(125, 130, (N, F.mx_scale_stride(K)), device="cuda", dtype=torch.uint8)
    out = F.project_mx((q, s), (qw, sw))
    pick = torch.tensor(np.concatenate([np.arange(70), M // 2 + np.arange(70), M - 1 - np.arange(140)]))
    a = mx.values(q[pick].cpu().numpy(), s[pick].cpu().numpy(), K)
    w = mx.values(qw.cpu().numpy(), sw.cpu().numpy(), K)
    bound = K * O.U32 * (np.abs(a) @ np.abs(w).T)
    assert np.all(np.abs(out[pick].cpu().double().numpy() - a @ w.T) <= bound)


def test_rows_to_quantise_past_32_bits():
    """More than 2^31 lanes, 2^33 bytes of elements and 2^35 of values; the rows looked at lie at both ends and between."""
    K = 4096
    R = (1 << 31) // (K // 8) + 77
    x = torch.empty((R, K), device="cuda", dtype=torch.bfloat16)
    pick = torch.tensor([0, 1, 1 << 19, (1 << 20) - 1, 1 << 20, 1 << 21, (1 << 21) + 1, R - 78, R - 77, R - 2, R - 1], device="cuda")
    x[pick] = (torch.randn((pick.numel(), K), device="cuda") * 3).bfloat16()
    q, s = F.quantize(x)
    want_q, want_s = mx.quantize(x[pick].double().cpu().numpy())
    assert np.array_equal(q[pick].cpu().numpy(), want_q) and np.array_equal(s[pick].cpu().numpy(), want_s)
    back = F.dequantize(q, s, torch.bfloat16)
    assert np.array_equal(back[pick].double().cpu().numpy(), mx.values(want_q, want_s, K))
