"""Token scoring (token_logprobs) and its gradient: the oracle pinned on the CPU,
the kernels against it on the GPU, within the error bounds of their fp32
arithmetic (``oracle.scores``)."""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

import paper_2609_14991_amd as F
from oracle import scores as O

torch = pytest.importorskip("torch")

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
LOWEST = {"float32": -3.4028234663852886e38, "bfloat16": -3.3895313892515355e38, "float16": -65504.0}


# ---------------------------------------------------------------------------
# the oracle (CPU)
# ---------------------------------------------------------------------------
def test_oracle_equals_log_softmax_and_its_gradient():
    rng = np.random.default_rng(1)
    T, S, B, V = 3, 2, 3, 17
    x = rng.standard_normal((T, S * B, V)) * 3
    tok = rng.integers(0, V, (T, S * B))
    par = rng.integers(0, B, (T, S * B))
    tok[1, 2], par[1, 2] = -1, -1
    tok[2, 0] = -1
    gl, ge = rng.standard_normal((T, S * B)), rng.standard_normal((T, S * B))
    o = O.scores(x, tok, par, S, B, 4)
    xt = torch.tensor(x, requires_grad=True)
    row = torch.tensor(O.rows_of(par, T, S, B))
    lp = torch.log_softmax(xt, 2)[torch.arange(T)[:, None], row.clamp(min=0)]
    live = row >= 0
    logp = torch.where(live & (torch.tensor(tok) >= 0), lp.gather(2, torch.tensor(tok).clamp(min=0)[:, :, None])[:, :, 0], 0.0)
    ent = torch.where(live, -(lp.exp() * lp).sum(2), 0.0)
    assert np.allclose(o["logp"], logp.detach().numpy(), atol=1e-12)
    assert np.allclose(o["entropy"], ent.detach().numpy(), atol=1e-12)
    top = torch.topk(lp, 4, 2)
    assert np.allclose(o["top_logp"][live.numpy()], top[0][live].detach().numpy(), atol=1e-12)
    assert np.array_equal(o["top"][live.numpy()], top[1][live].numpy())
    ((logp * torch.tensor(gl)).sum() + (ent * torch.tensor(ge)).sum()).backward()
    grad, _ = O.gradient(x, tok, par, S, B, gl, ge)
    assert np.allclose(grad, xt.grad.numpy(), atol=1e-12)


def test_oracle_gradient_equals_differences():
    rng = np.random.default_rng(2)
    T, S, B, V = 1, 1, 2, 6
    x = rng.standard_normal((T, B, V))
    tok, par = np.array([[3, 5]]), np.array([[1, 1]])
    gl, ge = rng.standard_normal((T, B)), rng.standard_normal((T, B))

    def total(y):
        o = O.scores(y, tok, par, S, B, 0)
        return (o["logp"] * gl).sum() + (o["entropy"] * ge).sum()

    grad, _ = O.gradient(x, tok, par, S, B, gl, ge)
    for h in range(B):
        for y in range(V):
            step = np.zeros_like(x)
            step[0, h, y] = 1e-5
            assert abs((total(x + step) - total(x - step)) / 2e-5 - grad[0, h, y]) < 1e-8


def test_oracle_rows_without_a_distribution():
    x = np.array([[[-np.inf] * 3, [1.0, np.inf, 0.0], [np.nan, 0.0, 0.0], [0.0, -np.inf, 0.0]]])
    o = O.scores(x, np.array([[0, 0, 1, 1]]), None, 4, 1, 2)
    assert np.array_equal(o["lse"][0, :1], [-np.inf]) and np.isnan(o["lse"][0, 1:3]).all()
    assert o["logp"][0, 0] == -np.inf and np.isnan(o["logp"][0, 1:3]).all() and o["logp"][0, 3] == -np.inf
    assert o["entropy"][0, 0] == 0.0 and abs(o["entropy"][0, 3] - np.log(2)) < 1e-15
    assert o["top"][0].tolist() == [[-1, -1], [-1, -1], [-1, -1], [0, 2]]


# ---------------------------------------------------------------------------
# refusals (CPU): nothing is launched
# ---------------------------------------------------------------------------
P = ctypes.c_void_p
SOME = P(4096)  # a pointer that no refused call follows


def _forward(logits=SOME, dtype=0, stride=8, T=2, S=1, B=2, V=8, tokens=SOME, parents=None, k=0, logp=SOME,
             entropy=None, lse=None, top=None, top_logp=None):
    return F.lib().token_logprobs(logits, dtype, stride, T, S, B, V, tokens, parents, k, logp, entropy, lse, top,
                                  top_logp, None)


def _backward(logits=SOME, dtype=0, stride=8, T=2, S=1, B=2, V=8, tokens=SOME, parents=None, logp=SOME, entropy=SOME,
              lse=SOME, gl=SOME, ge=None, grad=P(8192), g_stride=8):
    return F.lib().token_logprobs_backward(logits, dtype, stride, T, S, B, V, tokens, parents, logp, entropy, lse, gl,
                                           ge, grad, g_stride, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), "ARG"), (dict(dtype=-1), "ARG"), (dict(T=-1), "ARG"), (dict(S=-1), "ARG"), (dict(B=0), "ARG"),
    (dict(V=0), "ARG"), (dict(V=(1 << 24) + 1, stride=1 << 25), "ARG"), (dict(stride=7), "ARG"),
    (dict(stride=1 << 61), "ARG"), (dict(T=1 << 20, S=1 << 10), "UNSUPPORTED"), (dict(S=1 << 30, B=4), "UNSUPPORTED"),
    (dict(parents=SOME, B=33), "UNSUPPORTED"), (dict(logits=None), "ARG"), (dict(logits=P(4098)), "ARG"),
    (dict(logits=P(4097), dtype=1), "ARG")])
def test_refusals_of_both(bad, code):
    want = getattr(F, "FUSION_E_" + code)
    assert _forward(**bad) == want and F.fusion_last_error()
    assert _backward(**bad) == want


@pytest.mark.parametrize("bad", [dict(k=9), dict(k=-1), dict(tokens=None), dict(k=2), dict(k=2, top=SOME), dict(logp=None)])
def test_refusals_of_scoring(bad):
    assert _forward(**bad) == F.FUSION_E_ARG


@pytest.mark.parametrize("bad", [dict(gl=None), dict(lse=None), dict(grad=None), dict(tokens=None), dict(logp=None),
                                 dict(ge=SOME, entropy=None), dict(g_stride=7), dict(grad=P(8194)),
                                 dict(grad=SOME, g_stride=9)])
def test_refusals_of_the_gradient(bad):
    assert _backward(**bad) == F.FUSION_E_ARG


def test_empty_calls_touch_nothing():
    assert _forward(T=0, logits=None, tokens=None, logp=None) == F.FUSION_OK
    assert _forward(S=0, logits=None) == F.FUSION_OK
    assert _backward(T=0, logits=None, lse=None, grad=None) == F.FUSION_OK


def test_gradient_of_another_type_is_refused():
    with pytest.raises(ValueError):
        F.token_logprobs_backward(torch.zeros(1, 1, 4), 4, 1, 1, 1, 4, None, None, None, None, None, None, None,
                                  torch.zeros(1, 1, 4, dtype=torch.bfloat16), 4)


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def dev():
    return torch.device("cuda:0")


def _place(x, pad, offset):
    """logits [T, H, V] on the GPU, rows V + pad apart, the first one `offset` elements into its buffer,
    NaN in every element that is not theirs."""
    T, H, V = x.shape
    buf = torch.full((T * H * (V + pad) + offset + 8,), float("nan"), dtype=x.dtype, device=dev())
    view = buf[offset:offset + T * H * (V + pad)].view(T, H, V + pad)[:, :, :V]
    view.copy_(x)
    return view, V + pad


def _score(x, tokens, parents, S, B, k, pad=0, offset=0):
    T, H, V = x.shape
    view, stride = _place(x, pad, offset)
    tok = None if tokens is None else torch.tensor(tokens, dtype=torch.int32, device=dev())
    par = None if parents is None else torch.tensor(parents, dtype=torch.int32, device=dev())
    out = {n: torch.full((T, H), 7.0, device=dev()) for n in ("logp", "entropy", "lse")}
    top = torch.full((T, H, max(k, 1)), -9, dtype=torch.int32, device=dev())
    top_logp = torch.full((T, H, max(k, 1)), 7.0, device=dev())
    F.token_logprobs(view, stride, T, S, B, V, tok, par, k, out["logp"] if tokens is not None else None, out["entropy"],
                     out["lse"], top if k else None, top_logp if k else None)
    torch.cuda.synchronize()
    res = {n: t.cpu().numpy().astype(np.float64) for n, t in out.items()}
    res.update(top=top.cpu().numpy()[:, :, :k], top_logp=top_logp.cpu().numpy().astype(np.float64)[:, :, :k])
    return res, (view, stride, tok, par, out)


def _near(got, want, tol, what):
    same = np.isnan(want) & np.isnan(got) | (got == want)
    err = np.abs(np.where(same, 0.0, got) - np.where(same, 0.0, want))
    assert np.all(err <= tol), f"{what}: {np.argwhere(~(err <= tol))[:3]} {got[~(err <= tol)][:3]} {want[~(err <= tol)][:3]}"


def _check(x, tokens, parents, S, B, k, **place):
    res, keep = _score(x, tokens, parents, S, B, k, **place)
    ref = O.scores(x.double().numpy(), tokens, parents, S, B, k)
    if tokens is not None:
        _near(res["logp"], ref["logp"], ref["tol_logp"], "logp")
    _near(res["entropy"], ref["entropy"], ref["tol_entropy"], "entropy")
    _near(res["lse"], ref["lse"], ref["tol_lse"], "lse")
    assert np.array_equal(res["top"], ref["top"])
    _near(res["top_logp"], ref["top_logp"], ref["tol_top"], "alternatives")
    return res, keep


def _draw(rng, T, S, B, V, dtype="float32", scale=2.0):
    x = torch.tensor(rng.standard_normal((T, S * B, V)) * scale).to(DTYPES[dtype])
    tok = rng.integers(0, V, (T, S * B))
    tok[rng.random((T, S * B)) < 0.2] = -1
    par = None
    if B > 1:
        par = rng.integers(0, B, (T, S * B))
        par[rng.random((T, S * B)) < 0.15] = -1
    return x, tok, par


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 63, 64, 65, 255, 1000, 1023, 1024, 1025, 2050, 4095, 4096, 4097, 8190, 16385, 33001]


@pytest.mark.gpu
@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_every_width(V, dtype):
    rng = np.random.default_rng(V)
    k = (0, 1, 3, 8)[V % 4]
    x, tok, par = _draw(rng, 2, 3, 1, V, dtype)
    _check(x, tok, par, 3, 1, k)
    x, tok, par = _draw(rng, 2, 2, 3, V, dtype)
    _check(x, tok, par, 2, 3, 8, pad=int(rng.integers(0, 9)), offset=int(rng.integers(0, 8)))


@pytest.mark.gpu
@pytest.mark.parametrize("M,V,dtype", [(1, 130, "float32"), (4100, 1030, "float32"), (4097, 2050, "bfloat16"),
                                       (1030, 4100, "float16"), (1100, 8190, "float32"), (1, 131072, "bfloat16")])
def test_numbers_of_rows(M, V, dtype):
    """Both sides of the rules for how many waves share a row."""
    x, tok, par = _draw(np.random.default_rng(M + V), 1, M, 1, V, dtype)
    _check(x, tok, par, M, 1, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [5, 300, 1024, 3001, 20000])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_masked_and_broken_rows(V, dtype):
    rng = np.random.default_rng(V)
    x, tok, _ = _draw(rng, 1, 14, 1, V, dtype)
    tok[:] = rng.integers(0, V, tok.shape)
    x[0, 0] = -float("inf")
    x[0, 1] = -float("inf")
    x[0, 1, V // 2] = 1.5                       # a single token left
    x[0, 2, rng.random(V) < 0.9] = -float("inf")
    x[0, 3] = LOWEST[dtype]                     # every token masked by the lowest value: uniform
    x[0, 4] = LOWEST[dtype]
    x[0, 4, V - 1] = 2.0
    x[0, 5, V - 1] = float("nan")
    x[0, 6, 0] = float("inf")
    x[0, 7] = float("nan")
    x[0, 8] = -float("inf")
    x[0, 8, 0] = float("nan")
    x[0, 9] = float("inf")
    x[0, 10] = 0.0
    x[0, 11] = 60000.0
    x[0, 12, :V - 1] = -float("inf")            # only the last one
    x[0, 13, V // 2] = 40.0                     # nearly all of the probability
    tok[0, 1], tok[0, 4], tok[0, 13] = V // 2, V - 1, V // 2
    _check(x, tok, None, 14, 1, 8)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 1024, 1500, 9000])
@pytest.mark.parametrize("k", [1, 2, 8])
def test_ties_go_to_the_lowest_id(V, k):
    rng = np.random.default_rng(V + k)
    x = torch.tensor(rng.integers(-2, 3, (1, 12, V)).astype(np.float32))
    x[0, 0] = 1.0                                # all equal
    x[0, 1] = torch.arange(V) * 1e-3             # ascending: the last ones
    x[0, 2] = -torch.arange(V) * 1e-3
    x[0, 3] = -float("inf")
    x[0, 3, V - 3:] = 0.5                        # fewer than k
    x[0, 4, ::2] = -0.0                          # zeros of both signs are equal
    x[0, 4, 1::2] = 0.0
    x[0, 5] = -float("inf")
    x[0, 5, ::5] = 3.0
    tok = rng.integers(0, V, (1, 12))
    _check(x, tok, None, 12, 1, k)
    _check(x.bfloat16(), tok, None, 12, 1, k)


@pytest.mark.gpu
def test_confident_rows_keep_their_relative_accuracy():
    """Where one token holds nearly everything, log p = -log(1 + rest): the rest counts, not 1 + rest."""
    rng = np.random.default_rng(3)
    V, gaps = 1024, np.array([4.0, 8.0, 12.0, 16.0, 20.0, 25.0])
    x = torch.tensor(rng.standard_normal((1, 6, V)).astype(np.float32))
    tok = rng.integers(0, V, (1, 6))
    for i, g in enumerate(gaps):
        x[0, i, tok[0, i]] = x[0, i].max() + g
    res, _ = _check(x, tok, None, 6, 1, 1)
    ref = O.scores(x.double().numpy(), tok, None, 6, 1, 1)
    # the rest's terms: 3 |d| + 2 roundings of each exponential, |d| under 35; V / 64 + 40 additions
    rel = O.U32 * (3 * 35 + 2 + V / 64 + 40 + 8)
    assert np.all(np.abs(res["logp"] - ref["logp"]) <= rel * np.abs(ref["logp"]))
    # entropy: log s and the sum of d e, both of the rest
    assert np.all(np.abs(res["entropy"] - ref["entropy"]) <= 3 * rel * ref["entropy"])


@pytest.mark.gpu
def test_tokens_and_parents_out_of_range():
    rng = np.random.default_rng(4)
    x, _, _ = _draw(rng, 1, 2, 4, 100)
    tok = np.array([[5, 100, -2, -1, 1, 2, 3, 99]])
    par = np.array([[0, 1, 2, 3, 4, -2, -1, 3]])
    F.fusion_device_status()
    res, _ = _score(x, tok, par, 2, 4, 2)
    assert F.fusion_device_status() == F.FUSION_STATUS_BAD_TOKEN
    assert F.fusion_device_status() == 0
    good = np.where((tok < -1) | (tok >= 100), -1, tok)
    live = np.where((par < -1) | (par >= 4), -1, par)
    ref = O.scores(x.double().numpy(), good, live, 2, 4, 2)
    for h in range(8):
        broken = par[0, h] in (4, -2)
        assert np.isnan(res["logp"][0, h]) == (broken or h in (1, 2))
        assert np.isnan(res["lse"][0, h]) == broken == np.isnan(res["entropy"][0, h])
        if not broken:
            assert res["lse"][0, h] == ref["lse"][0, h] or abs(res["lse"][0, h] - ref["lse"][0, h]) <= ref["tol_lse"][0, h]
            assert res["top"][0, h].tolist() == ref["top"][0, h].tolist()
    x, tok, _ = _draw(rng, 1, 3, 1, 50)
    _score(x, None, None, 3, 1, 2)
    assert F.fusion_device_status() == 0


@pytest.mark.gpu
def test_each_output_alone_and_none_of_the_rest():
    rng = np.random.default_rng(5)
    T, S, B, V = 2, 2, 2, 1500
    x, tok, par = _draw(rng, T, S, B, V)
    whole, (view, stride, tok_d, par_d, _) = _score(x, tok, par, S, B, 3)
    for name in ("logp", "entropy", "lse"):
        out = torch.full((T * S * B + 16,), 7.0, device=dev())
        args = {n: out if n == name else None for n in ("logp", "entropy", "lse")}
        F.token_logprobs(view, stride, T, S, B, V, tok_d, par_d, 0, args["logp"], args["entropy"], args["lse"])
        got = out.cpu().numpy()
        assert np.array_equal(got[:T * S * B].reshape(T, -1), whole[name].astype(np.float32)) and (got[T * S * B:] == 7.0).all()
    top = torch.full((T * S * B * 3 + 16,), -9, dtype=torch.int32, device=dev())
    val = torch.full((T * S * B * 3 + 16,), 7.0, device=dev())
    F.token_logprobs(view, stride, T, S, B, V, None, par_d, 3, None, None, None, top, val)
    assert np.array_equal(top.cpu().numpy()[:T * S * B * 3].reshape(T, -1, 3), whole["top"])
    assert (top[T * S * B * 3:] == -9).all() and (val[T * S * B * 3:] == 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1, 3, 8, 9, 130, 1001, 1024, 2049, 4100, 9001])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("mode", ["logp", "entropy", "both"])
def test_gradient(V, dtype, mode):
    rng = np.random.default_rng(V)
    T, S, B = 2, 2, 4
    for use_parents in (False, True):
        x, tok, par = _draw(rng, T, S, B, V, dtype)
        if not use_parents:
            par = None
        else:
            tok[0, 0], tok[0, 1], par[0, 0], par[0, 1] = V // 2, V // 2, 2, 2  # the same token of the same row twice
            par[1, :4] = 1                                                     # rows that nothing extends
        x[0, 5, 0] = 30.0
        x[1, 6] = -float("inf")
        if V > 8:
            x[0, 2, 3:7] = -float("inf")
        gl = rng.standard_normal((T, S * B)).astype(np.float32) if mode != "entropy" else None
        ge = rng.standard_normal((T, S * B)).astype(np.float32) if mode != "logp" else None
        pad, offset, gpad = int(rng.integers(0, 5)), int(rng.integers(0, 8)), int(rng.integers(0, 5))
        _, (view, stride, tok_d, par_d, out) = _score(x, tok, par, S, B, 0, pad=pad, offset=offset)
        buf = torch.full((T, S * B, V + gpad), 7.0, dtype=DTYPES[dtype], device=dev())
        gl_d, ge_d = (None if g is None else torch.tensor(g, device=dev()) for g in (gl, ge))
        F.token_logprobs_backward(view, stride, T, S, B, V, tok_d, par_d, out["logp"], out["entropy"], out["lse"], gl_d,
                                  ge_d, buf, V + gpad)
        want, tol = O.gradient(x.double().numpy(), tok, par, S, B, gl, ge)
        got = buf.cpu().double().numpy()
        assert (got[:, :, V:] == 7.0).all()
        tol = tol + O.half_step(np.abs(want) + tol, dtype)
        _near(got[:, :, :V], want, tol, f"gradient, parents {use_parents}")
        # in place
        F.token_logprobs_backward(view, stride, T, S, B, V, tok_d, par_d, out["logp"], out["entropy"], out["lse"], gl_d,
                                  ge_d, view, stride)
        again = view.cpu().double().numpy()
        assert np.array_equal(again, got[:, :, :V], equal_nan=True)


@pytest.mark.gpu
def test_gradient_of_confident_tokens():
    """1 - p of a token with p near 1 comes from its log probability, not from x - lse."""
    rng = np.random.default_rng(6)
    V = 1024
    x = torch.tensor(rng.standard_normal((1, 5, V)).astype(np.float32))
    tok = rng.integers(0, V, (1, 5))
    for i, g in enumerate([2.0, 6.0, 10.0, 14.0, 18.0]):
        x[0, i, tok[0, i]] = x[0, i].max() + g
    gl = np.ones((1, 5), dtype=np.float32)
    _, (view, stride, tok_d, _, out) = _score(x, tok, None, 5, 1, 0)
    grad = torch.empty((1, 5, V), device=dev())
    F.token_logprobs_backward(view, stride, 1, 5, 1, V, tok_d, None, out["logp"], None, out["lse"],
                              torch.tensor(gl, device=dev()), None, grad, V)
    want, _ = O.gradient(x.double().numpy(), tok, None, 5, 1, gl)
    got = grad.cpu().double().numpy()
    # the own column: relative to itself, as the log probability it comes from (|d| under 30)
    own = np.take_along_axis(np.abs(got - want), tok[:, :, None], 2) / np.take_along_axis(want, tok[:, :, None], 2)
    assert own.max() <= O.U32 * (3 * 30 + V / 64 + 60)


@pytest.mark.gpu
def test_gradient_with_broken_rows_and_bad_tokens():
    rng = np.random.default_rng(7)
    x, tok, _ = _draw(rng, 1, 4, 1, 700)
    tok[0] = [3, 700, -5, 9]
    x[0, 3, 5] = float("nan")
    F.fusion_device_status()
    _, (view, stride, tok_d, _, out) = _score(x, tok, None, 4, 1, 0)
    assert F.fusion_device_status() == F.FUSION_STATUS_BAD_TOKEN
    grad = torch.full((1, 4, 700), 7.0, device=dev())
    one = torch.ones((1, 4), device=dev())
    F.token_logprobs_backward(view, stride, 1, 4, 1, 700, tok_d, None, out["logp"], None, out["lse"], one, None, grad, 700)
    assert F.fusion_device_status() == F.FUSION_STATUS_BAD_TOKEN
    got = grad.cpu()
    assert (got[0, 1:3] == 0).all() and torch.isnan(got[0, 3]).all() and torch.isfinite(got[0, 0]).all()


@pytest.mark.gpu
def test_graph_and_streams():
    """Captured once and replayed on new inputs; eager on a side stream; two streams at once."""
    rng = np.random.default_rng(8)
    T, S, B, V, k = 3, 2, 4, 1500, 4
    H = S * B
    xs = [_draw(rng, T, S, B, V) for _ in range(4)]
    x = torch.empty((T, H, V), device=dev())
    tok = torch.zeros((T, H), dtype=torch.int32, device=dev())
    par = torch.zeros((T, H), dtype=torch.int32, device=dev())
    gl = torch.tensor(rng.standard_normal((T, H)).astype(np.float32), device=dev())

    def buffers():
        return dict(logp=torch.empty((T, H), device=dev()), ent=torch.empty((T, H), device=dev()),
                    lse=torch.empty((T, H), device=dev()), top=torch.empty((T, H, k), dtype=torch.int32, device=dev()),
                    val=torch.empty((T, H, k), device=dev()), grad=torch.empty((T, H, V), device=dev()))

    def both(o):
        F.token_logprobs(x, V, T, S, B, V, tok, par, k, o["logp"], o["ent"], o["lse"], o["top"], o["val"])
        F.token_logprobs_backward(x, V, T, S, B, V, tok, par, o["logp"], o["ent"], o["lse"], gl, gl, o["grad"], V)

    def fill(i):
        x.copy_(xs[i][0])
        tok.copy_(torch.tensor(xs[i][1]))
        par.copy_(torch.tensor(xs[i][2]))

    fill(0)
    graphed, eager, side = buffers(), buffers(), buffers()
    both(graphed)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(graphed)
    for i in (1, 2, 3, 1):
        fill(i)
        g.replay()
        both(eager)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            both(side)
        both(eager)
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(graphed[n], eager[n]) and torch.equal(side[n], eager[n]), (i, n)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Rows behind the first 2^31 elements and 4 GiB of the logits."""
    T, H, V = 3, 2, 1000
    stride = (1 << 29) + 3  # the last two of the six rows begin past element 2^31, the last four past byte 2^31
    buf = torch.empty(5 * stride + V, dtype=torch.bfloat16, device=dev())
    view = torch.as_strided(buf, (T, H, V), (H * stride, stride, 1))
    x, tok, _ = _draw(np.random.default_rng(9), T, H, 1, V, "bfloat16")
    view.copy_(x)
    tok_d = torch.tensor(tok, dtype=torch.int32, device=dev())
    out = {n: torch.empty((T, H), device=dev()) for n in ("logp", "entropy", "lse")}
    F.token_logprobs(view, stride, T, H, 1, V, tok_d, None, 0, out["logp"], out["entropy"], out["lse"])
    ref = O.scores(x.double().numpy(), tok, None, H, 1, 0)
    for n in out:
        _near(out[n].cpu().double().numpy(), ref[n], ref["tol_" + n], n)
    gl = torch.ones((T, H), device=dev())
    F.token_logprobs_backward(view, stride, T, H, 1, V, tok_d, None, out["logp"], None, out["lse"], gl, None, view, stride)
    want, tol = O.gradient(x.double().numpy(), tok, None, H, 1, np.ones((T, H)))
    _near(view.cpu().double().numpy(), want, tol + O.half_step(np.abs(want) + tol, "bfloat16"), "gradient")
