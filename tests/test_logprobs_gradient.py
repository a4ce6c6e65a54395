"""The gradient of token scoring where a row's log sum exp is large against its differences: large logits, and rows
masked as a whole by a finite value.  p is held to the accuracy of the differences."""

from __future__ import annotations

import numpy as np
import pytest

import paper_2609_14991_amd as F
from oracle import scores as O
from test_logprobs import DTYPES, LOWEST, _near, _score, dev

torch = pytest.importorskip("torch")


def _bound(x, tok, par, S, B, gl, ge):
    """Gradient and error bound with p from the token's own log probability L of its row (the likeliest of them): the
    errors of L, two roundings of it (or two of an lse of less than 4 L), one of x - lse, those of the exponentials and
    the products."""
    T, H, V = x.shape
    row = O.rows_of(par, T, S, B)
    ref = O.scores(x, tok, par, S, B, 0)
    want, rounded_lse = O.gradient(x, tok, par, S, B, gl, ge)
    tol = np.zeros_like(want)
    for t in range(T):
        for r in range(H):
            kids = [h for h in range(H) if row[t, h] == r]
            told = [h for h in kids if tok[t, h] >= 0]
            if not told:  # nothing tells what lse left out
                tol[t, r] = rounded_lse[t, r]
                continue
            q = O.row_stats(x[t, r])
            if q["bad"] or q["empty"]:
                continue
            best = max(told, key=lambda h: ref["logp"][t, h])
            L, err = abs(ref["logp"][t, best]), ref["tol_logp"][t, best]
            lp = x[t, r] - q["m"] - q["ls"]
            p = q["p"]
            e = err + O.U32 * (8 * L + 4 * np.abs(lp) + 16 + B)
            for h in kids:
                a = abs(float(gl[t, h])) if gl is not None and tok[t, h] >= 0 else 0.0
                b = abs(float(ge[t, h])) if ge is not None else 0.0
                tol[t, r] += (a + b * (np.abs(lp) + q["H"] + 1)) * p * e + b * p * (ref["tol_entropy"][t, h] + e)
                tol[t, r] += len(kids) * O.U32 * (a + b) * p + 2.0 ** -126 * (a + 200 * b)
                if tok[t, h] >= 0:
                    y = tok[t, h]
                    tol[t, r, y] += a * (ref["tol_logp"][t, h] + 8 * O.U32 * (1 - p[y]) + 2 * len(kids) * O.U32)
    return want, tol


def _check(x, tok, par, S, B, gl, ge):
    """Not in place and in place, and from the entropy's gradient alone where there is one."""
    dtype = {t: n for n, t in DTYPES.items()}[x.dtype]
    T, H, V = x.shape
    xs = x.double().numpy()
    _, (view, stride, tok_d, par_d, out) = _score(x, tok, par, S, B, 0)
    up = lambda g: None if g is None else torch.tensor(g, device=dev())  # noqa: E731
    for a, b in {(True, ge is not None), (False, True) if ge is not None else (True, False)}:
        want, tol = _bound(xs, tok, par, S, B, gl if a else None, ge if b else None)
        tol = tol + O.half_step(np.abs(want) + tol, dtype)
        args = (view, stride, T, S, B, V, tok_d, par_d, out["logp"], out["entropy"], out["lse"], up(gl) if a else None,
                up(ge) if b else None)
        grad = torch.full((T, H, V), 7.0, dtype=x.dtype, device=dev())
        F.token_logprobs_backward(*args, grad, V)
        _near(grad.cpu().double().numpy(), want, tol, (a, b))
        over = view.clone()
        F.token_logprobs_backward(over, V, *args[2:], over, V)
        assert torch.equal(over, grad)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1, 7, 130, 1500, 9001])
@pytest.mark.parametrize("shift,step", [(0.0, 0.25), (100.0, 0.25), (12000.0, 0.25), (-12000.0, 0.25), (1.5e6, 1.0), (2.5e7, 2.0),
                                        (-2.5e7, 2.0)])
def test_gradient_under_a_common_shift(V, shift, step):
    """Logits that fp32 holds exactly at every shift, so that the gradient is the unshifted one's."""
    rng = np.random.default_rng(V)
    T, S, B = 2, 2, 3
    x = np.clip(np.rint(rng.standard_normal((T, S * B, V)) * 2 / step), -20, 20) * step
    xs = torch.tensor(x + shift).float()
    assert np.array_equal(xs.double().numpy() - shift, x)
    tok = np.where(rng.random((T, S * B)) < 0.5, x.argmax(axis=2), rng.integers(0, V, (T, S * B)))
    tok[1, 4] = -1
    par = rng.integers(0, B, (T, S * B))
    par[0, 1] = -1
    gl, ge = (rng.standard_normal((T, S * B)).astype(np.float32) for _ in range(2))
    _check(xs, tok, None, S, B, gl, ge)
    _check(xs, tok, par, S, B, gl, ge)
    _check(xs, tok, par, S, B, gl, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [1, 8, 33, 1024, 5000])
def test_gradient_of_rows_masked_as_a_whole(V, dtype):
    """Every token masked by one finite value: p = 1 / V, not 1."""
    rng = np.random.default_rng(V)
    values = [LOWEST[dtype], -30000.0, 60000.0, -1e4] + ([-1e9, 2.5e7, -1e20] if dtype != "float16" else [])
    x = torch.tensor(values)[None, :, None].expand(1, len(values), V).to(DTYPES[dtype]).contiguous()
    tok = rng.integers(0, V, (1, len(values)))
    gl, ge = (rng.standard_normal((1, len(values))).astype(np.float32) for _ in range(2))
    _check(x, tok, None, len(values), 1, gl, ge)
    _check(x, tok, None, len(values), 1, gl, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_gradient_of_large_logits_of_16_bits(dtype):
    rng = np.random.default_rng(3)
    V = 2050
    x = torch.tensor(rng.standard_normal((1, 8, V)) * 4 + 3000.0).to(DTYPES[dtype])
    tok = x.double().numpy().argmax(axis=2)
    tok[0, 1::2] = rng.integers(0, V, 4)
    gl, ge = (rng.standard_normal((1, 8)).astype(np.float32) for _ in range(2))
    _check(x, tok, None, 8, 1, gl, ge)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [1, 5, 1024, 5000])
def test_entropy_gradient_without_tokens(V, dtype):
    """Where no token tells what the rounding of lse left out: rows of large logits and rows masked as a whole, whose
    entropy's gradient is 0 (p is uniform), in place and not; and rows whose only slot chose no token."""
    rng = np.random.default_rng(V)
    values = [LOWEST[dtype], -30000.0, 60000.0, 0.0] + ([-1e9, 2.5e7] if dtype != "float16" else [])
    n = len(values) + 2
    x = torch.tensor(values + [9000.0, -9000.0])[None, :, None].expand(1, n, V).clone()
    x[0, -2:] += torch.tensor(np.rint(rng.standard_normal((2, V)) * 2).astype(np.float32)) * 8
    x = x.to(DTYPES[dtype])
    xs = x.double().numpy()
    ge = rng.standard_normal((1, n)).astype(np.float32)
    none = np.full((1, n), -1)
    for tok in (None, none):
        _, (view, stride, tok_d, _, out) = _score(x, tok, None, n, 1, 0)
        want, _ = O.gradient(xs, None, None, n, 1, None, ge)
        ref = O.scores(xs, None, None, n, 1, 0)
        tol = np.zeros_like(want)
        for r in range(n):
            q = O.row_stats(xs[0, r])
            lp = np.abs(xs[0, r] - q["m"] - q["ls"])
            # log s read twice, its error and the difference's; below 4096 lse's own rounding
            e = ref["tol_lse"][0, r] - 2 * O.U32 * abs(q["lse"]) + O.U32 * (4 * lp + 4 * q["ls"] + 20)
            e = e + (O.U32 * abs(q["lse"]) if abs(q["lse"]) < 4096 else 0.0)
            tol[0, r] = abs(ge[0, r]) * q["p"] * ((lp + q["H"] + 1) * e + ref["tol_entropy"][0, r] + e) + 2.0 ** -126 * 200
        tol = tol + O.half_step(np.abs(want) + tol, dtype)
        args = (view, stride, 1, n, 1, V, tok_d, None, out["logp"] if tok is not None else None, out["entropy"], out["lse"], None,
                torch.tensor(ge, device=dev()))
        grad = torch.full((1, n, V), 7.0, dtype=x.dtype, device=dev())
        F.token_logprobs_backward(*args, grad, V)
        _near(grad.cpu().double().numpy(), want, tol, "apart")
        over = view.clone()
        F.token_logprobs_backward(over, V, *args[2:], over, V)
        assert torch.equal(over, grad)


@pytest.mark.gpu
def test_a_bad_token_of_a_dead_slot_is_told_of():
    """As by the scores themselves; the gradient is that of the live slots."""
    rng = np.random.default_rng(4)
    x = torch.tensor(rng.standard_normal((1, 4, 60)).astype(np.float32))
    tok, par = np.array([[3, 60, 5, -1]]), np.array([[0, -1, 2, -1]])
    F.fusion_device_status()
    _, (view, stride, tok_d, par_d, out) = _score(x, tok, par, 1, 4, 0)
    assert F.fusion_device_status() == F.FUSION_STATUS_BAD_TOKEN
    grad, one = torch.empty((1, 4, 60), device=dev()), torch.ones((1, 4), device=dev())
    args = (view, stride, 1, 1, 4, 60, tok_d, par_d, out["logp"], out["entropy"], out["lse"])
    for gl, ge in ((one, None), (one, one), (None, one)):
        F.token_logprobs_backward(*args, gl, ge, grad, 60)
        assert F.fusion_device_status() == F.FUSION_STATUS_BAD_TOKEN
        assert (grad[0, [1, 3]] == 0).all() and torch.isfinite(grad).all() and (grad[0, [0, 2]] != 0).any()
    # without tokens to look at there is nothing to tell of
    F.token_logprobs_backward(view, stride, 1, 1, 4, 60, None, par_d, None, out["entropy"], out["lse"], None, one, grad, 60)
    assert F.fusion_device_status() == 0
