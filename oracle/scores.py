"""Oracle of token scoring and its gradient (test infrastructure only).

TEST INFRASTRUCTURE ONLY: used by the tests; the product path never imports it.

Per token (slot h of frame t), x the logits row it was chosen on, in float64:
log softmax of x at the token, the entropy -sum p log p, log sum exp, the k
largest log probabilities (ties to the lowest id), and the gradient of
sum(g_logp * logp) + sum(g_entropy * entropy) with respect to the logits.
"""

from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24


def rows_of(parents, T, S, B):
    """[T, H] row of each token among its frame's, -1 for a dead slot."""
    H = S * B
    own = np.broadcast_to(np.arange(H), (T, H))
    if parents is None:
        return own.copy()
    par = np.asarray(parents).reshape(T, H)
    return np.where(par < 0, -1, own // B * B + par)


def row_stats(x):
    """m, lse, entropy, E|x - m|, E(x - m)^2 of one row, and whether it is empty or bad."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or np.isposinf(x).any():
        return dict(m=np.nan, lse=np.nan, H=np.nan, d1=0.0, d2=0.0, empty=False, bad=True, p=np.full(x.shape, np.nan))
    m = x.max()
    if m == -np.inf:
        return dict(m=m, lse=m, H=0.0, d1=0.0, d2=0.0, empty=True, bad=False, p=np.zeros(x.shape))
    d = x - m
    e = np.exp(d)
    s = e.sum()
    z = np.where(np.isneginf(d), 0.0, d)
    # log s from the sum without one of the maxima: exact where that one holds nearly everything
    ls = np.log1p(np.delete(e, int(np.argmax(x))).sum())
    return dict(m=m, ls=ls, lse=m + ls, H=ls - (z * e).sum() / s, d1=-(z * e).sum() / s, d2=(z * z * e).sum() / s, empty=False,
                bad=False, p=e / s)


def scores(x, tokens, parents, S, B, k):
    """logits [T, H, V] float64 -> logp, entropy, lse [T, H], top tokens and log probabilities
    [T, H, k], and the error bounds of an fp32 evaluation, tol_logp, tol_entropy, tol_lse, tol_top."""
    x = np.asarray(x, dtype=np.float64)
    T, H, V = x.shape
    row = rows_of(parents, T, S, B)
    o = {n: np.zeros((T, H)) for n in ("logp", "entropy", "lse", "tol_logp", "tol_entropy", "tol_lse")}
    o["top"] = np.full((T, H, k), -1, dtype=np.int64)
    o["top_logp"] = np.full((T, H, k), -np.inf)
    o["tol_top"] = np.zeros((T, H, k))
    seen = {}
    # roundings of a row's sum: V / 64 values a lane one after the other, a few joins, the
    # wave's and the workgroup's reduction
    adds = V / 64 + 40
    for t in range(T):
        for h in range(H):
            r = int(row[t, h])
            if r < 0:
                o["lse"][t, h] = -np.inf
                continue
            if (t, r) not in seen:
                q = row_stats(x[t, r])
                if k and not q["bad"]:
                    best = np.argsort(-x[t, r], kind="stable")[:k]
                    q["best"] = best[x[t, r][best] > -np.inf]
                seen[(t, r)] = q
            q = seen[(t, r)]
            o["entropy"][t, h], o["lse"][t, h] = q["H"], q["lse"]
            tok = -1 if tokens is None else int(tokens[t, h])
            if q["bad"]:
                o["logp"][t, h] = np.nan if tok >= 0 else 0.0
                o["top_logp"][t, h] = np.nan
                continue
            if q["empty"]:
                o["logp"][t, h] = -np.inf if tok >= 0 else 0.0
                continue
            # relative error of the sum of exponentials: the argument's two roundings and its
            # difference's (3 |d|), the hardware's exponential (2), the additions; all but
            # the first of the share of the sum that is not the maximum itself
            part = -np.expm1(-q["ls"])  # (s - 1) / s
            tol_s = U32 * (3 * q["d1"] + (2 + adds) * part)
            tol_ls = tol_s + 4 * U32 * q["ls"]
            if tok >= 0:
                d = x[t, r, tok] - q["m"]
                o["logp"][t, h] = d - q["ls"]
                o["tol_logp"][t, h] = 0.0 if d == -np.inf else tol_ls + 2 * U32 * (abs(d) + abs(d - q["ls"]))
            o["tol_lse"][t, h] = tol_ls + 2 * U32 * abs(q["lse"])
            # sum of (x - m) e^(x - m): each product's own roundings, 3 d^2 more from the exponent
            o["tol_entropy"][t, h] = (tol_ls + U32 * ((adds + 6) * q["d1"] + 3 * q["d2"]) + tol_s * q["d1"]
                                      + 4 * U32 * q["H"])
            n = len(q.get("best", ()))
            for i in range(n):
                y = int(q["best"][i])
                d = x[t, r, y] - q["m"]
                o["top"][t, h, i] = y
                o["top_logp"][t, h, i] = d - q["ls"]
                o["tol_top"][t, h, i] = tol_ls + 2 * U32 * (abs(d) + abs(d - q["ls"]))
    return o


def gradient(x, tokens, parents, S, B, g_logp=None, g_entropy=None):
    """grad [T, H, V] float64 and the error bound of an fp32 evaluation from rounded lse, logp and entropy."""
    x = np.asarray(x, dtype=np.float64)
    T, H, V = x.shape
    row = rows_of(parents, T, S, B)
    grad, tol = np.zeros((T, H, V)), np.zeros((T, H, V))
    ref = scores(x, tokens, parents, S, B, 0)
    for t in range(T):
        for r in range(H):
            kids = [h for h in range(H) if row[t, h] == r]
            if not kids:
                continue
            q = row_stats(x[t, r])
            if q["bad"]:
                grad[t, r] = np.nan
                continue
            if q["empty"]:
                continue
            p = q["p"]
            lp = np.where(np.isneginf(x[t, r]), 0.0, x[t, r] - q["m"] - q["ls"])
            for h in kids:
                tok = -1 if tokens is None else int(tokens[t, h])
                gl = float(g_logp[t, h]) if g_logp is not None and tok >= 0 else 0.0
                ge = float(g_entropy[t, h]) if g_entropy is not None else 0.0
                one = np.zeros(V)
                if tok >= 0:
                    one[tok] = 1.0
                # 1 - p from what the other tokens hold
                away = np.where(one > 0, p.sum() - p, -p)
                if tok >= 0:
                    away[tok] = -np.expm1(lp[tok]) if np.isfinite(x[t, r, tok]) else 1.0
                grad[t, r] += gl * away - ge * p * (lp + q["H"])
                # p: lse's error and rounding, the difference's, the exponential's
                rel = ref["tol_lse"][t, h] + U32 * (4 * np.abs(lp) + 12 + B)
                size = p * (abs(gl) + abs(ge) * (np.abs(lp) + q["H"] + 1.0))
                # (what lies below fp32's normal range may be flushed: 2^-126)
                tol[t, r] += size * rel + 2.0 ** -126 * (abs(gl) + abs(ge) * 200) + abs(ge) * p * (ref["tol_entropy"][t, h] + ref["tol_lse"][t, h]
                                                         + 4 * U32 * (np.abs(lp) + q["H"]))
                if tok >= 0:
                    tol[t, r, tok] += abs(gl) * (ref["tol_logp"][t, h] + 8 * U32 * (1 - p[tok]))
                    # sums of several tokens' gradients: one rounding each of the larger
                    tol[t, r] += len(kids) * U32 * abs(gl) * (p if len(kids) > 1 else 0.0)
                    if len(kids) > 1:
                        tol[t, r, tok] += len(kids) * 2 * U32 * abs(gl)
    return grad, tol


def half_step(g, kind):
    """Largest rounding of g into a 16-bit type: half a unit in the last place, of the smallest normal below it."""
    if kind == "float32":
        return np.zeros_like(g)
    eps, tiny = (2.0 ** -7, 2.0 ** -126) if kind == "bfloat16" else (2.0 ** -10, 2.0 ** -14)
    return eps / 2 * np.maximum(np.abs(g), tiny)
