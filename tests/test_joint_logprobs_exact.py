"""Scoring from hidden states on logits that fp32 holds exactly: what is left of an error is the statistics' own."""

from __future__ import annotations

import numpy as np
import pytest

from oracle import projection
from oracle import scores as O
from test_joint_logprobs import _run
from workloads import to_bf16_bits

pytest.importorskip("torch")


def _exact_joint(rng, M, V, K=64):
    """Hidden states of -1, 0 and 1 and weights of whole 64ths: every sum is a whole number of 64ths, at most 31 large."""
    A = rng.integers(-1, 2, (M, K)).astype(np.float32)
    W = np.clip(np.rint(rng.standard_normal((V, K)) * 10), -31, 31).astype(np.float32) / 64
    return to_bf16_bits(A), to_bf16_bits(W)


# The sums of a row's parts are held to 2.4e-5 of all but the largest logit's share (see the kernel), and joining
# and finishing them takes another 40 roundings at most.
REST = 2.4e-5 + 40 * O.U32


@pytest.mark.gpu
@pytest.mark.parametrize("M,V", [(70, 1000), (300, 4100), (3, 40), (60000, 1030)])
@pytest.mark.parametrize("shift", [0.0, 8.0, 100.0, 1000.0, -1000.0, 16000.0])
def test_confident_tokens_under_a_common_shift(M, V, shift):
    """-log p of a token far above the rest, and the entropy, to the accuracy of the rest, however far all logits
    are from 0.  Both are sums of the other logits' shares alone: log(1 + rest) and (sum of d e^-d) / (1 + rest)."""
    rng = np.random.default_rng(M + V)
    A, W = _exact_joint(rng, M, V)
    bias = np.full(V, shift, dtype=np.float32)
    for gap in (3.0, 6.0, 9.0, 14.0):
        b = bias.copy()
        b[33] += np.float32(gap)
        tok = np.full((1, M), 33)
        got = _run(A, W, b, 1, M, 1, tok, None)
        rows = rng.choice(M, min(M, 70), replace=False)
        x = projection.joint_project(A[rows], W, b)
        assert np.array_equal(x, x.astype(np.float32)) and np.array_equal(x * 64, np.rint(x * 64))
        ref = O.scores(x[None], tok[:, rows], None, rows.size, 1, 0)
        first = x.argmax(axis=1) == 33
        logp, H, lse = (got[n][0, rows] for n in ("logp", "entropy", "lse"))
        # (the terms' own roundings: 3 of each difference, which is under 31 + 31 + gap)
        each = O.U32 * 3 * 80
        assert np.all(np.abs(logp - ref["logp"][0])[first] <= (REST + each) * np.abs(ref["logp"][0][first]))
        assert np.all(np.abs(H - ref["entropy"][0]) <= 2 * (REST + each) * ref["entropy"][0] + O.U32 * (~first))
        # a token below the largest: its distance from it once more, a rounding
        assert np.all(np.abs(logp - ref["logp"][0]) <= (REST + each) * (1 + np.abs(ref["logp"][0])))
        assert np.all(np.abs(lse - ref["lse"][0]) <= (REST + each) * (ref["lse"][0] - x.max(axis=1)) + 2 * O.U32 * np.abs(ref["lse"][0]))
        assert (logp <= 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1, 40, 1000])
def test_a_single_large_logit_is_certain(V):
    """Log probability and entropy are 0 (e^-1000 is no fp32), at every magnitude of the logit."""
    rng = np.random.default_rng(V)
    A, W = _exact_joint(rng, 30, V)
    for top in (2.0 ** 12, 2.0 ** 17, 3e6, 2.0 ** 23 + 1, 1e9, 1e20, 3e38):
        b = np.zeros(V, dtype=np.float32)
        b[V // 2] = np.float32(top)
        got = _run(A, W, b, 1, 30, 1, np.full((1, 30), V // 2), None)
        assert (got["logp"] == 0).all() and (np.abs(got["entropy"]) == 0).all(), top


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 1000])
@pytest.mark.parametrize("value", [1e4, -1e6, 3e6, -1e8, 1e9, -1e20])
def test_equal_logits_are_uniform_at_every_magnitude(V, value):
    """A vocabulary masked by one finite value, as a whole: log p = -log V."""
    rng = np.random.default_rng(V)
    A, W = _exact_joint(rng, 30, V)
    got = _run(np.zeros_like(A), W, np.full(V, value, dtype=np.float32), 1, 30, 1, rng.integers(0, V, (1, 30)), None)
    tol = (REST + 8 * O.U32) * np.log(V)
    assert np.all(np.abs(got["logp"] + np.log(V)) <= tol) and np.all(np.abs(got["entropy"] - np.log(V)) <= tol)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1, 3, 40, 127, 129, 1000])
def test_states_that_are_not_finite(V):
    """Rows whose logits all overflow to -infinity, to both infinities or are NaN: as the scores of those logits,
    whatever part of a column tile lies past the vocabulary."""
    rng = np.random.default_rng(V)
    M, K = 8, 64
    A, W = _exact_joint(rng, M, V, K)
    W[:, 5] = to_bf16_bits(np.full(V, -0.5, dtype=np.float32))   # state 5 lowers every logit
    W[:, 6] = to_bf16_bits(np.where(np.arange(V) % 2, 0.5, -0.5).astype(np.float32))
    A[1, 5] = to_bf16_bits(np.array([np.inf], dtype=np.float32))[0]
    A[2, 5] = to_bf16_bits(np.array([-np.inf], dtype=np.float32))[0]
    A[3, 6] = to_bf16_bits(np.array([np.inf], dtype=np.float32))[0]
    A[4, 0] = 0x7FC0                                              # NaN
    tok = rng.integers(0, V, (1, M))
    got = _run(A, W, None, 1, M, 1, tok, None)
    assert got["lse"][0, 1] == -np.inf and got["logp"][0, 1] == -np.inf and got["entropy"][0, 1] == 0
    for r in (2, 4) + ((3,) if V > 1 else ()):
        assert all(np.isnan(got[n][0, r]) for n in got)
    if V == 1:
        assert got["lse"][0, 3] == -np.inf
    assert all(np.isfinite(got[n][0, [0, 5, 6, 7]]).all() for n in got)
