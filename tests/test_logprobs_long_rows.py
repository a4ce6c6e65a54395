"""Token scoring and its gradient over rows of several chunks a wave: alternatives whose candidate list is cut on the
way, and gradients of batches whose waves go from chunk to chunk."""

from __future__ import annotations

import numpy as np
import pytest

import paper_2609_14991_amd as F
from oracle import scores as O
from test_logprobs import DTYPES, _near, _score, dev
from test_logprobs_gradient import _bound

torch = pytest.importorskip("torch")

CHUNK = 1024


def _waves(M, V):
    """Waves a row: the rule of token_logprobs."""
    if M >= 4096 or (M >= 2048 and V <= 4 * CHUNK) or V <= CHUNK:
        return 1
    if M >= 1024 or V <= 4 * CHUNK:
        return 4
    return 8 if M >= 256 or V <= 8 * CHUNK else 16


def _cuts(M, V, k):
    """Whether a wave cuts its candidate list before its row's end."""
    W = _waves(M, V)
    return W <= 8 and k > 4 and V >= 8 * W * CHUNK - CHUNK // 2


def _parts(M, V):
    """Waves a row of the gradient, and chunks of a row."""
    chunks = -(-V // CHUNK)
    return min(chunks, max(1, 65536 // M)), chunks


LONG = [(300, 66000, "bfloat16", 8, 1), (260, 70001, "float32", 5, 4), (1030, 33000, "float32", 8, 1),
        (1100, 32257, "float16", 6, 2), (4100, 8190, "float32", 8, 1), (4200, 7681, "bfloat16", 7, 4)]
GRADS = [(9000, 8190, "bfloat16"), (33000, 2050, "float32"), (7000, 9999, "float16"), (66000, 1025, "bfloat16")]


def test_the_rules_are_met():
    assert all(_cuts(M, V, k) for M, V, _, k, _ in LONG) and {_waves(M, V) for M, V, *_ in LONG} == {1, 4, 8}
    assert all(p < c for p, c in (_parts(M, V) for M, V, _ in GRADS))


def _rows(rng, M, V):
    """Rows of noise, of climbs that bring a chunk 10 to 100 candidates, of ties, of falls and of few live tokens."""
    x = rng.standard_normal((M, V), dtype=np.float32)
    col = np.arange(V, dtype=np.float32)
    for r in range(M):
        kind = r % 8
        if kind == 1:
            every = int(rng.integers(10, 100))
            x[r, r % every::every] = 8 + col[r % every::every] * np.float32(20.0 / V)   # climbs, in fp32 without ties
        elif kind == 2:
            x[r] = np.rint(x[r])                                                           # long ties, the largest at any place
        elif kind == 3:
            every = int(rng.integers(10, 40))
            x[r, ::every] = 6 + np.floor(col[::every] * np.float32(16.0 / V))            # climbs in steps: ties across the floor
        elif kind == 4:
            x[r] = -col * np.float32(10.0 / V)
        elif kind == 5:
            x[r, rng.random(V) < 0.999] = -np.inf
        elif kind == 6:
            x[r, : V - V // 5] -= 9
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("M,V,dtype,k,B", LONG)
def test_alternatives_of_long_rows(M, V, dtype, k, B):
    rng = np.random.default_rng(M + V)
    # (the rows are decided on the GPU all at once, by their number; the oracle sees a part of the streams)
    S = M // B
    x = torch.tensor(_rows(rng, S * B, V)).to(DTYPES[dtype])
    tok = rng.integers(0, V, (1, S * B))
    par = rng.integers(0, B, (1, S * B)) if B > 1 else None
    res, _ = _score(x[None], tok, par, S, B, k)
    for first in range(0, 48, 24):
        pick = slice((S // 48 * first) * B, (S // 48 * first) * B + 24 * max(B, 1))
        n = pick.stop - pick.start
        ref = O.scores(x[pick].double().numpy()[None], tok[:, pick], None if par is None else par[:, pick], n // B, B, k)
        for name, tol in (("logp", "tol_logp"), ("entropy", "tol_entropy"), ("lse", "tol_lse"), ("top_logp", "tol_top")):
            _near(res[name][:, pick], ref[name], ref[tol], name)
        assert np.array_equal(res["top"][:, pick], ref["top"])


@pytest.mark.gpu
@pytest.mark.parametrize("M,V,dtype", GRADS)
@pytest.mark.parametrize("B", [1, 4])
def test_gradient_of_waves_of_several_chunks(M, V, dtype, B):
    rng = np.random.default_rng(M + B)
    S = M // B
    M = S * B
    g = torch.Generator().manual_seed(M)
    x = (torch.randn((1, M, V), generator=g) * 2).to(DTYPES[dtype])
    # tokens at the ends of the row and of its chunks, and anywhere
    ends = np.array([0, CHUNK - 1, CHUNK, V - 1, (V - 1) // CHUNK * CHUNK, max(0, V // 2)])
    tok = np.where(rng.random((1, M)) < 0.7, rng.choice(ends, (1, M)), rng.integers(0, V, (1, M)))
    tok[rng.random((1, M)) < 0.1] = -1
    par = None
    if B > 1:
        par = rng.integers(0, B, (1, M))
        par[rng.random((1, M)) < 0.1] = -1
    gl, ge = (rng.standard_normal((1, M)).astype(np.float32) for _ in range(2))
    _, (view, stride, tok_d, par_d, out) = _score(x, tok, par, S, B, 0)
    gl_d, ge_d = torch.tensor(gl, device=dev()), torch.tensor(ge, device=dev())
    streams = np.unique(np.concatenate([[0, S - 1], rng.choice(S, 24 // B)]))
    pick = (streams[:, None] * B + np.arange(B)).reshape(-1)
    grad = torch.empty((1, M, V), dtype=x.dtype, device=dev())
    for a, b in ((True, False), (True, True)):
        args = (view, stride, 1, S, B, V, tok_d, par_d, out["logp"], out["entropy"], out["lse"], gl_d if a else None, ge_d if b else None)
        grad.fill_(7.0)
        F.token_logprobs_backward(*args, grad, V)
        want, tol = _bound(x[:, pick].double().numpy(), tok[:, pick], None if par is None else par[:, pick], streams.size, B, gl[:, pick],
                           ge[:, pick] if b else None)
        tol = tol + O.half_step(np.abs(want) + tol, dtype)
        _near(grad[:, torch.tensor(pick)].cpu().double().numpy(), want, tol, (a, b))
    # in place, over the whole batch
    F.token_logprobs_backward(*args, view, stride)
    assert torch.equal(view, grad)
