"""Token scoring straight from hidden states (joint_logprobs), and the output
layer's operators together as a recogniser uses them.  GPU checks against float64;
refusals on the CPU."""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

import oracle
import paper_2609_14991_amd as F
from oracle import mx, projection
from oracle import scores as O
from workloads import tiny_random_lm, tiny_random_phrases, to_bf16_bits

torch = pytest.importorskip("torch")

P = ctypes.c_void_p
SOME = P(4096)


def _call(A=SOME, W=SOME, K=64, T=2, S=1, B=2, V=100, tokens=SOME, parents=None, logp=SOME, entropy=None, lse=None, work=SOME,
          floats=1 << 20):
    return F.lib().joint_logprobs(A, W, None, K, T, S, B, V, tokens, parents, logp, entropy, lse, work, floats, None)


@pytest.mark.parametrize("bad,code", [
    (dict(T=-1), "ARG"), (dict(S=-1), "ARG"), (dict(B=0), "ARG"), (dict(V=0), "ARG"), (dict(K=4), "ARG"),
    (dict(K=60), "UNSUPPORTED"), (dict(A=None), "ARG"), (dict(W=None), "ARG"), (dict(work=None), "ARG"), (dict(A=P(4104)), "ARG"),
    (dict(tokens=None), "ARG"), (dict(logp=None), "ARG"), (dict(floats=3), "ARG"), (dict(parents=SOME, B=33), "UNSUPPORTED"),
    (dict(T=1 << 20, S=1 << 10), "UNSUPPORTED"), (dict(S=1 << 30, B=4), "UNSUPPORTED"), (dict(V=1 << 25), "UNSUPPORTED")])
def test_refusals(bad, code):
    assert _call(**bad) == getattr(F, "FUSION_E_" + code) and F.fusion_last_error()


def test_workspace_and_empty_calls():
    assert _call(T=0, A=None, W=None, work=None) == F.FUSION_OK
    for M, V, K in [(1, 1, 8), (256, 4096, 640), (76800, 4096, 640), (1000, 130, 64)]:
        n = F.joint_logprobs_workspace(M, V, K)
        assert 4 * M <= n <= 4 * M * (-(-V // 64))
    assert F.joint_logprobs_workspace(0, 100, 64) == 0
    for bad in [(-1, 10, 64), (1, 0, 64), (1, 10, 60), (1 << 30, 10, 64)]:
        with pytest.raises(F.FusionError):
            F.joint_logprobs_workspace(*bad)


def dev():
    return torch.device("cuda:0")


def _joint(rng, M, V, K, bias=True, scale=2.0):
    A = to_bf16_bits(rng.standard_normal((M, K), dtype=np.float32))
    W = to_bf16_bits(rng.standard_normal((V, K), dtype=np.float32) * np.float32(scale / np.sqrt(K)))
    return A, W, (rng.standard_normal(V).astype(np.float32) if bias else None)


def _up(a, dtype=None):
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a.astype(dtype or a.dtype)).to(dev())


def _run(A, W, bias, T, S, B, tok, par):
    V, K = W.shape
    H = S * B
    out = {n: torch.full((T * H + 16,), 7.0, device=dev()) for n in ("logp", "entropy", "lse")}
    work = torch.full((F.joint_logprobs_workspace(T * H, V, K) + 16,), float("nan"), device=dev())
    F.joint_logprobs(_up(A), _up(W), _up(bias), K, T, S, B, V, _up(tok, np.int32), _up(par, np.int32), out["logp"],
                     out["entropy"], out["lse"], work[:-16])
    torch.cuda.synchronize()
    assert torch.isnan(work[-16:]).all()
    res = {}
    for n, t in out.items():
        assert (t[T * H:] == 7.0).all()
        res[n] = t[:T * H].view(T, H).cpu().double().numpy()
    return res


def _check(A, W, bias, T, S, B, tok, par, frames=None):
    """Logits off by at most d each move lse and a log probability by 2 d and the entropy by 2 d (1 + E|x - m| + H):
    |dH/dx_y| = p_y |log p_y + H|, summed over y at most H + E|log p| = 2 H."""
    got = _run(A, W, bias, T, S, B, tok, par)
    H = S * B
    for t in range(T) if frames is None else frames:
        rows = slice(t * H, (t + 1) * H)
        x = projection.joint_project(A[rows], W, bias)[None]
        d = projection.fp32_error_bound(A[rows], W, bias).max(axis=1)
        own = O.rows_of(None if par is None else par[t:t + 1], 1, S, B)[0]
        d = np.where(own >= 0, d[own], 0.0)
        ref = O.scores(x, None if tok is None else tok[t:t + 1], None if par is None else par[t:t + 1], S, B, 0)
        # the statistics are joined over column tiles too: 64 more additions at most
        more = 64 * O.U32
        for n, grow in (("logp", 2.0), ("lse", 1.0), ("entropy", 2.0 * ref["entropy"][0] + 0.01)):
            want, tol = ref[n][0], ref["tol_" + n][0] * 2 + more * (1 + ref["entropy"][0]) + grow * d * 1.01
            same = got[n][t] == want
            assert np.all(same | (np.abs(np.where(same, 0.0, got[n][t]) - np.where(same, 0.0, want)) <= tol)), (n, t)
    return got


def _decoded(rng, T, S, B, V):
    tok = rng.integers(0, V, (T, S * B))
    tok[rng.random((T, S * B)) < 0.2] = -1
    par = None
    if B > 1:
        par = rng.integers(0, B, (T, S * B))
        par[rng.random((T, S * B)) < 0.15] = -1
    return tok, par


@pytest.mark.gpu
@pytest.mark.parametrize("T,S,B,V,K", [(1, 1, 1, 1, 8), (1, 1, 1, 16, 40), (3, 5, 1, 130, 64), (2, 4, 4, 1001, 136),
                                       (1, 64, 4, 4096, 640), (5, 13, 3, 257, 648), (2, 1, 7, 8190, 72), (1, 3, 1, 33000, 40)])
def test_scores_from_hidden_states(T, S, B, V, K):
    rng = np.random.default_rng(T + S + B + V + K)
    A, W, bias = _joint(rng, T * S * B, V, K)
    tok, par = _decoded(rng, T, S, B, V)
    _check(A, W, bias, T, S, B, tok, par)
    _check(A, W, None, T, S, B, tok, None)


@pytest.mark.gpu
@pytest.mark.parametrize("T,S,B,V,K", [(50, 10, 2, 1030, 200), (2, 700, 3, 1001, 136), (30, 128, 1, 2050, 72),
                                       (150, 55, 4, 2050, 72), (600, 64, 2, 130, 136)])
def test_every_tile_shape(T, S, B, V, K):
    rng = np.random.default_rng(T + V)
    A, W, bias = _joint(rng, T * S * B, V, K)
    tok, par = _decoded(rng, T, S, B, V)
    _check(A, W, bias, T, S, B, tok, par, frames=[0, T // 2, T - 1])


@pytest.mark.gpu
def test_the_token_logit_is_the_one_in_the_statistics():
    """A log probability of a certain token is -log(1 + rest): never above 0, and as exact as the rest."""
    rng = np.random.default_rng(11)
    M, V, K = 200, 900, 640
    A, W, _ = _joint(rng, M, V, K)
    x = projection.joint_project(A, W)
    tok = x.argmax(axis=1)[None]
    bias = np.zeros(V, dtype=np.float32)
    got = _run(A, W, bias, 1, M, 1, tok, None)
    assert (got["logp"] <= 0).all()
    # one token far above the rest: all rows' log probability of it is about -V e^-60 and rounds to -0
    bias[7] = 100.0
    got = _run(A, W, bias, 1, M, 1, np.full((1, M), 7), None)
    assert (got["logp"] <= 0).all() and (got["logp"] > -1e-20).all()


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 700, 4100])
def test_masked_tokens(V):
    """A bias of -inf masks tokens: some, all but one, all; a NaN breaks every row."""
    rng = np.random.default_rng(V)
    M, K = 40, 72
    A, W, bias = _joint(rng, M, V, K)
    tok = rng.integers(0, V, (1, M))
    bias[rng.random(V) < 0.9] = -np.inf
    tok[0, :5] = np.flatnonzero(np.isfinite(bias))[:5] if np.isfinite(bias).sum() >= 5 else 0
    got = _run(A, W, bias, 1, M, 1, tok, None)
    x = projection.joint_project(A, W, bias)[None]
    ref = O.scores(x, tok, None, M, 1, 0)
    d = projection.fp32_error_bound(A, W, np.where(np.isfinite(bias), bias, 0)).max()
    for n in ("logp", "lse", "entropy"):
        same = got[n] == ref[n]
        assert np.all(same | (np.abs(np.where(same, 0, got[n]) - np.where(same, 0, ref[n])) <= 2 * ref["tol_" + n] + 1e-5 + 16 * d)), n
    assert (got["logp"] == -np.inf).any()
    one = np.full(V, -np.inf, dtype=np.float32)
    one[V // 2] = 1.0
    got = _run(A, W, one, 1, M, 1, np.full((1, M), V // 2), None)
    assert (got["logp"] == 0).all() and (got["entropy"] == 0).all() and np.isfinite(got["lse"]).all()
    got = _run(A, W, np.full(V, -np.inf, dtype=np.float32), 1, M, 1, tok, None)
    assert (got["logp"] == -np.inf).all() and (got["lse"] == -np.inf).all() and (got["entropy"] == 0).all()
    one[V - 1] = np.nan
    got = _run(A, W, one, 1, M, 1, tok, None)
    assert all(np.isnan(got[n]).all() for n in got)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 700, 4100])
@pytest.mark.parametrize("low", [float(np.finfo(np.float32).min), -3e38, -1e30])
def test_tokens_masked_by_a_low_value(V, low):
    """As torch.finfo(...).min masks: single tokens, runs that fill whole tiles of columns, the whole vocabulary."""
    rng = np.random.default_rng(V)
    M, K = 40, 72
    A, W, bias = _joint(rng, M, V, K)
    tok = rng.integers(0, V, (1, M))
    for masked in (rng.random(V) < 0.3, np.arange(V) >= V // 4, np.arange(V) < V - 3, np.ones(V, dtype=bool)):
        b = np.where(masked, np.float32(low), bias).astype(np.float32)
        got = _run(A, W, b, 1, M, 1, tok, None)
        # in fp32 a masked logit is the mask: the product is far below its last place
        x = np.where(masked, float(np.float32(low)), projection.joint_project(A, W, np.where(masked, 0, b)))[None]
        ref = O.scores(x, tok, None, M, 1, 0)
        d = projection.fp32_error_bound(A, W, np.where(masked, 0, b)).max()
        for n in ("logp", "lse", "entropy"):
            tol = 2 * ref["tol_" + n] + 1e-5 + 16 * d
            assert np.all(np.abs(got[n] - ref[n]) <= tol), (n, int(masked.sum()))


@pytest.mark.gpu
def test_confident_rows_from_hidden_states():
    """One token far above the rest: -log p is the rest's sum, whose terms' differences the logits' errors bound."""
    rng = np.random.default_rng(14)
    M, V, K = 70, 1000, 128
    A, W, _ = _joint(rng, M, V, K, scale=1.0)
    x = projection.joint_project(A, W)
    for gap in (6.0, 10.0, 16.0):
        bias = np.zeros(V, dtype=np.float32)
        bias[33] = gap + 6.0
        tok = np.full((1, M), 33)
        got = _run(A, W, bias, 1, M, 1, tok, None)
        ref = O.scores(projection.joint_project(A, W, bias)[None], tok, None, M, 1, 0)
        d = projection.fp32_error_bound(A, W, bias).max()
        # each term of the rest off by a factor of e^(2 d), and the sums' roundings (1/16 of a part is held to 1e-5)
        assert np.all(np.abs(got["logp"] - ref["logp"]) <= (2.5 * d + 2e-5) * np.abs(ref["logp"]))
    assert x.shape == (M, V)


@pytest.mark.gpu
def test_bad_tokens_and_missing_outputs():
    rng = np.random.default_rng(12)
    A, W, bias = _joint(rng, 8, 50, 64)
    tok = np.array([[3, 50, -2, -1, 4, 5, 6, 7]])
    par = np.array([[0, 1, 2, 3, 4, -2, -1, 3]])
    F.fusion_device_status()
    got = _run(A, W, bias, 1, 2, 4, tok, par)
    assert F.fusion_device_status() == F.FUSION_STATUS_BAD_TOKEN
    assert np.isnan(got["logp"][0]).tolist() == [False, True, True, False, True, True, False, False]
    assert np.isnan(got["lse"][0]).tolist() == [False] * 4 + [True, True, False, False]
    assert got["lse"][0, 6] == -np.inf and got["entropy"][0, 6] == 0 and got["logp"][0, 6] == 0
    whole = _run(A, W, bias, 1, 8, 1, np.arange(8)[None], None)
    work = torch.empty(F.joint_logprobs_workspace(8, 50, 64), device=dev())
    for n in ("logp", "entropy", "lse"):
        out = torch.empty((1, 8), device=dev())
        a = {m: out if m == n else None for m in ("logp", "entropy", "lse")}
        F.joint_logprobs(_up(A), _up(W), _up(bias), 64, 1, 8, 1, 50, _up(np.arange(8), np.int32) if n == "logp" else None, None,
                         a["logp"], a["entropy"], a["lse"], work)
        assert np.array_equal(out.cpu().double().numpy(), whole[n])


@pytest.mark.gpu
def test_graph_replays():
    rng = np.random.default_rng(13)
    T, S, B, V, K = 2, 10, 4, 700, 128
    H = S * B
    W, bias = _up(_joint(rng, 1, V, K)[1]), _up(_joint(rng, 1, V, K)[2])
    A = torch.empty((T * H, K), dtype=torch.bfloat16, device=dev())
    tok_np, par_np = _decoded(rng, T, S, B, V)
    tok, par = _up(tok_np, np.int32), _up(par_np, np.int32)

    def buffers():
        return [torch.empty((T, H), device=dev()) for _ in range(3)] + [torch.empty(F.joint_logprobs_workspace(T * H, V, K), device=dev())]

    def call(b):
        F.joint_logprobs(A, W, bias, K, T, S, B, V, tok, par, *b)

    a, b = buffers(), buffers()
    A.normal_()
    call(a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(a)
    for i in range(3):
        A.normal_()
        g.replay()
        call(b)
        torch.cuda.synchronize()
        for u, v in zip(a[:3], b[:3]):
            assert torch.equal(u, v), i


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("S,B,k", [(6, 4, 4), (17, 1, 1)])
def test_quantise_project_decode_score_and_train(S, B, k):
    """The output layer held in 4 bits: states quantised, projected, decoded with LM and phrases, the chosen tokens
    scored on the rows they were chosen on, and the scores' gradient taken back to the logits."""
    rng = np.random.default_rng(20 + B)
    T, V, K, H = 9, 700, 320, S * B
    lm, ph = tiny_random_lm(rng, V, 4, n_sent=3000), tiny_random_phrases(rng, V, n=30, max_len=4, alphabet=30)
    glm, gtr = F.ngram_load_arrays(lm), F.boost_build_phrases(V, 0, ph)
    A = torch.tensor(rng.standard_normal((T * H, K))).bfloat16().to(dev())
    W = torch.tensor(rng.standard_normal((V, K)) * 2 / np.sqrt(K)).bfloat16().to(dev())
    bias = torch.zeros(V, device=dev())
    bias[0] = 2.0
    ss = F.mx_scale_stride(K)
    (qa, sa), (qw, sw) = [(torch.empty((R, K // 2), dtype=torch.uint8, device=dev()),
                           torch.empty((R, ss), dtype=torch.uint8, device=dev())) for R in (T * H, V)]
    F.mx_quantize(A, K, T * H, K, qa, sa)
    F.mx_quantize(W, K, V, K, qw, sw)
    logits = torch.empty((T, H, V), device=dev())
    F.joint_project_mx(qa, sa, qw, sw, bias, T * H, V, K, logits)
    ls = torch.full((H,), V, dtype=torch.int32, device=dev())
    bs = torch.zeros((H,), dtype=torch.int32, device=dev())
    sc = torch.from_numpy(np.tile(np.array([0.0] + [-np.inf] * (B - 1)), S)).to(dev()) if B > 1 else None
    mode = F.FUSION_BLANK_COMPETE if B > 1 else F.FUSION_BLANK_AM
    o = F.run(glm, gtr, logits, S, B, k, 0.5, 0.5, 0, mode, ls, bs, sc)
    tok, par = o["tokens"], o["parents"]
    out = {n: torch.empty((T, H), device=dev()) for n in ("logp", "entropy", "lse")}
    top, val = torch.empty((T, H, 3), dtype=torch.int32, device=dev()), torch.empty((T, H, 3), device=dev())
    F.token_logprobs(logits, V, T, S, B, V, tok, par, 3, out["logp"], out["entropy"], out["lse"], top, val)
    gl, ge = torch.ones((T, H), device=dev()), torch.full((T, H), 0.1, device=dev())
    grad = torch.empty_like(logits)
    F.token_logprobs_backward(logits, V, T, S, B, V, tok, par, out["logp"], out["entropy"], out["lse"], gl, ge, grad, V)
    assert F.fusion_device_status() == 0

    # the logits: the exact product of the quantised operands
    aq, wq = mx.quantize(A.cpu().double().numpy()), mx.quantize(W.cpu().double().numpy())
    a, w = mx.values(*aq, K), mx.values(*wq, K)
    x = a @ w.T + bias.cpu().double().numpy()
    got = logits.cpu().double().numpy().reshape(T * H, V)
    assert np.all(np.abs(got - x) <= K * O.U32 * (np.abs(a) @ np.abs(w).T) + O.U32 * np.abs(x) * 2)
    # the decode of these logits, by the oracle
    olm, otr = oracle.OracleLM(lm), oracle.OracleTrie(V, 0, ph)
    xs = logits.cpu().numpy()
    if B == 1:
        want = oracle.run(olm, otr, xs, S, B, k, 0.5, 0.5, 0, 0, [V] * H, [0] * H)
        assert np.array_equal(tok.cpu().numpy(), want["tokens"])
    # the scores and their gradient on these logits
    tn, pn = tok.cpu().numpy(), None if par is None else par.cpu().numpy()
    ref = O.scores(xs.astype(np.float64), tn, pn, S, B, 3)
    for n in out:
        have, same = out[n].cpu().double().numpy(), out[n].cpu().double().numpy() == ref[n]
        assert np.all(same | (np.abs(np.where(same, 0.0, have) - np.where(same, 0.0, ref[n])) <= ref["tol_" + n])), n
    assert np.array_equal(top.cpu().numpy(), ref["top"])
    g, tol = O.gradient(xs.astype(np.float64), tn, pn, S, B, np.ones((T, H)), np.full((T, H), np.float32(0.1)))
    assert np.all(np.abs(grad.cpu().double().numpy() - g) <= tol)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [4, 2])
def test_scores_after_a_projected_decode(k):
    """fusion_run_projected keeps no logits: its tokens scored from the hidden states equal the scores on the logits."""
    rng = np.random.default_rng(31)
    T, S, B, V, K = 11, 5, 4, 600, 256
    H = S * B
    lm = tiny_random_lm(rng, V, 3, n_sent=2000)
    glm = F.ngram_load_arrays(lm)
    A, W, bias = (_up(a) for a in _joint(rng, T * H, V, K))
    ls, bs = torch.full((1, H), V, dtype=torch.int32, device=dev()), torch.zeros((H,), dtype=torch.int32, device=dev())
    sc = torch.from_numpy(np.tile(np.array([0.0] + [-np.inf] * (B - 1)), S)).to(dev())
    tok, par = (torch.empty((T, H), dtype=torch.int32, device=dev()) for _ in range(2))
    chunk = torch.empty((4, H, V), device=dev())
    F.fusion_run_projected([glm], [0.5], None, A, W, bias, K, chunk, 4, T, S, B, V, k, 0.0, 0, F.FUSION_BLANK_COMPETE, ls, bs, sc,
                           tok, par)
    a, b = ([torch.empty((T, H), device=dev()) for _ in range(3)] for _ in range(2))
    F.joint_logprobs(A, W, bias, K, T, S, B, V, tok, par, *a, torch.empty(F.joint_logprobs_workspace(T * H, V, K), device=dev()))
    logits = F.project(A, W, bias).view(T, H, V)
    F.token_logprobs(logits, V, T, S, B, V, tok, par, 0, *b)
    # one live slot proposes k candidates: with 2 the first frame leaves two slots dead
    assert bool((tok.cpu() == -1).any()) == (k < B) and F.fusion_device_status() == 0
    d = 2 * projection.fp32_error_bound(A.cpu().numpy().view(np.uint16), W.cpu().numpy().view(np.uint16), bias.cpu().numpy()).max()
    for u, v in zip(a, b):
        u, v = u.cpu().double(), v.cpu().double()
        live = torch.isfinite(v)
        assert torch.equal(live, torch.isfinite(u))
        # two evaluations of each logit, and 200 roundings of either sum
        assert ((u - v).abs()[live] <= 2 * d * 14 + 400 * O.U32 * 14).all()  # entropy at most log 600 < 7, twice


@pytest.mark.gpu
def test_conveniences_equal_the_calls():
    rng = np.random.default_rng(33)
    T, S, B, V, K, k = 3, 4, 2, 300, 96, 3
    H = S * B
    A, W = torch.tensor(rng.standard_normal((T, H, K))).bfloat16().to(dev()), torch.tensor(rng.standard_normal((V, K)) / 5).bfloat16().to(dev())
    bias = torch.tensor(rng.standard_normal(V), dtype=torch.float32, device=dev())
    tok_np, par_np = _decoded(rng, T, S, B, V)
    tok, par = _up(tok_np, np.int32), _up(par_np, np.int32)
    logits = F.project(A.view(T * H, K), W, bias).view(T, H, V)
    o = F.score(logits, tok, par, B, k)
    raw = [torch.empty((T, H), device=dev()) for _ in range(3)] + [torch.empty((T, H, k), dtype=torch.int32, device=dev()), torch.empty((T, H, k), device=dev())]
    F.token_logprobs(logits, V, T, S, B, V, tok, par, k, *raw)
    for n, r in zip(("logp", "entropy", "lse", "top", "top_logp"), raw):
        assert torch.equal(o[n], r)
    gl = torch.tensor(rng.standard_normal((T, H)), dtype=torch.float32, device=dev())
    grad = F.score_backward(logits, o, tok, par, B, gl, gl)
    wide = torch.zeros((T, H, V + 7), device=dev())
    wide[:, :, :V] = logits
    view = wide[:, :, :V]
    assert torch.equal(F.score(view, tok, par, B)["logp"], o["logp"])
    assert F.score_backward(view, o, tok, par, B, gl, gl, in_place=True) is view
    assert torch.equal(view, grad) and (wide[:, :, V:] == 0).all()
    raw = [torch.empty((T, H), device=dev()) for _ in range(3)]
    F.joint_logprobs(A, W, bias, K, T, S, B, V, tok, par, *raw, torch.empty(F.joint_logprobs_workspace(T * H, V, K), device=dev()))
    p = F.score_projected(A, W, bias, tok, par, B)
    assert all(torch.equal(p[n], r) for n, r in zip(("logp", "entropy", "lse"), raw))
    assert F.score(logits)["logp"] is None and F.score_projected(A, W)["logp"] is None
    q, s = F.quantize(A.view(T * H, K))
    wq = F.quantize(W)
    x = F.project_mx(A.view(T * H, K), wq, bias)
    assert torch.equal(x, F.project_mx((q, s), wq, bias))
    ref = F.dequantize(q, s).double() @ F.dequantize(*wq).double().T + bias.double()
    assert (x.double() - ref).abs().max() <= 2 * K * O.U32 * (ref.abs().max() + K * 36)
    assert F.dequantize(q, s, torch.bfloat16).dtype == torch.bfloat16


def test_conveniences_refuse_what_the_calls_would_misread():
    """CPU tensors, other types, other shapes and orders: refused before anything is launched."""
    x, tok = torch.zeros((2, 4, 8)), torch.zeros((2, 4), dtype=torch.int32)
    for call in (lambda: F.score(x, tok), lambda: F.score_projected(x.bfloat16(), torch.zeros((8, 8), dtype=torch.bfloat16)),
                 lambda: F.quantize(torch.zeros((4, 32))), lambda: F.quantize(torch.zeros((2, 4, 32))), lambda: F.dequantize(torch.zeros((4, 16), dtype=torch.uint8), torch.zeros((4, 8), dtype=torch.uint8)),
                 lambda: F.score_backward(x, dict(logp=None, entropy=None, lse=None), tok, None, 1, torch.zeros((2, 4)))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_conveniences_refuse_other_types_shapes_and_orders():
    x, tok = torch.zeros((2, 4, 8), device=dev()), torch.zeros((2, 4), dtype=torch.int32, device=dev())
    for call in (lambda: F.score(x, tok.long()), lambda: F.score(x, tok[:, :2]), lambda: F.score(x, tok, B=3),
                 lambda: F.score(x.transpose(1, 2)), lambda: F.score(x[:, ::2], tok[:, ::2]), lambda: F.score(x.double()),
                 lambda: F.score(x, tok.t().contiguous().t()), lambda: F.quantize(x.to(torch.int32)),
                 lambda: F.project_mx(F.quantize(torch.zeros((4, 64), device=dev())), F.quantize(torch.zeros((4, 32), device=dev())))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_alternatives_are_the_fusion_steps_without_fusion():
    """With weights 0 the fused step's top-k are the acoustic alternatives, scores and all."""
    rng = np.random.default_rng(32)
    H, V, k = 9, 1100, 8
    glm = F.ngram_load_arrays(tiny_random_lm(rng, V, 3, n_sent=2000))
    x = torch.tensor((rng.standard_normal((H, V)) * 2).astype(np.float32), device=dev())
    state = torch.full((H,), V, dtype=torch.int32, device=dev())
    o = F.step(glm, None, x, state, torch.zeros_like(state), 0.0, 0.0, 0, k, F.FUSION_BLANK_COMPETE)
    top, val = torch.empty((1, H, k), dtype=torch.int32, device=dev()), torch.empty((1, H, k), device=dev())
    F.token_logprobs(x, V, 1, H, 1, V, None, None, k, None, None, None, top, val)
    assert torch.equal(top[0], o["tokens"]) and (val[0] - o["scores"]).abs().max() <= 1e-5
