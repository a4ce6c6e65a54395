"""Performance cases of the operators around the joint network's output layer.

Scoring: the log probabilities of the tokens that a decode chose, with the
entropy and the best alternatives of every row (what a recogniser reports as
word confidence), their gradient with respect to the logits (training of the
joint on decoded hypotheses), and the same log probabilities straight from the
joint's hidden states, for callers that never keep the logits.  Projection in
microscaled 4-bit floating point: quantisation of rows into blocks of 32 values
with a power-of-two scale, and the product of two operands in that format.

``own`` False computes the plain forms with elementary torch operations, True
calls the package.  Logits come in the two kinds of ``perf/cases.py``: "noise"
is N(0, 2) with +2 on blank, "speech" is N(0, 1) with +10 on the frame's token.
"""

from __future__ import annotations

import math

import torch

own = False

BLANK = 0
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # magnitudes of the 4-bit format
MIDDLES = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)   # halfway between neighbours: to the even code

MOST_LOGITS = 300 * 256 * 4096        # elements of the largest scored batch
MOST_PRODUCT = 76800 * 4096 * 640     # multiply-adds of the largest projection
MOST_ROWS = 38421 * 1184              # elements of the largest quantised operand


def listed():
    return [
        # confidence of one token of one stream, the smallest call
        dict(name="score_single", kind="score", T=1, S=1, B=1, V=128, dtype="float32", pad=0, k=4, logits="speech"),
        # one encoder chunk of 64 greedy streams
        dict(name="score_chunk", kind="score", T=13, S=64, B=1, V=1024, dtype="float32", pad=0, k=2, logits="speech"),
        # every decision of a 64 x 4 beam over 300 frames, each token scored on its parent slot's row
        dict(name="score_beam", kind="score", T=300, S=64, B=4, V=4096, dtype="float32", pad=0, k=4, logits="noise"),
        # teacher-forced scoring over a wide, odd vocabulary held in bf16 with padded rows
        dict(name="score_wide", kind="score", T=57, S=9, B=1, V=100003, dtype="bfloat16", pad=29, k=8, logits="noise"),
        # gradient of a small batch of beam hypotheses, an odd sub-word vocabulary
        dict(name="grad_beam", kind="grad", T=25, S=7, B=4, V=1001, dtype="float32", pad=0, entropy=True,
             logits="speech"),
        # gradient of a training batch in bf16, the widest sub-word vocabulary
        dict(name="grad_batch", kind="grad", T=250, S=64, B=1, V=8190, dtype="bfloat16", pad=2, entropy=False,
             logits="noise"),
        # one frame of a 64 x 4 beam scored from its hidden states
        dict(name="joint_frame", kind="joint", T=1, S=64, B=4, V=4096, K=640, bias=True),
        # a whole decode scored from its hidden states: 76,800 hypothesis-frames, logits of 1.26 GB never stored
        dict(name="joint_batch", kind="joint", T=300, S=64, B=4, V=4096, K=640, bias=True),
        # the hidden states of one frame into the 4-bit format and back
        dict(name="mx_rows_frame", kind="mx", R=256, K=640, dtype="bfloat16", pad=0),
        # an fp32 activation batch, rows inside a wider buffer
        dict(name="mx_rows_batch", kind="mx", R=38421, K=1184, dtype="float32", pad=24),
        # projection of one frame with the weight held in 4 bits: the states are quantised in the call
        dict(name="mx_project_frame", kind="mxproject", M=256, N=4096, K=640, bias=True),
        # projection of every frame of a batch
        dict(name="mx_project_batch", kind="mxproject", M=76800, N=4096, K=640, bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["score", "score", "grad", "joint", "mx", "mxproject"])
    if kind in ("score", "grad"):
        B = rng.choice([1, 1, 2, 4, 7, 16])
        V = _log_int(rng, 24, 131072)
        most = MOST_LOGITS // 4 if kind == "score" else 250 * 64 * 8190
        S = max(1, min(_log_int(rng, 1, 128), most // (B * V)))
        T = max(1, min(_log_int(rng, 1, 400), most // (S * B * V)))
        c = dict(kind=kind, T=T, S=S, B=B, V=V, dtype=rng.choice(list(DTYPES)), pad=rng.choice([0, 0, 1, 8, 37]),
                 logits=rng.choice(["noise", "speech"]))
        if kind == "score":
            c.update(k=min(V, rng.choice([0, 1, 2, 4, 5, 8])))
        else:
            c.update(entropy=rng.random() < 0.5)
        return c
    if kind == "joint":
        K, V = 8 * _log_int(rng, 4, 160), _log_int(rng, 24, 16384)
        B, S = rng.choice([1, 2, 4, 8]), _log_int(rng, 1, 64)
        return dict(kind="joint", T=max(1, min(_log_int(rng, 1, 300), MOST_PRODUCT // (S * B * V * K))), S=S, B=B, V=V,
                    K=K, bias=rng.random() < 0.7)
    K = 32 * _log_int(rng, 1, 64)
    if kind == "mx":
        return dict(kind="mx", R=max(1, min(_log_int(rng, 1, 60000), MOST_ROWS // K)), K=K,
                    dtype=rng.choice(list(DTYPES)), pad=rng.choice([0, 0, 8, 5]))
    N = _log_int(rng, 24, 16384)
    return dict(kind="mxproject", M=_log_int(rng, 1, max(1, min(76800, MOST_PRODUCT // (N * K)))), N=N, K=K,
                bias=rng.random() < 0.7)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _decoded(g, T, S, B, V):
    """Tokens [T, S * B] as a decode leaves them and, for a beam, the parents: a stream's slots
    come from any of its slots, and the frame that starts it has a single live one."""
    tok = torch.randint(0, V, (T, S, B), generator=g, device="cuda", dtype=torch.int32)
    tok[torch.rand((T, S, B), generator=g, device="cuda") < 0.4] = BLANK
    if B == 1:
        return tok.view(T, S), None
    par = torch.randint(0, B, (T, S, B), generator=g, device="cuda", dtype=torch.int32)
    par[0] = 0
    par[0, :, B - 1] = -1  # a dead slot: fewer candidates than slots
    tok[0, :, B - 1] = -1
    return tok.view(T, S * B), par.view(T, S * B)


def _logits(g, case, tok):
    """[T, S * B, V] joint outputs of the case's type, rows ``pad`` elements apart beyond V."""
    T, S, B, V = case["T"], case["S"], case["B"], case["V"]
    x = torch.randn((T, S * B, V + case["pad"]), generator=g, device="cuda")
    if case["logits"] == "noise":
        x.mul_(2.0)
        x[:, :, BLANK] += 2.0
    else:
        x.scatter_add_(2, tok.clamp(min=0).long()[:, :, None], torch.full((T, S * B, 1), 10.0, device="cuda"))
    return x.to(DTYPES[case["dtype"]])[:, :, :V]


def _hidden(g, M, N, K, bias):
    A = torch.randn((M, K), generator=g, device="cuda").bfloat16()
    W = (torch.randn((N, K), generator=g, device="cuda") * (2.0 / math.sqrt(K))).bfloat16()
    b = None
    if bias:
        b = 0.1 * torch.randn(N, generator=g, device="cuda")
        b[BLANK] += 2.0
    return A, W, b


def _scale_stride(K):
    return (K // 32 + 7) // 8 * 8


def _pack(code, e):
    """Element codes [R, K] and block exponents [R, K / 32] as the bytes that a weight file holds."""
    R, K = code.shape
    q = (code[:, 0::2] | (code[:, 1::2] << 4)).to(torch.uint8).contiguous()
    s = torch.zeros((R, _scale_stride(K)), device="cuda", dtype=torch.uint8)
    s[:, :K // 32] = (e + 127).to(torch.uint8)
    return q, s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(2609 * seed + 14991)
    st = dict(case=dict(case))
    kind = case["kind"]
    if kind in ("score", "grad"):
        T, H, V = case["T"], case["S"] * case["B"], case["V"]
        tok, par = _decoded(g, T, case["S"], case["B"], V)
        st.update(x=_logits(g, case, tok), tok=tok, par=par)
        st["out"] = {n: torch.empty((T, H), device="cuda") for n in ("logp", "entropy", "lse")}
        if kind == "score":
            k = case["k"]
            st["top"] = (torch.empty((T, H, k), device="cuda", dtype=torch.int32), torch.empty((T, H, k), device="cuda"))
        else:
            st["gl"] = torch.randn((T, H), generator=g, device="cuda") / T
            st["ge"] = 0.01 * torch.rand((T, H), generator=g, device="cuda") if case["entropy"] else None
            st["grad"] = torch.empty((T, H, V), device="cuda", dtype=st["x"].dtype)
    elif kind == "joint":
        T, H, V = case["T"], case["S"] * case["B"], case["V"]
        tok, par = _decoded(g, T, case["S"], case["B"], V)
        A, W, b = _hidden(g, T * H, V, case["K"], case["bias"])
        st.update(A=A, W=W, b=b, tok=tok, par=par)
        st["out"] = {n: torch.empty((T, H), device="cuda") for n in ("logp", "entropy", "lse")}
    elif kind == "mx":
        R, K = case["R"], case["K"]
        x = torch.randn((R, K + case["pad"]), generator=g, device="cuda")
        x *= torch.exp2(torch.randint(-6, 7, (R, 1), generator=g, device="cuda").float())  # rows of unlike magnitude
        x[:, :32] *= torch.rand((R, 1), generator=g, device="cuda") >= 0.02  # some blocks hold nothing
        x = x.to(DTYPES[case["dtype"]])
        st.update(x=x[:, :K], q=torch.empty((R, K // 2), device="cuda", dtype=torch.uint8),
                  s=torch.empty((R, _scale_stride(K)), device="cuda", dtype=torch.uint8),
                  back=torch.empty((R, K), device="cuda"))
    else:
        M, N, K = case["M"], case["N"], case["K"]
        A, W, b = _hidden(g, M, N, K, case["bias"])
        code, e = _quantized(W)  # the weight as it is held, made once when the model is loaded
        wq, ws = _pack(code, e)
        st.update(A=A, wq=wq, ws=ws, b=b, q=torch.empty((M, K // 2), device="cuda", dtype=torch.uint8),
                  s=torch.empty((M, _scale_stride(K)), device="cuda", dtype=torch.uint8),
                  logits=torch.empty((M, N), device="cuda"))
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _quantized(x):
    """Codes [R, K] and exponents [R, K / 32] of the blocks of 32: the block's power of two puts
    its largest magnitude in [4, 8); elements round to the nearest level, halfway to the even code."""
    R, K = x.shape
    v = x.double().reshape(R, K // 32, 32)
    top = v.abs().amax(2)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp_(min=-127)
    m = (v * torch.exp2(-e.double())[:, :, None]).abs()
    mid = torch.tensor(MIDDLES, device=x.device, dtype=torch.float64)
    code = torch.bucketize(m, mid)                       # halfway goes down
    up = (code % 2 == 1) & (m == mid[code.clamp(max=6)])  # but up from an odd code
    code = code + up.long() + 8 * torch.signbit(v)
    return code.reshape(R, K), e


def _values(code, e):
    lev = torch.tensor(LEVELS, device=code.device)
    v = torch.where(code >= 8, -lev[code % 8], lev[code % 8])
    return (v.reshape(e.shape[0], -1, 32) * torch.exp2(e.double())[:, :, None]).float().reshape(code.shape)


def _unpacked(q, s, K):
    code = torch.stack((q & 15, q >> 4), 2).reshape(q.shape[0], K).long()
    return _values(code, s[:, :K // 32].int() - 127)


def _row_of(tok, par, B):
    """Row of each token among a frame's, and whether there is one."""
    T, H = tok.shape
    h = torch.arange(H, device="cuda")
    if par is None:
        return h.expand(T, H), torch.ones((T, H), device="cuda", dtype=torch.bool)
    return h // B * B + par.clamp(min=0), par >= 0


def _stats(x):
    """x - max, log of the sum of its exponentials, lse and entropy of every row.  The largest
    element's 1 is kept out of the sum: where it is nearly all of it, the rest decides."""
    m = x.amax(2, keepdim=True)
    d = x - m
    e = torch.exp(d)
    ones = (d == 0).sum(2, keepdim=True)
    rest = torch.where(d < 0, e, 0.0).sum(2, keepdim=True)
    ls = torch.log1p(rest + (ones - 1))
    return d, ls, (m + ls)[:, :, 0], (ls - (e * d).sum(2, keepdim=True) / (ones + rest))[:, :, 0]


def _scores(x, tok, par, B, d, ls, lse, ent):
    row, live = _row_of(tok, par, B)
    at = torch.arange(x.shape[0], device="cuda")[:, None]
    lp = d[at, row, tok.clamp(min=0).long()] - ls[at, row, 0]
    return (torch.where(live & (tok >= 0), lp, 0.0), torch.where(live, ent[at, row], 0.0),
            torch.where(live, lse[at, row], -math.inf))


def _best(d, ls, row, live, k):
    """The k largest log probabilities of each token's row, ties to the lowest id."""
    T, H, V = d.shape
    left, ids, at = d.clone(), torch.arange(V, device="cuda"), torch.arange(T, device="cuda")[:, None]
    tops, vals = [], []
    for _ in range(k):
        v = left.amax(2, keepdim=True)
        i = torch.where(left == v, ids, V).amin(2, keepdim=True)
        left.scatter_(2, i, -math.inf)
        tops.append(torch.where(live, i[:, :, 0][at, row], -1).int())
        vals.append(torch.where(live, (v - ls)[:, :, 0][at, row], -math.inf))
    if not k:
        return torch.empty((T, H, 0), device="cuda", dtype=torch.int32), torch.empty((T, H, 0), device="cuda")
    return torch.stack(tops, 2), torch.stack(vals, 2)


def _plain_score(st):
    c, x = st["case"], st["x"].float()
    d, ls, lse, ent = _stats(x)
    row, live = _row_of(st["tok"], st["par"], c["B"])
    tops, vals = _best(d, ls, row, live, c["k"])
    return _scores(x, st["tok"], st["par"], c["B"], d, ls, lse, ent) + (tops, vals)


def _plain_grad(st):
    c, x = st["case"], st["x"].float()
    T, H, V = x.shape
    B, S = c["B"], c["S"]
    d, ls, lse, ent = _stats(x)
    logp, entropy, lse_of = _scores(x, st["tok"], st["par"], B, d, ls, lse, ent)
    row, live = _row_of(st["tok"], st["par"], B)
    scored = live & (st["tok"] >= 0)
    # what the tokens of a stream send to each of its rows
    to = (row % B).view(T, S, 1, B) == torch.arange(B, device="cuda")[:, None]
    gl = torch.where(scored, st["gl"], 0.0)
    per = (to * gl.view(T, S, 1, B)).sum(3).view(T, H, 1)
    lp = d - ls
    p = torch.exp(lp)
    grad = -per * p
    if c["entropy"]:
        per = (to * torch.where(live, st["ge"], 0.0).view(T, S, 1, B)).sum(3).view(T, H, 1)
        grad -= per * p * (lp + ent[:, :, None])
    at = (torch.arange(T, device="cuda")[:, None] * H + row) * V + st["tok"].clamp(min=0).long()
    grad.view(-1).scatter_add_(0, at.reshape(-1), gl.reshape(-1))
    return logp, entropy, lse_of, grad.to(st["x"].dtype)


def _plain_joint(st):
    c = st["case"]
    x = st["A"].float() @ st["W"].float().T
    if st["b"] is not None:
        x += st["b"]
    x = x.view(c["T"], c["S"] * c["B"], c["V"])
    return _scores(x, st["tok"], st["par"], c["B"], *_stats(x))


def _plain_mx(st):
    return _values(*_quantized(st["x"]))


def _plain_mx_project(st):
    K = st["case"]["K"]
    x = _values(*_quantized(st["A"])) @ _unpacked(st["wq"], st["ws"], K).T
    return x if st["b"] is None else x + st["b"]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(st):
    c = st["case"]
    kind = c["kind"]
    if not own:
        return {"score": _plain_score, "grad": _plain_grad, "joint": _plain_joint, "mx": _plain_mx,
                "mxproject": _plain_mx_project}[kind](st)
    import paper_2609_14991_amd as F

    if kind in ("score", "grad"):
        o, x, k = st["out"], st["x"], c.get("k", 0)
        T, S, B, V, ld = c["T"], c["S"], c["B"], c["V"], c["V"] + c["pad"]
        tops, vals = st["top"] if k else (None, None)
        F.token_logprobs(x, ld, T, S, B, V, st["tok"], st["par"], k, o["logp"], o["entropy"], o["lse"], tops, vals)
        if kind == "score":
            return (o["logp"], o["entropy"], o["lse"]) + st["top"]
        F.token_logprobs_backward(x, ld, T, S, B, V, st["tok"], st["par"], o["logp"], o["entropy"], o["lse"], st["gl"],
                                  st["ge"], st["grad"], V)
        return o["logp"], o["entropy"], o["lse"], st["grad"]
    if kind == "joint":
        o = st["out"]
        work = torch.empty(F.joint_logprobs_workspace(c["T"] * c["S"] * c["B"], c["V"], c["K"]), device="cuda")
        F.joint_logprobs(st["A"], st["W"], st["b"], c["K"], c["T"], c["S"], c["B"], c["V"], st["tok"], st["par"],
                         o["logp"], o["entropy"], o["lse"], work)
        return o["logp"], o["entropy"], o["lse"]
    if kind == "mx":
        R, K = c["R"], c["K"]
        F.mx_quantize(st["x"], K + c["pad"], R, K, st["q"], st["s"])
        F.mx_dequantize(st["q"], st["s"], R, K, st["back"], K)
        return st["back"]
    M, N, K = c["M"], c["N"], c["K"]
    F.mx_quantize(st["A"], K, M, K, st["q"], st["s"])
    F.joint_project_mx(st["q"], st["s"], st["wq"], st["ws"], st["b"], M, N, K, st["logits"])
    return st["logits"]


def work(case):
    kind = case["kind"]
    if kind in ("score", "grad", "joint"):
        M, V = case["T"] * case["S"] * case["B"], case["V"]
        held = M * (8 if case["B"] > 1 else 4)  # tokens, and parents of a beam
        if kind == "joint":
            K = case["K"]
            return {"bytes": 2 * K * (M + V) + 4 * V * case["bias"] + held + 12 * M, "flops": 2 * M * V * K + 5 * M * V}
        size = 4 if case["dtype"] == "float32" else 2
        if kind == "score":
            return {"bytes": M * V * size + held + M * (12 + 8 * case["k"]), "flops": 5 * M * V}
        # the forward reads the logits, the gradient is written once; a step keeps nothing else of their size
        return {"bytes": 2 * M * V * size + held + 12 * M + 4 * M * (1 + case["entropy"]), "flops": 9 * M * V}
    if kind == "mx":
        n = case["R"] * case["K"]
        size = 4 if case["dtype"] == "float32" else 2
        return {"bytes": n * size + 2 * (n // 2 + n // 32) + 4 * n, "flops": 4 * n}
    M, N, K = case["M"], case["N"], case["K"]
    return {"bytes": 2 * M * K + N * K // 2 + N * K // 32 + 4 * N * case["bias"] + 4 * M * N,
            "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------
# the definitions in float64, frame by frame
# ---------------------------------------------------------------------------
def _exact_rows(x, tok, par, S, B):
    """log softmax of each token's row [H, V] of one frame, and which tokens have one."""
    H = x.shape[0]
    if par is None:
        return torch.log_softmax(x, 1), torch.ones(H, dtype=torch.bool, device="cuda")
    base = torch.arange(S, device="cuda").repeat_interleave(B) * B
    return torch.log_softmax(x, 1)[base + par.long().clamp(min=0)], par >= 0


def _exact_frame(x, tok, par, S, B):
    lp, live = _exact_rows(x, tok, par, S, B)
    has = live & (tok >= 0)
    t = tok.long().clamp(min=0)
    logp = torch.where(has, lp.gather(1, t[:, None])[:, 0], 0.0)
    entropy = torch.where(live, -(lp.exp() * lp.clamp(min=-1e300)).sum(1), 0.0)
    one = torch.zeros((), dtype=torch.float64, device="cuda")
    base = x if par is None else x[torch.arange(S, device="cuda").repeat_interleave(B) * B + par.long().clamp(min=0)]
    lse = torch.where(live, torch.logsumexp(base, 1), one - math.inf)
    return logp, entropy, lse, lp, live, has


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("score", "grad", "joint"):
        T, S, B, V = case["T"], case["S"], case["B"], case["V"]
        H = S * B
        outs = [torch.empty((T, H), dtype=torch.float64, device="cuda") for _ in range(3)]
        vals = torch.empty((T, H, case.get("k", 0)), dtype=torch.float64, device="cuda")
        grad = torch.empty((T, H, V), dtype=torch.float64, device="cuda") if kind == "grad" else None
        for t in range(T):
            tok, par = st["tok"][t], None if st["par"] is None else st["par"][t]
            if kind == "joint":
                x = st["A"][t * H:(t + 1) * H].double() @ st["W"].double().T
                x = x if st["b"] is None else x + st["b"].double()
            else:
                x = st["x"][t].double()
            x.requires_grad_(kind == "grad")
            logp, entropy, lse, lp, live, has = _exact_frame(x, tok, par, S, B)
            for o, v in zip(outs, (logp, entropy, lse)):
                o[t] = v.detach()
            if kind == "grad":
                total = (logp * st["gl"][t].double()).sum()
                if case["entropy"]:
                    total = total + (entropy * st["ge"][t].double()).sum()
                grad[t] = torch.autograd.grad(total, x)[0]
            elif kind == "score" and case["k"]:
                vals[t] = torch.where(live[:, None], torch.topk(lp, case["k"], 1)[0], -math.inf)
        if kind == "score":
            return tuple(outs) + (None, vals)
        return tuple(outs) + ((grad,) if kind == "grad" else ())
    if kind == "mx":
        return _exact_mx(st["x"])
    low, high = (st["wq"] & 15).long(), (st["wq"] >> 4).long()
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device="cuda")
    W = torch.empty((case["N"], case["K"]), dtype=torch.float64, device="cuda")
    W[:, 0::2], W[:, 1::2] = table[low], table[high]
    W *= torch.exp2(st["ws"][:, :case["K"] // 32].double() - 127).repeat_interleave(32, 1)
    x = _exact_mx(st["A"]) @ W.T
    return x if st["b"] is None else x + st["b"].double()


def _exact_mx(x):
    """Each block divided by its power of two and rounded, half to even, to the grid of its magnitude."""
    R, K = x.shape
    v = x.double().reshape(R, K // 32, 32)
    top = v.abs().amax(2, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, 1.0))) - 2)
    m = v / scale
    step = torch.where(m.abs() < 2, 0.5, torch.where(m.abs() < 4, 1.0, 2.0))
    return ((torch.round(m / step) * step).clamp(-6, 6) * scale).reshape(R, K)
