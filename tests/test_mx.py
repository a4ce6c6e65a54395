"""Rows in microscaled 4-bit floating point (mx_quantize, mx_dequantize) and their
product (joint_project_mx): the oracle pinned on the CPU, the kernels against it
on the GPU.  Quantisation is exact; a product's outputs lie within the bound of
any fp32 sum of its exact products."""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

import paper_2609_14991_amd as F
from oracle import mx as O

torch = pytest.importorskip("torch")

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
U32 = 2.0 ** -24


# ---------------------------------------------------------------------------
# the oracle (CPU)
# ---------------------------------------------------------------------------
def test_oracle_rounds_as_the_format_says():
    x = np.zeros((1, 32))
    x[0, :20] = [6.0, 0.25, 0.250001, 0.75, 0.7499, 1.25, 1.75, 2.5, 2.50001, 3.5, 3.4999, 5.0, 5.0001, 7.9, -0.75, -5.0,
                 -0.0, 0.1, 4.0, -1.0]
    q, s = O.quantize(x)
    got = O.values(q, s, 32)[0, :20]
    assert s[0, 0] == 127
    assert got.tolist() == [6.0, 0.0, 0.5, 1.0, 0.5, 1.0, 2.0, 2.0, 3.0, 4.0, 3.0, 4.0, 6.0, 6.0, -1.0, -4.0, 0.0, 0.0, 4.0,
                            -1.0]
    assert q[0, 0] & 15 == 7 and q[0, 0] >> 4 == 0 and q[0, 8] & 15 == 8  # 6.0 in the low half; -0.0 keeps its sign


def test_oracle_scales():
    for top, e in [(4.0, 0), (7.99, 0), (8.0, 1), (1.0, -2), (3.4028234663852886e38, 125), (2.0 ** -149, -127), (0.0, -127),
                   (2.0 ** -125, -127), (2.0 ** -124, -126)]:
        x = np.zeros((2, 64))
        x[1, 33] = -top
        assert O.quantize(x)[1][1, 1] == e + 127, top
    x[0, 3], x[1, 40] = np.nan, -np.inf
    q, s = O.quantize(x)
    assert s.shape == (2, 8) and s[0].tolist() == [255] + [0] * 7 and s[1, 1] == 255 and not q[0].any()
    assert np.isnan(O.values(q, s, 64)[0, :32]).all() and (O.values(q, s, 64)[0, 32:] == 0).all()


# ---------------------------------------------------------------------------
# refusals (CPU): nothing is launched
# ---------------------------------------------------------------------------
P = ctypes.c_void_p
SOME = P(4096)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=5), "ARG"), (dict(R=-1), "ARG"), (dict(K=0), "ARG"), (dict(K=48, stride=48), "UNSUPPORTED"),
    (dict(stride=63), "ARG"), (dict(stride=1 << 62), "ARG"), (dict(x=None), "ARG"), (dict(q=None), "ARG"),
    (dict(s=None), "ARG"), (dict(x=P(4098)), "ARG"), (dict(x=P(4097), dtype=1), "ARG"), (dict(q=P(4104)), "ARG"),
    (dict(s=P(4100)), "ARG"), (dict(R=1 << 30, K=1024, stride=1024), "UNSUPPORTED")])
def test_refusals_of_rows(bad, code):
    a = dict(x=SOME, dtype=0, stride=64, R=2, K=64, q=SOME, s=SOME)
    a.update(bad)
    want = getattr(F, "FUSION_E_" + code)
    assert F.lib().mx_quantize(a["x"], a["dtype"], a["stride"], a["R"], a["K"], a["q"], a["s"], None) == want
    assert F.lib().mx_dequantize(a["q"], a["s"], a["R"], a["K"], a["x"], a["dtype"], a["stride"], None) == want


@pytest.mark.parametrize("bad,code", [
    (dict(M=-1), "ARG"), (dict(N=0), "ARG"), (dict(K=0), "ARG"), (dict(K=40), "UNSUPPORTED"), (dict(A=None), "ARG"),
    (dict(sA=None), "ARG"), (dict(W=None), "ARG"), (dict(sW=None), "ARG"), (dict(out=None), "ARG"), (dict(A=P(4104)), "ARG"),
    (dict(sW=P(4100)), "ARG"), (dict(M=1 << 24, K=1024), "UNSUPPORTED"), (dict(N=1 << 24, K=1024), "UNSUPPORTED"),
    (dict(N=1 << 25, K=32), "UNSUPPORTED")])
def test_refusals_of_the_product(bad, code):
    a = dict(A=SOME, sA=SOME, W=SOME, sW=SOME, M=4, N=8, K=64, out=SOME)
    a.update(bad)
    rc = F.lib().joint_project_mx(a["A"], a["sA"], a["W"], a["sW"], None, a["M"], a["N"], a["K"], a["out"], None)
    assert rc == getattr(F, "FUSION_E_" + code)


def test_empty_calls_touch_nothing():
    assert F.lib().mx_quantize(None, 0, 64, 0, 64, None, None, None) == F.FUSION_OK
    assert F.lib().mx_dequantize(None, None, 0, 64, None, 0, 64, None) == F.FUSION_OK
    assert F.lib().joint_project_mx(None, None, None, None, None, 0, 8, 64, None, None) == F.FUSION_OK


def test_scale_stride():
    assert [F.mx_scale_stride(K) for K in (32, 256, 288, 640)] == [8, 8, 16, 24] == [O.scale_stride(K) for K in (32, 256, 288, 640)]


# ---------------------------------------------------------------------------
# GPU
# ---------------------------------------------------------------------------
def dev():
    return torch.device("cuda:0")


def _quantize(x, pad=0, offset=0):
    """q and scales of x [R, K] (a torch CPU tensor), from rows K + pad apart; guards behind both outputs."""
    R, K = x.shape
    buf = torch.full((R * (K + pad) + offset + 8,), float("nan"), dtype=x.dtype, device=dev())
    view = buf[offset:offset + R * (K + pad)].view(R, K + pad)[:, :K]
    view.copy_(x)
    ss = F.mx_scale_stride(K)
    q = torch.full((R * K // 2 + 64,), 0xA5, dtype=torch.uint8, device=dev())
    s = torch.full((R * ss + 64,), 0xA5, dtype=torch.uint8, device=dev())
    F.mx_quantize(view, K + pad, R, K, q, s)
    torch.cuda.synchronize()
    assert (q[R * K // 2:] == 0xA5).all() and (s[R * ss:] == 0xA5).all()
    return q[:R * K // 2].view(R, K // 2), s[:R * ss].view(R, ss)


def _check_rows(x, **place):
    q, s = _quantize(x, **place)
    R, K = x.shape
    want_q, want_s = O.quantize(x.double().numpy())
    assert np.array_equal(s.cpu().numpy(), want_s)
    assert np.array_equal(q.cpu().numpy(), want_q)
    back = O.values(want_q, want_s, K)
    for name, t in DTYPES.items():
        out = torch.full((R * (K + 3) + 16,), 7.0, dtype=t, device=dev())
        F.mx_dequantize(q, s, R, K, out, K + 3)
        got = out.cpu()
        rows = got[:R * (K + 3)].view(R, K + 3)
        assert (rows[:, K:] == 7.0).all() and (got[R * (K + 3):] == 7.0).all()
        want = torch.tensor(back).to(t)  # one rounding of the exact value
        assert torch.equal(torch.nan_to_num(rows[:, :K].float(), nan=1e9), torch.nan_to_num(want.float(), nan=1e9)), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("R,K", [(1, 32), (3, 64), (5, 96), (2, 256), (7, 288), (64, 640), (33, 1184), (1000, 32)])
def test_rows(R, K, dtype):
    rng = np.random.default_rng(R * K)
    x = rng.standard_normal((R, K)) * 2.0 ** rng.integers(-8, 9, (R, 1))
    x[rng.random((R, K)) < 0.1] = 0.0
    x[0, :32] = 0.0
    x = torch.tensor(x).to(DTYPES[dtype])
    _check_rows(x)
    _check_rows(x, pad=int(rng.integers(1, 9)), offset=int(rng.integers(1, 8)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_every_value_of_16_bits(dtype):
    """Every bit pattern as the block's largest value and as a smaller one under several largest ones."""
    bits = np.arange(1 << 16, dtype=np.uint16)
    v = torch.from_numpy(bits.view(np.int16)).view(DTYPES[dtype])
    x = torch.zeros((1 << 16, 32), dtype=DTYPES[dtype])
    x[:, 5] = v
    _check_rows(x)
    finite = torch.isfinite(v.float())
    blocks = v[finite][:(int(finite.sum()) // 30) * 30].reshape(-1, 30)
    for top in (1.0, 6.0, 200.0, 2.0 ** -10):
        x = torch.zeros((blocks.shape[0], 32), dtype=DTYPES[dtype])
        x[:, 1:31] = torch.where(blocks.abs() <= top, blocks, torch.zeros((), dtype=DTYPES[dtype]))
        x[:, 0] = top
        _check_rows(x)


@pytest.mark.gpu
def test_halfway_values_at_every_scale():
    """The midpoints between levels and their fp32 neighbours, from the largest scale to below the smallest."""
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=np.float32)
    near = np.concatenate([mid, np.nextafter(mid, 0, dtype=np.float32), np.nextafter(mid, 9, dtype=np.float32)])
    rows = []
    for e in list(range(-149, -115)) + list(range(-3, 4)) + list(range(115, 126)):
        for top in (4.0, 7.5):
            row = np.zeros(32, dtype=np.float32)
            row[:21] = near
            row[21:28] = -mid
            row[28] = top
            row[29], row[30] = -0.0, 6.0 if top == 7.5 else 3.99
            rows.append(np.ldexp(row, e).astype(np.float32))  # (rounded where it falls below the normal range)
    _check_rows(torch.tensor(np.stack(rows)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_broken_and_extreme_blocks(dtype):
    big = float(torch.finfo(DTYPES[dtype]).max)
    small = float(torch.finfo(DTYPES[dtype]).tiny)
    x = torch.zeros((6, 96), dtype=DTYPES[dtype])
    x[0, 40] = float("nan")
    x[1, 0], x[1, 95] = float("inf"), -float("inf")
    x[2, :32], x[2, 32:64] = big, -big
    x[3, :40] = small
    x[4, 3], x[4, 4] = small / 2, -small / 8
    x[5, 64:] = 1.0
    x[5, 70] = float("nan")
    _check_rows(x)


def _operands(rng, M, N, K, spread=2, bias=True):
    def one(R):
        q = rng.integers(0, 256, (R, K // 2), dtype=np.uint8)
        s = np.full((R, O.scale_stride(K)), 0, dtype=np.uint8)
        s[:, :K // 32] = rng.integers(127 - spread, 128 + spread, (R, K // 32))
        return q, s

    return one(M) + one(N) + ((rng.standard_normal(N).astype(np.float32) if bias else None),)


def _product(qa, sa, qw, sw, bias, K):
    M, N = qa.shape[0], qw.shape[0]
    t = [torch.from_numpy(np.ascontiguousarray(a)).to(dev()) for a in (qa, sa, qw, sw)]
    b = None if bias is None else torch.from_numpy(bias).to(dev())
    out = torch.full((M * N + 64,), float("nan"), device=dev())
    F.joint_project_mx(*t, b, M, N, K, out)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    assert np.isnan(got[M * N:]).all()
    return got[:M * N].reshape(M, N)


def _check_product(qa, sa, qw, sw, bias, K, rows=None):
    got = _product(qa, sa, qw, sw, bias, K).astype(np.float64)
    if rows is not None:
        got, qa, sa = got[rows], qa[rows], sa[rows]
    A, W = O.values(qa, sa, K), O.values(qw, sw, K)
    exact = A @ W.T + (0.0 if bias is None else bias.astype(np.float64))
    g = (K - 1) * U32 / (1 - (K - 1) * U32)
    e = g * (np.abs(A) @ np.abs(W).T)
    bound = e + U32 * (np.abs(exact) + e)
    bad = np.argwhere(~(np.abs(got - exact) <= bound))
    assert bad.size == 0, f"{bad.shape[0]} outputs outside the bound, first {bad[:3]}"


@pytest.mark.gpu
def test_product_of_single_elements():
    """One element of A against one of W at every place of two stages: each finds its partner and its own scales."""
    K = 512
    qa, sa, qw, sw, _ = _operands(np.random.default_rng(1), K, 16, K, 0, False)
    qa[:], qw[:] = 0, 0
    rng = np.random.default_rng(2)
    sa[:, :K // 32] = rng.integers(100, 150, sa[:, :K // 32].shape)
    sw[:, :K // 32] = rng.integers(100, 150, sw[:, :K // 32].shape)
    for k in range(K):
        qa[k, k // 2] = 7 << (4 * (k & 1))  # row k of A: 6.0 at place k
    qw[:] = rng.integers(0, 256, qw.shape, dtype=np.uint8)
    got = _product(qa, sa, qw, sw, None, K)
    want = O.values(qa, sa, K) @ O.values(qw, sw, K).T  # a single product each: exact
    assert np.array_equal(got.astype(np.float64), want)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (1, 16, 64), (5, 130, 96), (256, 4096, 640), (129, 1001, 288), (300, 777, 512),
                                   (33, 4099, 1056), (1100, 1030, 224), (2100, 1001, 160), (2200, 2050, 352)])
def test_product(M, N, K):
    a = _operands(np.random.default_rng(M + N + K), M, N, K)
    _check_product(*a, K)
    _check_product(*a[:4], None, K)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(33001, 2050, 96), (32768, 2048, 640), (9000, 130, 256), (70001, 100, 64), (40000, 1001, 32),
                                   (33000, 1030, 1056), (130000, 130, 288), (8200, 1002, 768),
                                   (16500, 517, 160), (50000, 2001, 96), (70000, 200, 640)])
def test_product_of_many_rows(M, N, K):
    a = _operands(np.random.default_rng(M), M, N, K)
    rows = np.unique(np.concatenate([np.random.default_rng(1).choice(M, 150), [0, M - 1]]))
    _check_product(*a, K, rows=rows)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(40, 70, 352), (9000, 1000, 352)])
def test_product_ignores_bytes_behind_the_scales_and_spreads_nan(M, N, K):
    rng = np.random.default_rng(5)
    qa, sa, qw, sw, bias = _operands(rng, M, N, K)
    clean = _product(qa, sa, qw, sw, bias, K)
    sa[:, K // 32:], sw[:, K // 32:] = 255, 255
    assert np.array_equal(_product(qa, sa, qw, sw, bias, K), clean)
    sa[7, 3], sw[11, 10] = 255, 255
    qa[7, 48:64], qw[11, 160:176] = 0, 0  # as mx_quantize leaves a block with a NaN
    got = _product(qa, sa, qw, sw, bias, K)
    nan = np.zeros((M, N), dtype=bool)
    nan[7], nan[:, 11] = True, True
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(got[~nan], clean[~nan])


@pytest.mark.gpu
def test_quantised_projection_is_near_the_bf16_one():
    """Rows quantised by the library, projected, against the exact product of the values they stand for."""
    rng = np.random.default_rng(6)
    M, N, K = 77, 300, 640
    A = torch.tensor(rng.standard_normal((M, K))).bfloat16()
    W = torch.tensor(rng.standard_normal((N, K)) * 2 / np.sqrt(K)).bfloat16()
    qa, sa = (t.cpu().numpy() for t in _quantize(A))
    qw, sw = (t.cpu().numpy() for t in _quantize(W))
    _check_product(qa, sa, qw, sw, None, K)


@pytest.mark.gpu
def test_graph_replays():
    rng = np.random.default_rng(7)
    M, N, K = 130, 260, 320
    x = torch.empty((M, K), dtype=torch.bfloat16, device=dev())
    W = torch.tensor(rng.standard_normal((N, K))).bfloat16().to(dev())
    ss = F.mx_scale_stride(K)
    qw, sw = torch.empty((N, K // 2), dtype=torch.uint8, device=dev()), torch.empty((N, ss), dtype=torch.uint8, device=dev())
    F.mx_quantize(W, K, N, K, qw, sw)

    def buffers():
        return (torch.empty((M, K // 2), dtype=torch.uint8, device=dev()), torch.empty((M, ss), dtype=torch.uint8, device=dev()),
                torch.empty((M, N), device=dev()), torch.empty((M, K), device=dev()))

    def call(q, s, out, back):
        F.mx_quantize(x, K, M, K, q, s)
        F.joint_project_mx(q, s, qw, sw, None, M, N, K, out)
        F.mx_dequantize(q, s, M, K, back, K)

    a, b = buffers(), buffers()
    x.normal_()
    call(*a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(*a)
    for i in range(3):
        x.normal_()
        g.replay()
        call(*b)
        torch.cuda.synchronize()
        for u, v in zip(a, b):
            assert torch.equal(u, v), i
