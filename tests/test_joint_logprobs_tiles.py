"""Scoring from hidden states over every tile shape of its statistics kernel, with a K of more stages than a shape
keeps in flight and with shorter ones."""

from __future__ import annotations

import numpy as np
import pytest

from test_joint_logprobs import _check, _decoded, _joint

pytest.importorskip("torch")

CUS = 256


def _shape(M, V):
    """Rows and columns of a tile: the rule of joint_logprobs."""
    tiles = lambda bm, bn: -(-M // bm) * -(-V // bn)  # noqa: E731
    if tiles(256, 256) >= 1000 and V > 128:
        return 256, 256
    for bm, bn in ((128, 128), (64, 128), (64, 64)):
        if tiles(bm, bn) > CUS:
            return bm, bn
    return 32, 64


# T, S, B, V
SIZES = {(256, 256): (20, 413, 4, 2050), (128, 128): (3, 1000, 1, 2001), (64, 128): (3, 350, 2, 1001), (64, 64): (5, 104, 2, 1030),
         (32, 64): (2, 13, 3, 700)}


def test_every_shape_is_taken():
    for shape, (T, S, B, V) in SIZES.items():
        assert _shape(T * S * B, V) == shape


@pytest.mark.gpu
@pytest.mark.parametrize("K", [40, 128, 328, 584])
@pytest.mark.parametrize("shape", list(SIZES))
def test_every_shape(shape, K):
    T, S, B, V = SIZES[shape]
    rng = np.random.default_rng(K + V)
    A, W, bias = _joint(rng, T * S * B, V, K)
    tok, par = _decoded(rng, T, S, B, V)
    _check(A, W, bias, T, S, B, tok, par, frames=[0, T - 1])
