"""The 4-bit projection by panels (joint_project_mx where the output's stores bound it): its compiled lengths of K,
and few rows of many columns, whose only row tile lies past the operand for the most part."""

from __future__ import annotations

import numpy as np
import pytest

from test_mx import _check_product, _operands

pytest.importorskip("torch")


def _panel_steps(M, N, K):
    """Steps of 128 along K that the panel kernel takes, 0 where tiles are taken: the rule of joint_project_mx."""
    tiles = -(-M // 128) * -(-N // 128)
    drifts = N % 32 != 0 and K <= 128 and tiles >= 4500
    return -(-K // 128) if K <= 768 and tiles >= 512 and not drifts else 0


FEW = [(1, 65500, 640), (53, 65536, 640), (64, 65409, 288), (65, 65440, 768), (33, 131000, 32), (7, 70000, 416)]
LENGTHS = [(9000, 1000, K) for K in (96, 128, 160, 256, 288, 384, 416, 448, 512, 544, 640, 672, 768)]


def test_every_length_is_taken():
    assert {_panel_steps(*s) for s in LENGTHS} == {1, 2, 3, 4, 5, 6}
    assert all(_panel_steps(*s) for s in FEW)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", FEW)
def test_few_rows_of_many_columns(M, N, K):
    _check_product(*_operands(np.random.default_rng(M + N), M, N, K), K)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", LENGTHS)
def test_every_length_of_k(M, N, K):
    rows = np.unique(np.concatenate([np.random.default_rng(K).choice(M, 200), [0, 63, 64, M - 1]]))
    _check_product(*_operands(np.random.default_rng(K), M, N, K), K, rows=rows)
