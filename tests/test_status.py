"""fusion_device_status gathers the bits of every kernel that sets one, and clears them."""

from __future__ import annotations

import numpy as np
import pytest

import paper_2609_14991_amd as F
from workloads import tiny_random_lm

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_bits_of_all_sources_at_once_and_apart():
    V, K, H = 40, 64, 4
    glm = F.ngram_load_arrays(tiny_random_lm(np.random.default_rng(1), V, 3, n_sent=200))
    x = torch.zeros((1, H, V), device="cuda")
    A, W = torch.zeros((1, H, K), device="cuda").bfloat16(), torch.zeros((V, K), device="cuda").bfloat16()
    good = torch.zeros((1, H), dtype=torch.int32, device="cuda")
    bad = torch.full((1, H), V, dtype=torch.int32, device="cuda")
    state = torch.full((1, H), V, dtype=torch.int32, device="cuda")
    lost = torch.full((1, H), 1 << 30, dtype=torch.int32, device="cuda")
    boost = torch.zeros(H, dtype=torch.int32, device="cuda")
    term = torch.empty(H, dtype=torch.float64, device="cuda")
    score, joint = (lambda t: F.score(x, t)), (lambda t: F.score_projected(A, W, None, t))
    end = lambda s: F.fusion_end_scores([glm], [1.0], s, H, None, term)  # noqa: E731
    step = lambda s: F.step(glm, None, x[0], s[0], boost, 0.5, 0.0, 0, 1, F.FUSION_BLANK_AM)  # noqa: E731
    TOKEN, LM = F.FUSION_STATUS_BAD_TOKEN, F.FUSION_STATUS_BAD_LM_STATE
    F.fusion_device_status()
    for calls, want in [(((score, bad),), TOKEN), (((joint, bad),), TOKEN), (((end, lost),), LM), (((step, lost),), LM),
                        (((score, bad), (end, lost)), TOKEN | LM), (((joint, bad), (score, good), (step, lost)), TOKEN | LM),
                        (((score, bad), (joint, bad), (end, lost), (step, lost)), TOKEN | LM),
                        (((score, good), (joint, good), (end, state), (step, state)), 0)]:
        for call, arg in calls:
            call(arg)
        assert F.fusion_device_status() == want
        assert F.fusion_device_status() == 0
