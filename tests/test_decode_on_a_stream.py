"""The decode's conveniences on a stream that is not torch's current one, while that is at work: fused rows are
cleared on the stream that writes them, and no output takes memory that the current stream still uses."""

from __future__ import annotations

import numpy as np
import pytest

import paper_2609_14991_amd as F
from workloads import tiny_random_lm

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

T, S, B, V, K = 5, 6, 4, 700, 128
H = S * B


def _decoders():
    rng = np.random.default_rng(2)
    glm = F.ngram_load_arrays(tiny_random_lm(rng, V, 3, n_sent=2000))
    x = torch.from_numpy((rng.standard_normal((T, H, V)) * 2).astype(np.float32)).to("cuda")
    A, W = torch.randn((H, K), device="cuda").bfloat16(), torch.randn((V, K), device="cuda").bfloat16()

    def states():
        return (torch.full((1, H), V, dtype=torch.int32, device="cuda"), torch.zeros(H, dtype=torch.int32, device="cuda"),
                torch.from_numpy(np.tile(np.array([0.0] + [-np.inf] * (B - 1)), S)).to("cuda"))

    greedy = lambda st, s: F.run(glm, None, x, H, 1, 1, 0.5, 0.0, 0, F.FUSION_BLANK_AM, st[0][0], st[1], None,  # noqa: E731
                                 want_fused=True, stream=s)
    beam = lambda st, s: F.run_lms([glm], [0.5], None, x, S, B, 4, 0.0, 0, F.FUSION_BLANK_COMPETE, st[0], st[1], st[2],  # noqa: E731
                                   want_fused=True, stream=s)
    step = lambda st, s: F.step(glm, None, x[0], st[0][0], st[1], 0.5, 0.0, 0, 4, F.FUSION_BLANK_COMPETE,  # noqa: E731
                                want_fused=True, stream=s)
    steps = lambda st, s: F.step_lms([glm], [0.5], None, x[0], st[0], st[1], 0.0, 0, 4, F.FUSION_BLANK_COMPETE,  # noqa: E731
                                     want_fused=True, stream=s)
    project = lambda st, s: dict(logits=F.project(A, W, stream=s))  # noqa: E731
    return states, dict(run=greedy, run_lms=beam, step=step, step_lms=steps, project=project)


@pytest.mark.parametrize("name", ["run", "run_lms", "step", "step_lms", "project"])
def test_a_call_beside_a_busy_current_stream(name):
    states, calls = _decoders()
    call = calls[name]
    want = call(states(), None)
    big = torch.randn((4096, 4096), device="cuda")
    st, side = states(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        big @ big
    late = [torch.full_like(t, 77) for t in want.values() if t is not None]   # written behind the products ..
    del late                                                                  # .. and free for the current stream only
    got = call(st, side.cuda_stream)
    side.synchronize()
    early = {n: None if t is None else t.cpu() for n, t in got.items()}
    torch.cuda.synchronize()
    for n, t in want.items():
        assert t is None and got[n] is None or torch.equal(got[n], t) and torch.equal(early[n], t.cpu()), n
