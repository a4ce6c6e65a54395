"""The scoring conveniences beside torch's autograd: a gradient written over logits that a graph has saved is seen
by that graph, and the gradient that score_backward gives is autograd's."""

from __future__ import annotations

import pytest

import paper_2609_14991_amd as F

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

T, H, V = 3, 4, 130


def _inputs():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((T, H, V), generator=g, device="cuda")
    tok = torch.randint(0, V, (T, H), generator=g, device="cuda", dtype=torch.int32)
    return x, tok, torch.randn((T, H), generator=g, device="cuda")


def test_a_graph_that_saved_the_logits_refuses_after_a_gradient_in_place():
    x, tok, gl = _inputs()
    for in_place in (False, True):
        leaf = torch.ones((T, H, V), device="cuda", requires_grad=True)
        logits = leaf * x
        y = logits.exp().sum() + (logits * logits).sum()   # saves the logits
        scored = F.score(logits.detach(), tok)
        assert not scored["logp"].requires_grad
        F.score_backward(logits.detach(), scored, tok, None, 1, gl, None, in_place=in_place)
        if in_place:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()
        else:
            y.backward()
            assert torch.isfinite(leaf.grad).all()


def test_in_place_on_a_view_and_in_inference_mode():
    x, tok, gl = _inputs()
    wide = torch.zeros((T, H, V + 6), device="cuda")
    wide[:, :, :V] = x
    view, was = wide[:, :, :V], wide._version
    grad = F.score_backward(x, F.score(x, tok), tok, None, 1, gl)
    assert x._version == 0
    assert torch.equal(F.score_backward(view, F.score(view, tok), tok, None, 1, gl, in_place=True), grad) and wide._version > was
    with torch.inference_mode():
        y = x.clone()
        assert torch.equal(F.score_backward(y, F.score(y, tok), tok, None, 1, gl, in_place=True), grad)


def test_the_gradient_goes_on_through_autograd():
    """Logits that require a gradient: score's results are without one, score_backward's is what autograd takes on,
    twice with an earlier graph of the same leaves alive."""
    x, tok, gl = _inputs()
    w = torch.randn((V, V), device="cuda", requires_grad=True)
    grads = []
    for _ in range(2):
        logits = x @ w / 9
        scored = F.score(logits, tok)
        assert not scored["logp"].requires_grad and not scored["entropy"].requires_grad
        logits.backward(F.score_backward(logits, scored, tok, None, 1, gl))
        grads.append(w.grad.clone())
        w.grad = None
    x64, w64, gl64 = x.double(), w.double(), gl.double()
    lp = torch.log_softmax(x64 @ w64 / 9, 2)
    want = torch.autograd.grad((lp.gather(2, tok.long()[:, :, None])[:, :, 0] * gl64).sum(), w)[0].double()
    assert torch.equal(grads[0], grads[1])
    # logits off by d: V + 2 roundings of their sums' terms.  p is then off by a factor of e^(2 d) and by its own 30
    # roundings, the gradient of w by that in every term of its sum over the rows, and by the sum's own roundings
    u = 2.0 ** -24
    d = (V + 2) * u * (x64.abs() @ w64.abs()).max() / 9
    one = torch.nn.functional.one_hot(tok.long(), V)
    terms = (x64.abs().reshape(-1, V).T @ (gl64.abs()[:, :, None] * (one + lp.exp())).reshape(-1, V)) / 9
    assert ((grads[0].double() - want).abs() <= (2.1 * d + (30 + T * H + 2) * u) * terms).all()
