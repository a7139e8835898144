"""The example that runs the products consumed in place together: its gradients against autograd in 64 bits, its loss over steps, and a single
token's score against the same token's loss in a batch."""
import gc
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def lm():
    import lm_step
    yield lm_step
    gc.collect()


def reference(m, tokens, targets, order, offsets):
    """Losses in the sorted order and gradients, for the given routing."""
    w = {k: v.double().requires_grad_(True) for k, v in m.w.items()}
    f = torch.nn.functional
    x = w["embed"][tokens]
    x1 = f.gelu(x @ w["up"] + w["up_bias"], approximate="tanh") @ w["down"] + w["down_bias"] + x
    xs, parts = x1[order], []
    for e in range(m.experts):
        a, b = int(offsets[e]), int(offsets[e + 1])
        h = f.gelu(xs[a:b] @ w["e_up"][e] + w["e_up_bias"][e], approximate="tanh")
        parts.append(xs[a:b] + h @ w["e_down"][e] + w["e_down_bias"][e])
    loss = f.cross_entropy(torch.cat(parts) @ w["head"].t(), targets[order], ignore_index=-100, reduction="none")
    return w, loss


@pytest.mark.parametrize("dtype,limit", [("f32", 1e-5), ("f16", 1e-2), ("bf16", 8e-2)])
def test_gradients(lm, dtype, limit):
    """Relative error (2-norm) of every weight's gradient.  A value passes about ten roundings of its type on its way (activations kept, gradients
    handed on): ten times the unit roundoff, and twice that for what cancels; fp32's 1e-5 leaves room for sums of a thousand terms."""
    m = lm.Model(dtype, vocab=331, width=64, experts=5, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    tokens = torch.randint(0, m.vocab, (203,), generator=g, device="cuda")
    targets = torch.randint(0, m.vocab, (203,), generator=g, device="cuda")
    targets[::7] = -100
    s = m.forward(tokens, targets)
    scale = 64.0 if dtype == "f16" else 1.0
    grads = m.backward(s, torch.full((203,), scale / 100, device="cuda"))
    w, loss = reference(m, tokens, targets, s["order"], s["offsets"])
    assert float((s["loss"].double() - loss.detach()).abs().max()) <= limit * 10
    loss.sum().div(100).backward()
    assert set(grads) == set(w) - {"router"}
    for name, got in grads.items():
        want = w[name].grad
        off = float((got.double() / scale - want).norm() / want.norm())
        assert off <= limit, (name, off)


def test_loss_falls_and_one_token_scores_alike(lm):
    losses = lm.main("bf16", 12)
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.8 * losses[0]
    m = lm.Model("f32")
    tokens = torch.arange(40, device="cuda")
    targets = (tokens * 7 + 3) % m.vocab
    s = m.forward(tokens, targets)
    batch = torch.empty(40, device="cuda")
    batch[s["order"]] = s["loss"]
    for i in (0, 13, 39):
        assert abs(float(m.score(tokens[i], targets[i])) - float(batch[i])) <= 1e-4
