"""The example that runs gated layers, scores and the distillation loss together: its gradients against autograd in 64 bits, and a single token's
scores against the same token's in a batch."""
import gc
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def ex():
    import distill_step
    yield distill_step
    gc.collect()


def reference(m, tokens, index, teacher, scale):
    w = {k: v.double().requires_grad_(True) for k, v in m.w.items()}
    f = torch.nn.functional
    x = w["embed"][tokens]
    gate, up = (x @ w["both"]).chunk(2, 1)
    y = x + (f.silu(gate) * up) @ w["down"]
    logs = torch.log_softmax(scale * (y @ w["head"].t()), 1)
    q = torch.log_softmax(scale * teacher.double(), 1)
    return w, (q.exp() * (q - logs.gather(1, index))).sum(1)


@pytest.mark.parametrize("dtype,limit", [("f32", 1e-5), ("f16", 1e-2), ("bf16", 8e-2)])
def test_gradients(ex, dtype, limit):
    """Relative error (2-norm) of every weight's gradient.  A value passes about eight roundings of its type on its way (activations kept, gradients handed
    on): eight times the unit roundoff, and two and a half times that for what cancels; fp32's 1e-5 leaves room for sums of a thousand terms."""
    scale = 0.75
    teacher, m = ex.Model(dtype, vocab=331, width=64, inner=184, seed=3), ex.Model(dtype, vocab=331, width=64, inner=136, seed=4)
    tokens = torch.randint(0, 331, (203,), generator=torch.Generator("cuda").manual_seed(5), device="cuda")
    lesson = teacher.scores(tokens, top=6, scale=scale)
    s = m.forward(tokens)
    loss = m.loss(s, lesson["top_index"], lesson["top_logprob"], scale)
    times = 64.0 if dtype == "f16" else 1.0
    grads = m.backward(s, lesson["top_index"], lesson["top_logprob"], torch.full((203,), times / 100, device="cuda"), scale)
    w, want = reference(m, tokens, lesson["top_index"], lesson["top_logprob"], scale)
    assert float((loss.double() - want.detach()).abs().max()) <= limit * 10
    want.sum().div(100).backward()
    assert set(grads) == set(w)
    for name, got in grads.items():
        off = float((got.double() / times - w[name].grad).norm() / w[name].grad.norm())
        assert off <= limit, (name, off)


def test_runs_and_scores_one_token(ex):
    assert len(ex.main("bf16", 3)) == 3
    m = ex.Model("f32")
    tokens = torch.arange(40, device="cuda")
    batch = m.scores(tokens, targets=(tokens * 7 + 3) % m.vocab, top=5)
    for i in (0, 13, 39):
        one = m.scores(tokens[i:i + 1], targets=((tokens * 7 + 3) % m.vocab)[i:i + 1], top=5)
        for k in ("logprob", "entropy", "top_logprob"):
            assert float((one[k][0] - batch[k][i]).abs().max()) <= 1e-4
