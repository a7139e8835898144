"""Tokens that do not count (their target is ignored or outside the vocabulary) have no say in a projection's cross entropy and its gradient,
whatever their row of X, their lse and their dloss hold: every other result is the same to the bit as with zeros in those places."""
import gc
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
IGNORE = -100
# small tiles, tiles whose wave groups alternate, rows at odd alignment (G's rows are padded to whole vectors), more tiles than compute units
SIZES = [(20, 300, 64), (77, 1003, 41), (300, 4096, 256), (2310, 9000, 128)]


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def inputs(dtype, T, V, D, seed=5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    X = torch.empty((T, D), device="cuda").normal_(0.0, 1.0, generator=g).to(TORCH[dtype])
    W = torch.empty((V, D), device="cuda").normal_(0.0, 2.0 / math.sqrt(D), generator=g).to(TORCH[dtype])
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    out = torch.rand(T, generator=g, device="cuda") < 0.2
    out[1], out[2], out[3] = True, True, False
    t[out] = IGNORE
    t[1], t[2] = V, -1
    return X, W, t, out


def gradient(gs, dtype, X, W, t, lse, dloss):
    (T, D), V = X.shape, W.shape[0]
    dX, dW = torch.full_like(X, 5.0), torch.full_like(W, 5.0)
    gs.xent_backward(X, W, t, lse, dloss, dX, dW, ignore_index=IGNORE, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D, backward=True)))
    return dX, dW


def clean(gs, dtype, T, V, D):
    """Inputs with zeros in the places that do not count, and their gradients."""
    X, W, t, out = inputs(dtype, T, V, D)
    X[out] = 0
    lse, dloss = torch.empty(T, device="cuda"), torch.full((T,), 1.0 / T, device="cuda")
    gs.xent_forward(X, W, t, None, lse, ignore_index=IGNORE, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D)))
    dloss[out] = 0
    return X, W, t, out, lse, dloss, gradient(gs, dtype, X, W, t, lse, dloss)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_rows_that_do_not_count(gs, dtype, T, V, D):
    X, W, t, out, lse, dloss, (dX, dW) = clean(gs, dtype, T, V, D)
    big = float(torch.finfo(TORCH[dtype]).max)
    for value in (big, -big, math.inf, math.nan):
        X[out] = value                           # of either sign in the logits: W's entries are
        gX, gW = gradient(gs, dtype, X, W, t, lse, dloss)
        assert bool((gX[out] == 0).all()), (value, int((gX[out] != 0).sum()))
        assert torch.equal(gX, dX), value
        if math.isfinite(value):                 # (dW = G^T X: zero times what is not finite is NaN there as in the definition)
            assert torch.equal(gW, dW), (value, int((gW != dW).sum()))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_lse_that_does_not_count(gs, dtype, T, V, D):
    X, W, t, out, lse, dloss, (dX, dW) = clean(gs, dtype, T, V, D)
    for value in (math.inf, -math.inf, math.nan):
        lse[out] = value
        gX, gW = gradient(gs, dtype, X, W, t, lse, dloss)
        assert torch.equal(gX, dX) and torch.equal(gW, dW), value


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_dloss_that_does_not_count(gs, dtype, T, V, D):
    """A mean over no token at all leaves 1 / 0 or 1e8 there; f16's scale is that of the tokens that count."""
    X, W, t, out, lse, dloss, (dX, dW) = clean(gs, dtype, T, V, D)
    assert bool((dW != 0).any())
    for value in (1e8, -1e30, math.inf, math.nan):
        dloss[out] = value
        gX, gW = gradient(gs, dtype, X, W, t, lse, dloss)
        assert torch.equal(gX, dX) and torch.equal(gW, dW), value


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D", SIZES)
def test_losses_beside_rows_that_do_not_count(gs, dtype, T, V, D):
    X, W, t, out = inputs(dtype, T, V, D)
    ws, big = workspace(gs.xent_workspace_bytes(dtype, T, V, D)), float(torch.finfo(TORCH[dtype]).max)
    want, lse, loss, full = (torch.empty(T, device="cuda") for _ in range(4))
    X[out] = 0
    gs.xent_forward(X, W, t, want, lse, ignore_index=IGNORE, workspace=ws)
    for value in (big, -big, big / 16, math.inf, math.nan):
        X[out] = value
        gs.xent_forward(X, W, t, loss, full, ignore_index=IGNORE, workspace=ws)
        assert torch.equal(full[~out], lse[~out]) and torch.equal(loss[~out], want[~out]), value
        assert bool((loss[t == IGNORE] == 0).all())
