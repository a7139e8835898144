"""A batch whose X has more than 2^32 elements, at an odd number of tokens (X is copied to whole vectors of tokens for the vocabulary's gradient)."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()
    torch.cuda.empty_cache()                     # (other modules count the device memory that is in use)


def test_odd_batch_beyond_32_bits(gs):
    """dW of 16 entries.  One token in 997 has a loss that counts for something, so of the million terms of a sum n = 1052 are not zero: off by
    (n + 8) u sum|G||x| at most, beside G's rounding to f16 (2^-11, and 2^-39 of the largest dloss below its normal range), the probabilities'
    (2 e_z + 4e-6) and the result's."""
    T, V, D = 1048579, 16, 4104
    X = torch.empty((T, D), dtype=torch.float16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for at in range(0, T, 65536):
        X[at:at + 65536] = torch.empty((min(65536, T - at), D), device="cuda").normal_(0.0, 1.0, generator=g).half()
    W = torch.empty((V, D), device="cuda").normal_(0.0, D ** -0.5, generator=g).half()
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    lse, dloss = torch.empty(T, device="cuda"), torch.zeros(T, device="cuda")
    dloss[::997] = 1.0 / 64
    dloss[-1] = 1.0 / 64
    n = int((dloss != 0).sum())
    gs.xent_forward(X, W, None, None, lse, workspace=torch.empty(gs.xent_workspace_bytes("f16", T, V, D), dtype=torch.uint8, device="cuda"))
    dW = torch.empty_like(W)
    gs.xent_backward(X, W, t, lse, dloss, None, dW, workspace=torch.empty(gs.xent_workspace_bytes("f16", T, V, D, backward=True), dtype=torch.uint8, device="cuda"))
    which = torch.nonzero(dloss)[:, 0]
    x, w, at = X[which].double(), W.double(), t[which]
    z = x @ w.t()
    p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
    one = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    G = (p - one) / 64
    e_z = (D + 1) * U * (x.abs() @ w.abs().t()).amax(1, keepdim=True)
    want = G.t() @ x
    limit = (G.abs() * (2.0 ** -11 * 1.01 + (n + 10) * U) + p / 64 * (4 * e_z + 1e-5) + 2.0 ** -39 / 64 + 4 * U / 64).t() @ x.abs()
    bad = ~((dW.double() - want).abs() <= 1.01 * limit + 2.0 ** -11 * want.abs() + 2.0 ** -25)
    assert not bool(bad.any()), (int(bad.sum()), float(((dW.double() - want).abs() / limit).max()))
