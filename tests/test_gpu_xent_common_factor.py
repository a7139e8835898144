"""G of the loss's gradient is rounded to 16 bits, and most of it is -dloss at the targets.  Where all tokens share one dloss, its rounding must
not become a factor of both gradients."""
import gc
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,V,D", [(401, 1343, 232), (77, 4099, 128), (1000, 3000, 256), (3001, 9000, 64), (3, 2000, 768)])
def test_gradients_of_a_mean_have_no_common_factor(gs, dtype, T, V, D):
    """The results' component along the exact ones is 1 to a quarter of the unit roundoff: the results' own roundings, and those of the probabilities,
    have no common sign and average out over 2304 elements and more (to a fiftieth of the unit roundoff and less)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    X = torch.empty((T, D), device="cuda").normal_(0.0, 1.0, generator=g).to(TORCH[dtype])
    W = torch.empty((V, D), device="cuda").normal_(0.0, 2.0 / math.sqrt(D), generator=g).to(TORCH[dtype])
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    x, w = X.double(), W.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1).float()
    p = torch.exp(z - lse.double()[:, None])
    G = p - torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    ws = torch.empty(gs.xent_workspace_bytes(dtype, T, V, D, backward=True), dtype=torch.uint8, device="cuda")
    for factor in (1.0 / T, 1.0, 100.0 / 3):
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        dloss = torch.full((T,), factor, device="cuda")
        gs.xent_backward(X, W, t, lse, dloss, dX, dW, workspace=ws)
        for got, want in ((dX, G @ w * dloss[0].double()), (dW, G.t() @ x * dloss[0].double())):
            along = float((got.double() * want).sum() / (want * want).sum())
            assert abs(along - 1) <= ROUND[dtype] / 4, (factor, along - 1)
