"""Results of so many small tiles that a launch of a thread per lane would need more than the 2^32 threads it may have: every one of them is there."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROWS = 1100000000


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()
    torch.cuda.empty_cache()                     # (other modules count the device memory that is in use)


def rows(n):
    """Small whole numbers, exact in f16 beside a factor of two."""
    return (torch.arange(n, device="cuda", dtype=torch.int32) % 1021).to(torch.float16).view(n, 1)


def test_product(gs):
    A, B = rows(ROWS), torch.full((1, 1), 2.0, dtype=torch.float16, device="cuda")
    C = torch.full((ROWS, 1), 7.5, dtype=torch.float16, device="cuda")
    gs.gemm_fused(gs.gemm_problem("f16", ROWS, 1, 1, out_dtype="f16"), A, B, C, act="relu")
    assert int((C != 2 * A).sum()) == 0


def test_grouped(gs):
    A, B = rows(ROWS), torch.full((3, 1, 1), 2.0, dtype=torch.float16, device="cuda")
    C = torch.full((ROWS, 1), 7.5, dtype=torch.float16, device="cuda")
    B[1] = 1.0
    off = torch.tensor([0, 1000, ROWS - 500000000, ROWS], dtype=torch.int32, device="cuda")
    gs.grouped_gemm(gs.grouped_problem("f16", 3, ROWS, 1, 1, 0, "f16"), off, A, B, C)
    A[:1000] *= 2
    A[ROWS - 500000000:] *= 2
    assert int((C != A).sum()) == 0


def test_grouped_gradient(gs):
    """A matrix of one element to each of twenty million groups, the first and the last ten of them empty."""
    G = 20000000
    off = torch.arange(G + 1, dtype=torch.int32, device="cuda").clamp_(10, G - 10)
    A, dY = rows(G), torch.full((G, 1), 2.0, dtype=torch.float16, device="cuda")
    dW = torch.full((G, 1, 1), 7.5, dtype=torch.float16, device="cuda")
    gs.grouped_wgrad(gs.grouped_problem("f16", G, G, 1, 1, 0, "f16"), off, A, dY, dW)
    want = 2 * A
    want[:10], want[-10:] = 0, 0
    assert int((dW.view(G, 1) != want).sum()) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_loss(gs, dtype):
    """lse moves by no more than a logit's error, 2 u |x w|, and 2e-6 + 2 u |lse| of the exponentials and sums."""
    T, V = 200000003, 100
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.empty((T, 1), device="cuda", dtype=dtype).uniform_(-2.0, 2.0, generator=g)
    W = torch.empty((V, 1), device="cuda", dtype=dtype).normal_(0.0, 1.0, generator=g)
    t = torch.arange(T, device="cuda") % V
    loss, lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    n = gs.xent_workspace_bytes("bf16" if dtype is torch.bfloat16 else "f32", T, V, 1)
    gs.xent_forward(X, W, t, loss, lse, workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
    step, bad = 4000000, 0
    for at in range(0, T, step):
        z = X[at:at + step].double() @ W.double().t()
        want = torch.logsumexp(z, 1)
        limit = 2 * U * z.abs().amax(1) + 2e-6 + 2 * U * want.abs()
        bad += int(((lse[at:at + step].double() - want).abs() > limit).sum())
        bad += int(((loss[at:at + step].double() - (want - z.gather(1, t[at:at + step, None])[:, 0])).abs() > 2 * limit).sum())
    assert bad == 0


def test_plain_product(gs):
    A, B = rows(ROWS), torch.full((1, 1), 2.0, dtype=torch.float16, device="cuda")
    C = torch.full((ROWS, 1), 7.5, dtype=torch.float16, device="cuda")
    gs.gemm(gs.gemm_problem("f16", ROWS, 1, 1, out_dtype="f16"), A, B, C)
    assert int((C != 2 * A).sum()) == 0


def test_plain_batches(gs):
    """Thirty million products of two rows, a column and two terms."""
    n = 30000000
    A, B = (rows(4 * n) % 29).view(n, 2, 2), torch.full((n, 2, 1), 2.0, dtype=torch.float16, device="cuda")
    B[:, 1] = 3.0
    C = torch.full((n, 2, 1), 7.5, dtype=torch.float16, device="cuda")
    gs.bmm(gs.gemm_problem("f16", 2, 1, 2, batch=n, out_dtype="f16"), A, B, C)
    assert int((C[:, :, 0] != 2 * A[:, :, 0] + 3 * A[:, :, 1]).sum()) == 0
