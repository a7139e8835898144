"""Products grouped by expert beside rows of any pitch, scaled, and with one matrix that all groups share."""
import gc
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}      # half a subnormal step


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


def draw(shape, dtype, seed, sigma=1.0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    wide = torch.empty(tuple(shape[:-1]) + (shape[-1] + pad,), device="cuda").normal_(0.0, sigma, generator=g).to(TORCH[dtype])
    return wide[..., :shape[-1]]


def guarded(shape, dtype, pad):
    """An output in a frame of sevens, each matrix of a stack in one of its own: (view, check)."""
    wide = torch.full(tuple(shape[:-2]) + (shape[-2] + 2, shape[-1] + pad), 7.0, dtype=TORCH[dtype], device="cuda")
    view = wide[..., 1:-1, :shape[-1]]

    def untouched():
        assert bool((wide[..., 0, :] == 7).all()) and bool((wide[..., -1, :] == 7).all()) and bool((wide[..., :, shape[-1]:] == 7).all())
    return view, untouched


def close(got, want, bound, dtype, what):
    limit = bound + ROUND[dtype] * want.abs() + TINY[dtype]
    bad = ~((got.double() - want).abs() <= limit)
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - want).abs() / limit).nan_to_num(1e9).max()), torch.nonzero(bad)[:3].tolist())


def slope64(z):
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("sizes,N,K", [([0, 17, 64, 1, 130], 96, 64), ([3, 0, 45], 33, 41), ([700, 0, 1300], 520, 264)])
@pytest.mark.parametrize("pad", [1, 8, 13])
def test_rows_of_any_pitch(gs, dtype, out, sizes, N, K, pad):
    """A, B, C, dW and what is kept and read again in rows (and matrices) further apart than they are long; alpha = -0.75.  A sum of K terms is
    off by at most (K + 4) u sum|a||b| with alpha and the epilogue's operations, silu by 16 u |z| more, its slope by 64 u of its factor."""
    G, rows, alpha = len(sizes), sum(sizes), -0.75
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32), device="cuda")
    for tb in (0, 1):
        A, dY = draw((rows, K), dtype, 1, pad=pad), draw((rows, N), dtype, 2, pad=pad)
        W = draw((G, N, K) if tb else (G, K, N), dtype, 3, 1 / math.sqrt(K), pad=pad)
        R, Z = draw((rows, N), out, 4, pad=pad), draw((rows, N), out, 5, pad=pad)
        p = gs.grouped_problem(dtype, G, rows, N, K, tb, out)
        (C, c_fine), (kept, k_fine), (dZ, z_fine), (dW, w_fine) = (guarded(s, out, pad) for s in ((rows, N), (rows, N), (rows, N), tuple(W.shape)))
        gs.grouped_gemm(p, off, A, W, C, act="silu", preact=kept, residual=R, alpha=alpha)
        gs.grouped_act_grad(p, off, A, W, Z, dZ, "silu", alpha=alpha)
        gs.grouped_wgrad(p, off, A, dY, dW)
        at = 0
        for g, n in enumerate(sizes):
            r = slice(at, at + n)
            w = W[g].double().t() if tb else W[g].double()
            a, d, res, pre = A[r].double(), dY[r].double(), R[r].double(), Z[r].double()
            z, e = alpha * (a @ w), (K + 4) * U * abs(alpha) * (a.abs() @ w.abs())
            close(kept[r], z, e, out, ("kept", g))
            close(C[r], z / (1 + torch.exp(-z)) + res, 1.13 * e + 16 * U * z.abs() + U * res.abs(), out, ("forward", g))
            close(dZ[r], z * slope64(pre), 1.13 * e + 64 * U * z.abs(), out, ("gradient", g))
            want, lim = a.t() @ d, (n + 4) * U * (a.abs().t() @ d.abs())
            close(dW[g], want.t() if tb else want, lim.t() if tb else lim, out, ("dW", g))
            at += n
        for f in (c_fine, k_fine, z_fine, w_fine):
            f()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("sizes,N,K", [([5, 0, 90, 33], 96, 64), ([300, 1000], 776, 264), ([7, 8], 33, 41)])
def test_one_matrix_for_all_groups(gs, dtype, sizes, N, K):
    """A distance of zero between the groups' B: the groups share it, each with its own bias."""
    G, rows = len(sizes), sum(sizes)
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32), device="cuda")
    for tb in (0, 1):
        A, W, bias = draw((rows, K), dtype, 1), draw((N, K) if tb else (K, N), dtype, 2, 1 / math.sqrt(K)), draw((G, N), dtype, 3, 0.5)
        C = torch.empty((rows, N), dtype=TORCH[dtype], device="cuda")
        gs.grouped_gemm(gs.grouped_problem(dtype, G, rows, N, K, tb, dtype), off, A, W.expand(G, *W.shape), C, bias=bias)
        b = bias.double().repeat_interleave(torch.tensor(sizes, device="cuda"), 0)
        a, w = A.double(), W.double().t() if tb else W.double()
        close(C, a @ w + b, (K + 4) * U * (a.abs() @ w.abs() + b.abs()), dtype, tb)


def test_odd_output_widths_of_many_groups(gs):
    """Rows that are no whole cache lines, of outputs on both sides of the sizes from which they are stored through the L2."""
    for G, rows, N, K in ((64, 5000, 65, 40), (8, 40000, 1001, 72)):
        sizes = [rows // G] * G
        off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32), device="cuda")
        n = sum(sizes)
        A, W = draw((n, K), "bf16", 1), draw((G, K, N), "bf16", 2, 1 / math.sqrt(K))
        C, fine = guarded((n, N), "bf16", 0)
        gs.grouped_gemm(gs.grouped_problem("bf16", G, n, N, K, 0, "bf16"), off, A, W, C)
        a, w = A.double().view(G, -1, K), W.double()
        close(C, torch.bmm(a, w).view(n, N), (K + 4) * U * torch.bmm(a.abs(), w.abs()).view(n, N), "bf16", G)
        fine()
