"""Products that are consumed in place (epilogue with bias, activation and residual; products grouped by expert; their gradients) against the
definitions in 64 bits.

Tolerances.  u = 2^-24 is the unit roundoff of fp32.  A product's sum of K terms in any order is off by at most (K + 1) u sum|a||b| (first
order); the activations have slopes of at most 1.13 and are evaluated to within 16 u |z| (gelu and silu: an exponential whose argument is
off by 4 u |argument|, the sigmoid's derivative times its argument stays below 0.3); a result is rounded once to its type."""
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


def guarded(shape, dtype, pad=0):
    """An output between values that nothing may touch: (view, check)."""
    rows, cols = shape
    flat = torch.full((rows + 2, cols + pad), 7.0, dtype=TORCH[dtype], device="cuda")
    view = flat[1:1 + rows, :cols]

    def untouched():
        assert bool((flat[0] == 7).all()) and bool((flat[1 + rows:] == 7).all()) and bool((flat[1:1 + rows, cols:] == 7).all())
    return view, untouched


def act64(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    z = z.detach().clone().requires_grad_(True)
    (torch.relu(z) if act == "relu" else act64(z, act)).sum().backward()
    return z.grad


def close(got, want, bound, dtype, what=""):
    got = got.double()
    limit = bound + ROUND[dtype] * want.abs() + TINY[dtype]
    bad = ~((got - want).abs() <= limit)
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got - want).abs() / limit).nan_to_num(1e9).max()), torch.nonzero(bad)[:3].tolist())


def problem_operands(dtype, M, N, K, ta, tb, pad, seed):
    A = draw((K, M) if ta else (M, K), dtype, seed, pad=pad)
    B = draw((N, K) if tb else (K, N), dtype, seed + 1, 1 / math.sqrt(K), pad=pad)
    a, b = A.double(), B.double()
    return A, B, (a.t() if ta else a), (b.t() if tb else b)


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


SHAPES = [(1, 1, 1), (1, 96, 64), (1, 640, 768), (2, 7, 3), (5, 33, 17), (16, 256, 200), (31, 64, 129), (64, 64, 64), (65, 130, 257), (100, 1000, 72),
          (129, 255, 513), (256, 256, 256), (257, 384, 1024), (513, 768, 520), (1030, 1100, 190), (128, 128, 4096), (2048, 2304, 320), (4100, 768, 1536)]


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_forward(gs, dtype, out, M, N, K):
    """Every activation with bias, kept values and residual in some combination, both layouts of B, rows of any pitch."""
    for i, (act, tb, bias, keep, residual, pad, alpha) in enumerate([("gelu", 0, True, True, False, 0, 1.0), ("none", 1, True, False, True, 8, 1.0),
                                                                     ("silu", 0, False, True, True, 3, -0.75), ("relu", 1, True, False, False, 1, 2.0)]):
        A, B, a, b = problem_operands(dtype, M, N, K, 0, tb, pad, 100 * i + M)
        p = gs.gemm_problem(dtype, M, N, K, 0, tb, out_dtype=out)
        bv = draw((N,), dtype, 5, 0.5) if bias else None
        R = draw((M, N), out, 6, 1.0, pad) if residual else None
        C, fine = guarded((M, N), out, pad)
        Z, z_fine = guarded((M, N), out, pad) if keep else (None, None)
        gs.gemm_fused(p, A, B, C, bias=bv, act=act, preact=Z, residual=R, alpha=alpha, workspace=workspace(gs.gemm_fused_workspace_bytes(p)))
        z = alpha * (a @ b) + (bv.double() if bias else 0)
        e = (K + 4) * U * (abs(alpha) * (a.abs() @ b.abs()) + (bv.double().abs() if bias else 0))
        y = act64(z, act)
        close(C, y + (R.double() if residual else 0), 1.13 * e + 16 * U * z.abs() + (U * R.double().abs() if residual else 0), out, (act, tb))
        fine()
        if keep:
            close(Z, z, e, out, "kept")
            z_fine()


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("M,N,K", [(1, 5, 3), (33, 65, 40), (129, 256, 513), (520, 776, 264), (2050, 1024, 512)])
def test_transposed_a(gs, dtype, out, M, N, K):
    A, B, a, b = problem_operands(dtype, M, N, K, 1, 0, 0, M)
    p = gs.gemm_problem(dtype, M, N, K, 1, 0, out_dtype=out)
    R = draw((M, N), out, 3)
    C, fine = guarded((M, N), out)
    gs.gemm_fused(p, A, B, C, residual=R, workspace=workspace(gs.gemm_fused_workspace_bytes(p)))
    close(C, a @ b + R.double(), (K + 4) * U * (a.abs() @ b.abs()) + U * R.double().abs(), out)
    fine()


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("M,N,K", [(1, 3, 2), (1, 768, 96), (37, 65, 40), (130, 257, 513), (512, 776, 264), (2050, 1536, 384)])
def test_activation_gradient(gs, dtype, out, M, N, K):
    for act, tb, pad in (("gelu", 1, 0), ("silu", 0, 4), ("relu", 1, 1), ("none", 0, 0)):
        A, B, a, b = problem_operands(dtype, M, N, K, 0, tb, pad, M)
        p = gs.gemm_problem(dtype, M, N, K, 0, tb, out_dtype=out)
        Z = draw((M, N), out, 9, 2.0, pad)
        C, fine = guarded((M, N), out, pad)
        gs.gemm_act_grad(p, A, B, Z, C, act, workspace=workspace(gs.gemm_fused_workspace_bytes(p)))
        d, e = a @ b, (K + 4) * U * (a.abs() @ b.abs())
        close(C, d * slope64(Z.double(), act), 1.13 * e + 64 * U * d.abs(), out, act)
        fine()
        inplace = Z.clone() if pad == 0 else None
        if inplace is not None:                                        # over the values it reads
            gs.gemm_act_grad(p, A, B, inplace, inplace, act, workspace=workspace(gs.gemm_fused_workspace_bytes(p)))
            assert torch.equal(inplace, C)


def test_activation_gradient_against_differences(gs):
    """The pair forward and gradient: the gradient is the forward's slope, by central differences of the forward itself in fp32."""
    M, N, K = 64, 96, 1
    A, B = torch.ones((M, K), device="cuda"), torch.zeros((K, N), device="cuda")
    z = torch.linspace(-6, 6, M * N, device="cuda").reshape(M, N).contiguous()
    p = gs.gemm_problem("f32", M, N, K)
    h = 2.0 ** -5
    for act in ("gelu", "silu"):
        up, down, one = (torch.empty((M, N), device="cuda") for _ in range(3))
        for sign, o in ((h, up), (-h, down)):
            # identity product: row r of A picks nothing, the values come as a residual of a product without activation, then through one
            zz = torch.empty((M, N), device="cuda")
            gs.gemm_fused(p, A, B, zz, residual=z + sign)
            eye = torch.eye(N, device="cuda")
            gs.gemm_fused(gs.gemm_problem("f32", M, N, N), zz, eye, o, act=act)
        gs.gemm_act_grad(p, A, torch.ones((K, N), device="cuda"), z, one, act)
        # error of the difference: h^2/6 times the third derivative (below 2 for both), and rounding 8 u |y| / h
        assert float(((up - down) / (2 * h) - one).abs().max()) <= 2 * h * h / 6 + 8 * U * 7 / h


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_extreme_values(gs, dtype):
    """Infinities, NaN and the type's largest values before the activation; relu and its gradient at zero."""
    big = float(torch.finfo(TORCH[dtype]).max)
    z = torch.tensor([[0.0, -0.0, math.inf, -math.inf, math.nan, big, -big, 1.0]], device="cuda").to(TORCH[dtype]).repeat(3, 1).contiguous()
    A, B = torch.zeros((3, 8), dtype=TORCH[dtype], device="cuda"), torch.zeros((8, 8), dtype=TORCH[dtype], device="cuda")
    p = gs.gemm_problem(dtype, 3, 8, 8, out_dtype=dtype)
    for act in ("none", "relu", "gelu", "silu"):
        y = torch.empty_like(z)
        gs.gemm_fused(p, A, B, y, bias=z[0].contiguous(), act=act)
        zz = z[0].double()
        # -inf: relu 0; the others -inf * 0, which is NaN in their definitions too
        want = {"none": zz, "relu": torch.where(zz < 0, torch.zeros_like(zz), zz), "gelu": act64(zz, "silu"), "silu": act64(zz, "silu")}[act]
        want[-1] = act64(torch.ones((), dtype=torch.float64, device="cuda"), act)
        want[6] = want[6] if act == "none" else 0.0
        got = y.double()
        for row in got:
            assert torch.equal(torch.isnan(row), torch.isnan(want)), (act, row, want)
            ok = ~torch.isnan(want)
            assert bool(((row[ok] == want[ok]) | ((row[ok] - want[ok]).abs() <= ROUND[dtype] * want[ok].abs() + 1e-6)).all()), (act, row, want)
        g = torch.empty_like(z)
        ones = torch.ones((8, 8), dtype=TORCH[dtype], device="cuda")
        gs.gemm_act_grad(p, torch.ones_like(A), ones, z, g, act)
        if act == "relu":
            assert g[0].tolist() == [0.0, 0.0, 8.0, 0.0, 0.0, 8.0, 0.0, 8.0]
        if act in ("gelu", "silu"):
            assert g[0][:2].tolist() == [4.0, 4.0] and float(g[0][5]) == 8.0 and float(g[0][6]) == 0.0


def test_residual_in_place_and_no_workspace(gs):
    """C may be its own residual; without a workspace a split product runs unsplit, with the same result to rounding."""
    M, N, K = 256, 512, 8192
    A, B, a, b = problem_operands("bf16", M, N, K, 0, 1, 0, 1)
    p = gs.gemm_problem("bf16", M, N, K, 0, 1, out_dtype="f32")
    assert gs.gemm_fused_workspace_bytes(p) > 0
    R = draw((M, N), "f32", 3)
    for ws in (None, workspace(gs.gemm_fused_workspace_bytes(p)), workspace(4096)):
        C = R.clone()
        gs.gemm_fused(p, A, B, C, residual=C, workspace=ws)
        close(C, a @ b + R.double(), (K + 4) * U * (a.abs() @ b.abs()) + U * R.double().abs(), "f32")


def offsets_of(sizes, lead=0):
    return torch.tensor(np.concatenate([[lead], lead + np.cumsum(sizes)]).astype(np.int32), device="cuda")


GROUPS = [[1], [0], [5], [0, 0, 3], [1, 1, 1, 1], [0, 17, 0, 64, 1, 130, 0], [256, 0, 257, 300], [1000, 3, 0, 500, 129], [2] * 70 + [0] * 60 + [40]]


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("sizes", GROUPS, ids=lambda s: "%dx%d" % (len(s), sum(s)))
@pytest.mark.parametrize("N,K", [(96, 64), (33, 45), (520, 264)])
def test_grouped(gs, dtype, out, sizes, N, K):
    """Forward with each group's bias, the gradient of the rows and of each group's weights and bias; rows that belong to no group stay."""
    G, lead, tail = len(sizes), 2, 3
    rows = sum(sizes) + lead + tail
    off = offsets_of(sizes, lead)
    for tb, act in ((0, "gelu"), (1, "none")):
        A = draw((rows, K), dtype, 1)
        A[:lead] = math.nan                                            # of no group: never read
        A[rows - tail:] = math.nan
        W = draw((G, N, K) if tb else (G, K, N), dtype, 2, 1 / math.sqrt(K))
        bias, dY = draw((G, N), dtype, 3, 0.5), draw((rows, N), dtype, 4)
        dY[:lead] = math.nan
        dY[rows - tail:] = math.nan
        p = gs.grouped_problem(dtype, G, rows, N, K, tb, out)
        back = gs.grouped_problem(dtype, G, rows, K, N, 1 - tb, out)
        C, fine = guarded((rows, N), out)
        Z, z_fine = guarded((rows, N), out)
        dA, da_fine = guarded((rows, K), out)
        C.fill_(3.0), Z.fill_(3.0), dA.fill_(3.0)
        dW, db = torch.full((G,) + tuple(W.shape[1:]), 9.0, dtype=TORCH[out], device="cuda"), torch.full((G, N), 9.0, dtype=TORCH[out], device="cuda")
        gs.grouped_gemm(p, off, A, W, C, bias=bias, act=act, preact=Z)
        gs.grouped_gemm(back, off, dY, W, dA)
        gs.grouped_wgrad(p, off, A, dY, dW)
        gs.bias_grad(dY, db, offsets=off, workspace=workspace(gs.bias_grad_workspace_bytes(G, rows, N, dtype)))
        for f in (fine, z_fine, da_fine):
            f()
        at = lead
        for g, n in enumerate(sizes):
            w = W[g].double()
            w = w.t() if tb else w
            a, d, r = A[at:at + n].double(), dY[at:at + n].double(), slice(at, at + n)
            z, e = a @ w + bias[g].double(), (K + 4) * U * (a.abs() @ w.abs() + bias[g].double().abs())
            close(Z[r], z, e, out, ("kept", g))
            close(C[r], act64(z, act), 1.13 * e + 16 * U * z.abs(), out, ("forward", g))
            close(dA[r], d @ w.t(), (N + 4) * U * (d.abs() @ w.t().abs()), out, ("dA", g))
            want, lim = a.t() @ d, (n + 4) * U * (a.abs().t() @ d.abs())
            close(dW[g], want.t() if tb else want, lim.t() if tb else lim, out, ("dW", g))
            close(db[g], d.sum(0), (n + 4) * U * d.abs().sum(0), out, ("db", g))
            at += n
        for t in (C, Z, dA):
            assert bool((t[:lead] == 3).all()) and bool((t[at:] == 3).all())


def test_grouped_activation_gradient_and_residual(gs):
    sizes, N, K = [40, 0, 90, 3], 264, 96
    G, rows = len(sizes), sum(sizes)
    off = offsets_of(sizes)
    A, W, Z, R = draw((rows, K), "bf16", 1), draw((G, K, N), "bf16", 2, 0.1), draw((rows, N), "bf16", 3), draw((rows, N), "bf16", 4, 1.0, 2)
    p = gs.grouped_problem("bf16", G, rows, N, K, 0, "bf16")
    dz, y = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, N), dtype=torch.bfloat16, device="cuda")
    gs.grouped_act_grad(p, off, A, W, Z, dz, "gelu")
    gs.grouped_gemm(p, off, A, W, y, residual=R)
    at = 0
    for g, n in enumerate(sizes):
        r = slice(at, at + n)
        d, e = A[r].double() @ W[g].double(), (K + 4) * U * (A[r].double().abs() @ W[g].double().abs())
        close(dz[r], d * slope64(Z[r].double(), "gelu"), 1.13 * e + 64 * U * d.abs(), "bf16")
        close(y[r], d + R[r].double(), e + U * R[r].double().abs(), "bf16")
        at += n


def test_grouped_large_tiles(gs):
    """Groups of many tiles, whose large tiles are taken, and one that ends inside a tile."""
    for dtype in ("f16", "bf16"):
        sizes, N, K = [2048, 1000, 0, 7100], 1536, 768
        G, rows = len(sizes), sum(sizes)
        off = offsets_of(sizes)
        A, W, dY = draw((rows, K), dtype, 1), draw((G, K, N), dtype, 2, 1 / math.sqrt(K)), draw((rows, N), dtype, 3)
        p = gs.grouped_problem(dtype, G, rows, N, K, 0, dtype)
        C, dW = torch.empty((rows, N), dtype=TORCH[dtype], device="cuda"), torch.empty((G, K, N), dtype=TORCH[dtype], device="cuda")
        gs.grouped_gemm(p, off, A, W, C, act="silu")
        gs.grouped_wgrad(p, off, A, dY, dW)
        at = 0
        for g, n in enumerate(sizes):
            a, w, d = A[at:at + n].double(), W[g].double(), dY[at:at + n].double()
            z = a @ w
            close(C[at:at + n], act64(z, "silu"), 1.13 * (K + 4) * U * (a.abs() @ w.abs()) + 16 * U * z.abs(), dtype, g)
            close(dW[g], a.t() @ d, (n + 4) * U * (a.abs().t() @ d.abs()), dtype, g)
            at += n


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("M,N,K", [(8192, 3072, 768), (8001, 4096, 520), (4100, 5124, 328), (8192, 768, 3072)])
def test_large_tiles(gs, dtype, out, M, N, K):
    """The tiles of large products (256 and 192 columns, whole and split), whose epilogues store in whole lines, with everything read and kept."""
    for tb in (0, 1):
        A, B, a, b = problem_operands(dtype, M, N, K, 0, tb, 0, M + tb)
        p = gs.gemm_problem(dtype, M, N, K, 0, tb, out_dtype=out)
        ws = workspace(gs.gemm_fused_workspace_bytes(p))
        d, e = a @ b, (K + 4) * U * (a.abs() @ b.abs())
        bias, R, Z = draw((N,), dtype, 5, 0.5), draw((M, N), out, 6), draw((M, N), out, 7)
        C, fine = guarded((M, N), out)
        kept, kept_fine = guarded((M, N), out)
        gs.gemm_fused(p, A, B, C, bias=bias, act="gelu", preact=kept, residual=R, workspace=ws)
        z, ez = d + bias.double(), e + (K + 4) * U * bias.double().abs()
        close(kept, z, ez, out, "kept")
        close(C, act64(z, "gelu") + R.double(), 1.13 * ez + 16 * U * z.abs() + U * R.double().abs(), out, "forward")
        gs.gemm_act_grad(p, A, B, Z, C, "silu", workspace=ws)
        close(C, d * slope64(Z.double(), "silu"), 1.13 * e + 64 * U * d.abs(), out, "gradient")
        fine(), kept_fine()


def test_large_tiles_beside_rows_of_any_pitch(gs):
    """Aligned operands, but C, the residual and the kept values in rows that start anywhere."""
    M, N, K = 4100, 3072, 768
    A, B, a, b = problem_operands("bf16", M, N, K, 0, 1, 0, 3)
    p = gs.gemm_problem("bf16", M, N, K, 0, 1, out_dtype="bf16")
    d, e = a @ b, (K + 4) * U * (a.abs() @ b.abs())
    for c_pad, r_pad in ((0, 5), (3, 0), (1, 7)):
        R = draw((M, N), "bf16", 6, 1.0, r_pad)
        C, fine = guarded((M, N), "bf16", c_pad)
        gs.gemm_fused(p, A, B, C, residual=R, workspace=workspace(gs.gemm_fused_workspace_bytes(p)))
        close(C, d + R.double(), e + U * R.double().abs(), "bf16", (c_pad, r_pad))
        gs.gemm_act_grad(p, A, B, R, C, "gelu", workspace=workspace(gs.gemm_fused_workspace_bytes(p)))
        close(C, d * slope64(R.double(), "gelu"), 1.13 * e + 64 * U * d.abs(), "bf16", (c_pad, r_pad))
        fine()


def test_elements_beyond_32_bits(gs):
    """Results of more than 2^31 elements: the last rows of a product with everything beside it, and of a grouped one."""
    M, N, K = 70000, 32768, 64
    A, B, bias = draw((M, K), "bf16", 1), draw((N, K), "bf16", 2, 0.1), draw((N,), "bf16", 3)
    p = gs.gemm_problem("bf16", M, N, K, 0, 1, out_dtype="bf16")
    C, kept = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    C[-300:] = 0.25
    gs.gemm_fused(p, A, B, C, bias=bias, act="relu", preact=kept, residual=C)
    rows = slice(M - 300, M)
    z, e = A[rows].double() @ B.double().t() + bias.double(), (K + 4) * U * (A[rows].double().abs() @ B.double().abs().t() + bias.double().abs())
    close(kept[rows], z, e, "bf16")
    close(C[rows], act64(z, "relu") + 0.25, e + U * z.abs(), "bf16")
    sizes = [40000, 29990, 10]
    W = draw((3, N, K), "bf16", 4, 0.1)
    gs.grouped_gemm(gs.grouped_problem("bf16", 3, M, N, K, 1, "bf16"), offsets_of(sizes), A, W, C)
    for g, r in ((1, slice(69700, 69990)), (2, slice(69990, 70000))):
        a, w = A[r].double(), W[g].double().t()
        close(C[r], a @ w, (K + 4) * U * (a.abs() @ w.abs()), "bf16")
    db = torch.empty((3, N), dtype=torch.float32, device="cuda")
    gs.bias_grad(kept, db, offsets=offsets_of(sizes))
    close(db[2], kept[69990:].double().sum(0), 14 * U * kept[69990:].double().abs().sum(0), "f32")


def test_groups_without_a_row(gs):
    """No rows at all: nothing to compute, and gradients of zeros."""
    p = gs.grouped_problem("f16", 3, 0, 40, 24, 0, "f16")
    A, dY, off = torch.empty((0, 24), dtype=torch.float16, device="cuda"), torch.empty((0, 40), dtype=torch.float16, device="cuda"), offsets_of([0, 0, 0])
    W, C = draw((3, 24, 40), "f16", 1), torch.empty((0, 40), dtype=torch.float16, device="cuda")
    gs.grouped_gemm(p, off, A, W, C)
    dW, db = torch.full((3, 24, 40), 5.0, dtype=torch.float16, device="cuda"), torch.full((3, 40), 5.0, dtype=torch.float16, device="cuda")
    gs.grouped_wgrad(p, off, A, dY, dW)
    gs.bias_grad(dY, db, offsets=off)
    assert bool((dW == 0).all()) and bool((db == 0).all())


def test_offsets_outside_the_rows_are_cut(gs):
    """Offsets beyond the rows, negative or decreasing: nothing outside C and dW is written."""
    rows, N, K = 100, 64, 48
    A, W, dY = draw((rows, K), "f16", 1), draw((4, K, N), "f16", 2), draw((rows, N), "f16", 3)
    p = gs.grouped_problem("f16", 4, rows, N, K, 0, "f16")
    for off in ([-5, 20, 60, 1000, 2000], [0, 50, 30, 80, 100], [2 ** 31 - 1] * 5, [-2 ** 31] * 5):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        C, fine = guarded((rows, N), "f16")
        gs.grouped_gemm(p, o, A, W, C)
        dW, w_fine = guarded((4 * K, N), "f16")
        gs.grouped_wgrad(p, o, A, dY, dW.view(4, K, N))
        db, b_fine = guarded((4, N), "f16")
        gs.bias_grad(dY, db, offsets=o)
        torch.cuda.synchronize()
        fine(), w_fine(), b_fine()


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("rows,N,pad", [(1, 1, 0), (0, 5, 0), (3, 7, 1), (100, 512, 0), (4097, 768, 8), (20000, 33, 0)])
def test_bias_grad(gs, dtype, out, rows, N, pad):
    dY = draw((rows, N), dtype, 1, pad=pad)
    want, lim = dY.double().sum(0), (rows + 4) * U * dY.double().abs().sum(0)
    need = gs.bias_grad_workspace_bytes(1, rows, N, dtype)
    for ws in (workspace(need), None, workspace(max(4, need // 3))):
        db = torch.full((N,), 9.0, dtype=TORCH[out], device="cuda")
        gs.bias_grad(dY, db, workspace=ws)
        close(db, want, lim, out)


def test_streams_and_graph(gs):
    """On the caller's stream, and captured: a replay gives what the eager call gives."""
    M, N, K = 300, 512, 256
    A, B, _, _ = problem_operands("bf16", M, N, K, 0, 1, 0, 1)
    p = gs.gemm_problem("bf16", M, N, K, 0, 1, out_dtype="bf16")
    bias, want, got = draw((N,), "bf16", 2), torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    ws = workspace(gs.gemm_fused_workspace_bytes(p))
    gs.gemm_fused(p, A, B, want, bias=bias, act="gelu", workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gs.gemm_fused(p, A, B, got, bias=bias, act="gelu", stream=side, workspace=ws)
    side.synchronize()
    assert torch.equal(want, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gs.gemm_fused(p, A, B, got, bias=bias, act="gelu", workspace=ws)
    for seed in (3, 4, 5):
        A.copy_(draw((M, K), "bf16", seed))
        graph.replay()
        torch.cuda.synchronize()
        gs.gemm_fused(p, A, B, want, bias=bias, act="gelu", workspace=ws)
        assert torch.equal(want, got)
