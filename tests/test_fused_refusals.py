"""What the products that are consumed in place refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    return binding


@pytest.fixture(scope="module")
def at():
    buf = ctypes.create_string_buffer(4096)
    at.keep = buf
    return (ctypes.addressof(buf) + 255) // 256 * 256


def fused(gs, at, p, e=None, A=True, B=True, C=True, lda=64, ldb=64, ldc=64):
    return gs.lib.gensor_gemm_fused(ctypes.byref(p), ctypes.byref(e) if e else None, 1.0, at if A else None, lda, at if B else None, ldb, at if C else None, ldc,
                                    None, 0, None)


def epilogue(gs, **k):
    e = gs.Epilogue()
    for name, v in k.items():
        setattr(e, name, v)
    return e


def test_product(gs, at):
    ok = gs.gemm_problem("f16", 64, 64, 64)
    for kw in (dict(A=False), dict(B=False), dict(C=False), dict(lda=63), dict(ldb=63), dict(ldc=63)):
        assert fused(gs, at, ok, **kw) == INVALID, kw
    for M, N, K in ((0, 64, 64), (64, -1, 64), (64, 64, 0)):
        assert fused(gs, at, gs.gemm_problem("f16", M, N, K)) == INVALID
    assert fused(gs, at, gs.gemm_problem("f16", 64, 64, 64, batch=2)) == INVALID            # not one product
    assert fused(gs, at, gs.gemm_problem("f16", 64, 64, 64, 1, 1)) == UNSUPPORTED
    assert fused(gs, at, gs.gemm_problem("f16", 64, 64, 64, out_dtype="bf16")) == UNSUPPORTED
    assert fused(gs, at, gs.gemm_problem("f16", 64, 2 ** 31 - 100, 64), ldb=2 ** 31, ldc=2 ** 31) == UNSUPPORTED
    assert fused(gs, at, ok, lda=2 ** 28) == UNSUPPORTED                                    # rows beyond 32-bit offsets
    assert fused(gs, at, ok, epilogue(gs, preact=at + 256, ld_preact=2 ** 28)) == UNSUPPORTED


def test_epilogue(gs, at):
    ok = gs.gemm_problem("f16", 64, 64, 64)
    for kw in (dict(act=4), dict(act=-1), dict(grad=2), dict(grad=1, act=1), dict(preact=at, ld_preact=64), dict(preact=at + 256, ld_preact=63),
               dict(residual=at, ld_residual=10), dict(grad=1, preact=at, ld_preact=64, bias=at), dict(grad=1, preact=at, ld_preact=64, residual=at, ld_residual=64)):
        assert fused(gs, at, ok, epilogue(gs, **kw)) == INVALID, kw


def test_groups(gs, at):
    def run(p, offsets=True, A=True, lda=64, ldb=64, stride=4096, ldc=64, e=None):
        return gs.lib.gensor_grouped_gemm(ctypes.byref(p), at if offsets is True else offsets, ctypes.byref(e) if e else None, 1.0, at if A else None, lda, at, ldb, stride,
                                          at, ldc, None)
    ok = gs.grouped_problem("f16", 4, 64, 64, 64)
    assert run(gs.grouped_problem("f16", 4, 0, 64, 64)) == 0                                # no rows: nothing to do
    for kw in (dict(offsets=None), dict(offsets=at + 1), dict(A=False), dict(lda=63), dict(ldb=63), dict(ldc=63), dict(stride=-1), dict(e=epilogue(gs, act=9))):
        assert run(ok, **kw) == INVALID, kw
    assert run(gs.gemm_problem("f16", 64, 64, 64)) == INVALID                               # not grouped
    assert run(gs.grouped_problem("f16", 0, 64, 64, 64)) == INVALID
    assert run(gs.grouped_problem("f16", 2, -1, 64, 64)) == INVALID
    t = gs.grouped_problem("f16", 4, 64, 64, 64)
    t.transA = 1
    assert run(t) == INVALID

    def wgrad(p, offsets=True, dW=True, lda=64, lddy=64, lddw=64, stride=4096):
        return gs.lib.gensor_grouped_wgrad(ctypes.byref(p), at if offsets else None, at, lda, at, lddy, at if dW else None, lddw, stride, None)
    for kw in (dict(offsets=False), dict(dW=False), dict(lda=63), dict(lddy=63), dict(lddw=63), dict(stride=4095), dict(stride=-1)):
        assert wgrad(ok, **kw) == INVALID, kw

    def bias(dtype=1, out=1, groups=4, rows=64, N=64, dY=True, ld=64, offsets=True, db=True):
        return gs.lib.gensor_bias_grad(dtype, out, groups, rows, N, at if dY else None, ld, at if offsets else None, at if db else None, None, 0, None)
    for kw in (dict(dtype=3), dict(out=-1), dict(groups=0), dict(rows=-1), dict(N=0), dict(dY=False), dict(ld=63), dict(offsets=False), dict(db=False)):
        assert bias(**kw) == INVALID, kw
    assert bias(out=2) == UNSUPPORTED and bias(groups=70000) == UNSUPPORTED


def test_cross_entropy(gs, at):
    def forward(dtype=1, T=8, V=100, D=64, X=True, W=True, targets=True, ldx=64, ldw=64, loss=True, lse=True, ws=True, room=4096):
        return gs.lib.gensor_xent_forward(dtype, T, V, D, at if X else None, ldx, at if W else None, ldw, at if targets else None, -100, at if loss else None,
                                          at if lse else None, at if ws else None, room, None)
    for kw in (dict(dtype=7), dict(T=0), dict(V=-1), dict(D=0), dict(X=False), dict(W=False), dict(targets=False), dict(ldx=63), dict(ldw=63),
               dict(loss=False, lse=False)):
        assert forward(**kw) == INVALID, kw
    assert forward(ws=False) == WORKSPACE and forward(room=100) == WORKSPACE
    assert forward(T=2 ** 30) == UNSUPPORTED

    def backward(targets=True, lse=True, dloss=True, dX=True, dW=True, lddx=64, lddw=64, room=4096):
        return gs.lib.gensor_xent_backward(1, 8, 100, 64, at, 64, at, 64, at if targets else None, -100, at if lse else None, at if dloss else None,
                                           at if dX else None, lddx, at if dW else None, lddw, at, room, None)
    for kw in (dict(targets=False), dict(lse=False), dict(dloss=False), dict(dX=False, dW=False), dict(lddx=63), dict(lddw=63)):
        assert backward(**kw) == INVALID, kw
    assert backward(room=300) == WORKSPACE


def test_workspaces(gs):
    assert gs.gemm_fused_workspace_bytes(gs.gemm_problem("bf16", 256, 512, 8192, 0, 1)) > 0
    assert gs.lib.gensor_gemm_fused_workspace_bytes(None) == 0
    assert gs.lib.gensor_xent_workspace_bytes(1, 0, 10, 10, 0) == 0 and gs.lib.gensor_xent_workspace_bytes(9, 5, 10, 10, 1) == 0
    assert gs.bias_grad_workspace_bytes(1, 10, 10) == 0 and gs.bias_grad_workspace_bytes(1, 8192, 64) > 0
    small, large = (gs.xent_workspace_bytes("f16", T, 50257, 768, backward=True) for T in (64, 8192))
    assert 50257 * 64 * 2 < small < large < 400 * 2 ** 20                                   # a batch's logits would be 823 MB


def test_workspaces_of_many_shapes(gs):
    """What a call needs is found for any shape, within the limits that the gradient's pieces have: 256 MiB of G, 64 of partial tiles, dX's sums and X."""
    import random
    rng = random.Random(1)
    for _ in range(60):
        dtype = rng.choice(["f16", "bf16", "f32"])
        T, V, D = (int(10 ** rng.uniform(0, e)) for e in (4.5, 5.3, 3.5))
        es, forward, backward = (4 if dtype == "f32" else 2), gs.xent_workspace_bytes(dtype, T, V, D), gs.xent_workspace_bytes(dtype, T, V, D, backward=True)
        assert 8 * T <= forward <= 2 * 4 * T * (V // 16 + 2) + 4 * T + 1024
        vec = 16 // es                                       # G's rows are whole vectors
        least = (T + vec - 1) // vec * vec * min(V, 256) * es
        assert least <= backward <= max(2 ** 28, least) + 2 ** 26 + T * D * 4 + (T + 8) * D * es + 4096


def test_binding_checks_shapes_and_types(gs):
    import torch
    p = gs.gemm_problem("f16", 4, 8, 16)
    A, B, C = torch.zeros(4, 16, dtype=torch.float16), torch.zeros(16, 8, dtype=torch.float16), torch.zeros(4, 8)
    with pytest.raises(ValueError):                          # not on the device
        gs.gemm_fused(p, A, B, C)
    with pytest.raises(ValueError):
        gs.gemm_fused(p, A, B, C, act="tanh")
    with pytest.raises(ValueError):
        gs.bias_grad(torch.zeros(3, 4, dtype=torch.float64), torch.zeros(4))


def test_library_exports_what_the_header_declares(gs, tmp_path):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gensor_fused.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(gensor_[a-z0-9_]+)\s*\(", text))
    assert names == set(gs.FUSED_EXPORTS) and not names & set(gs.EXPORTS)
    raw = ctypes.CDLL(gs.LIB_PATH)
    for n in names:
        assert getattr(raw, n) is not None, n
    src = tmp_path / "sz.c"
    src.write_text('#include "gensor_fused.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void){printf("%zu %zu %zu %zu %d\\n",'
                   'sizeof(gensor_epilogue), offsetof(gensor_epilogue, bias), offsetof(gensor_epilogue, ld_preact),'
                   'offsetof(gensor_epilogue, ld_residual), GENSOR_ACT_SILU);return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    e = gs.Epilogue
    assert got == [ctypes.sizeof(e), e.bias.offset, e.ld_preact.offset, e.ld_residual.offset, gs.ACT["silu"]]
