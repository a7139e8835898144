"""What the gated layers, the scores and the distillation loss refuse, on the host, before anything is launched (no GPU needed)."""
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


def test_gated(gs, at):
    def run(p, act=3, A=True, B=True, C=True, lda=64, ldb=64, far=4096, ldc=64, Z=None, ldz=64, far_z=4096, bias=None):
        return gs.lib.gensor_gated_gemm(ctypes.byref(p), act, 1.0, at if A else None, lda, at if B else None, ldb, far, bias, at if C else None, ldc, Z, ldz, far_z, None)
    ok = gs.gemm_problem("f16", 64, 64, 64)
    for kw in (dict(act=4), dict(act=-1), dict(A=False), dict(B=False), dict(C=False), dict(lda=63), dict(ldb=63), dict(ldc=63), dict(far=-1), dict(Z=at),
               dict(Z=at + 256, ldz=63), dict(Z=at + 256, far_z=-64), dict(Z=at + 256, far_z=0), dict(Z=at + 256, far_z=4095), dict(Z=at + 256, ldz=127, far_z=64),
               dict(Z=at - 4096 * 4)):
        assert run(ok, **kw) == INVALID, kw
    for M, N, K in ((0, 64, 64), (64, -1, 64), (64, 64, 0)):
        assert run(gs.gemm_problem("f16", M, N, K)) == INVALID
    assert run(gs.gemm_problem("f16", 64, 64, 64, batch=2)) == INVALID and run(gs.gemm_problem("f16", 64, 64, 64, 1, 0)) == INVALID
    assert run(gs.gemm_problem("f16", 64, 64, 64, out_dtype="bf16")) == UNSUPPORTED
    assert run(gs.gemm_problem("f16", 64, 2 ** 30, 64), ldb=2 ** 30, ldc=2 ** 30) == UNSUPPORTED
    assert run(ok, lda=2 ** 28) == UNSUPPORTED and run(ok, far=2 ** 30) == UNSUPPORTED
    assert run(ok, Z=at + 256, ldz=2 ** 28, far_z=2 ** 40) == UNSUPPORTED

    def grad(p=ok, act=3, A=True, Z=at, dZ=at + 1024, ldz=64, far_z=4096, ldd=64, far_d=4096, H=None, ldh=64, lda=64, ldb=64):
        return gs.lib.gensor_gated_act_grad(ctypes.byref(p), act, 1.0, at if A else None, lda, at, ldb, Z, ldz, far_z, dZ, ldd, far_d, H, ldh, None)
    for kw in (dict(act=9), dict(A=False), dict(Z=None), dict(dZ=None), dict(ldz=63), dict(ldd=63), dict(far_z=100), dict(far_d=100), dict(lda=63), dict(ldb=63),
               dict(H=at + 512, ldh=63), dict(H=at), dict(H=at + 1024), dict(H=at + 4096 * 4), dict(dZ=at, ldd=65), dict(dZ=at, far_d=5000), dict(dZ=at + 4096 * 4), dict(Z=at + 4096 * 4, dZ=at)):
        assert grad(**kw) == INVALID, kw


def test_scores(gs, at):
    def run(dtype=1, T=8, V=100, D=64, X=True, W=True, targets=True, ldx=64, ldw=64, scale=1.0, logprob=True, lse=True, top=0, index=None, values=None, ws=True, room=4096):
        return gs.lib.gensor_logprobs(dtype, T, V, D, at if X else None, ldx, at if W else None, ldw, scale, at if targets else None, -100, at if logprob else None,
                                      at if lse else None, None, top, index, values, at if ws else None, room, None)
    both = dict(index=at, values=at)
    for kw in (dict(dtype=7), dict(T=0), dict(V=-1), dict(D=0), dict(X=False), dict(W=False), dict(targets=False), dict(ldx=63), dict(ldw=63), dict(logprob=False, lse=False),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(top=-1, **both), dict(top=65, **both), dict(V=5, top=6, **both),
               dict(top=3), dict(top=3, index=at), dict(top=3, values=at), dict(top=3, index=at + 4, values=at), dict(index=at, values=at)):
        assert run(**kw) == INVALID, kw
    assert run(ws=False) == WORKSPACE and run(room=100) == WORKSPACE and run(T=2 ** 30) == UNSUPPORTED
    assert gs.logprobs_workspace_bytes("f16", 8, 100, 64, 101) == 0 and gs.logprobs_workspace_bytes("f16", 8, 100, 64, 65) == 0
    assert gs.logprobs_workspace_bytes("f16", 0, 100, 64, 0) == 0


def test_teacher(gs, at):
    def forward(dtype=1, T=8, V=100, D=64, X=True, W=True, ldx=64, ldw=64, scale=1.0, k=4, index=at, teacher=at, normalize=1, loss=True, lse=True, ws=True, room=4096):
        return gs.lib.gensor_distill_forward(dtype, T, V, D, at if X else None, ldx, at if W else None, ldw, scale, k, index, teacher, normalize, at if loss else None,
                                             at if lse else None, at if ws else None, room, None)

    def backward(dtype=1, T=8, V=100, D=64, X=True, W=True, ldx=64, ldw=64, scale=1.0, k=4, index=at, teacher=at, normalize=1, lse=True, dloss=True, dX=True, dW=True, lddx=64,
                 lddw=64, ws=True, room=4096):
        return gs.lib.gensor_distill_backward(dtype, T, V, D, at if X else None, ldx, at if W else None, ldw, scale, k, index, teacher, normalize, at if lse else None,
                                              at if dloss else None, at if dX else None, lddx, at if dW else None, lddw, at if ws else None, room, None)
    for kw in (dict(dtype=7), dict(T=0), dict(V=-1), dict(D=0), dict(X=False), dict(W=False), dict(ldx=63), dict(ldw=63), dict(scale=0.0), dict(scale=float("inf")), dict(k=0),
               dict(k=257), dict(index=None), dict(index=at + 4), dict(teacher=None), dict(normalize=2)):
        assert forward(**kw) == INVALID and backward(**kw) == INVALID, kw
    assert forward(loss=False, lse=False) == INVALID
    for kw in (dict(lse=False), dict(dloss=False), dict(dX=False, dW=False), dict(lddx=63), dict(lddw=63)):
        assert backward(**kw) == INVALID, kw
    for run in (forward, backward):
        assert run(ws=False) == WORKSPACE and run(room=100) == WORKSPACE and run(T=2 ** 30) == UNSUPPORTED


def test_workspaces_of_many_shapes(gs):
    """384 MiB of logits of a piece at most, or one row of tiles' where that is more; and the distillation's beside the cross entropy's."""
    import random
    rng = random.Random(2)
    for _ in range(60):
        dtype = rng.choice(["f16", "bf16", "f32"])
        T, V, D = (int(10 ** rng.uniform(0, e)) for e in (4.5, 5.3, 3.5))
        top, k = rng.randint(0, min(V, 64)), rng.randint(1, 256)
        n = gs.logprobs_workspace_bytes(dtype, T, V, D, top)
        # sums: 16 bytes of a slab of 16 rows or more; maxima: 4 of as many; both of whole tiles
        rows = V + 256
        assert 24 * T <= n <= 24 * T + (max(3 * 2 ** 27, 1024 * T) if top else 0) + T * rows // 16 * 20 + 4096
        assert gs.distill_workspace_bytes(dtype, T, V, D, k) <= 28 * T + T * rows // 16 * 16 + 4096
        head = gs.distill_workspace_bytes(dtype, T, V, D, k, backward=True) - gs.xent_workspace_bytes(dtype, T, V, D, backward=True)
        assert 4 * T + 8 * T * k <= head <= 8 * T * (k + 1) + 256
    assert gs.distill_workspace_bytes("f16", 8, 100, 64, 0) == 0 and gs.distill_workspace_bytes("f16", 8, 100, 64, 257, backward=True) == 0


def test_binding_checks_shapes_and_types(gs):
    import torch
    p = gs.gemm_problem("f16", 4, 8, 16)
    A, B, C = torch.zeros(4, 16, dtype=torch.float16), torch.zeros(2, 16, 8, dtype=torch.float16), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="A: "):               # not on the device
        gs.gated_gemm(p, A, B, C)
    with pytest.raises(ValueError, match="act: "):
        gs.gated_gemm(p, A, B, C, act="tanh")
    with pytest.raises(ValueError, match="X: "):
        gs.logprobs(torch.zeros(3, 4, dtype=torch.float64), torch.zeros(5, 4, dtype=torch.float64))
    with pytest.raises(ValueError, match="X: "):
        gs.distill_forward(torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, 2, dtype=torch.int64), torch.zeros(3, 2), None, None)


def test_tensors_of_another_device_are_refused(gs, monkeypatch):
    monkeypatch.setattr(gs, "_current", (lambda: 1, lambda device: 100 + device))

    class On:
        def __init__(self, n):
            self.n, self.device, self.device_index, self.cuda_stream = n, f"cuda:{n}", n, 7

        def get_device(self):
            return self.n
    assert gs._on_current_device(None, A=On(1), B=None) == 101 and gs._on_current_device(On(1), A=On(1)) == 7
    with pytest.raises(ValueError, match="B: "):
        gs._on_current_device(None, A=On(1), B=On(0))
    with pytest.raises(ValueError, match="stream: "):
        gs._on_current_device(On(0), A=On(1))


def test_library_exports_what_the_header_declares(gs, tmp_path):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gensor_lm.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(gensor_[a-z0-9_]+)\s*\(", text))
    assert names == set(gs.LM_EXPORTS) and not names & (set(gs.EXPORTS) | set(gs.FUSED_EXPORTS))
    raw = ctypes.CDLL(gs.LIB_PATH)
    for n in names:
        assert getattr(raw, n) is not None, n
    src = tmp_path / "sz.c"
    src.write_text('#include "gensor_lm.h"\n#include <stdio.h>\nint main(void){printf("%d %d\\n", GENSOR_TOP_MAX, GENSOR_TEACHER_MAX);return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split() == [str(gs.TOP_MAX), str(gs.TEACHER_MAX)]
