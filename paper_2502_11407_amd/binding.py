"""ctypes face of libgensor.so (include/gensor.h, include/gensor_fused.h and include/gensor_lm.h).  Argument marshalling only: every step
of the operators runs in the library's HIP kernels, the constructor in its C++ host code.
PyTorch is used for device memory and the current stream, nothing else.

Importing this module loads the library and raises if it has not been built
(python -m paper_2502_11407_amd.csrc.build, or __graft_entry__.build()).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgensor.so")

GENSOR_OK = 0
STATUS = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "NO_SCHEDULE", 4: "WORKSPACE", 5: "DEVICE"}
DTYPE = {"f32": 0, "f16": 1, "bf16": 2}
OP_GEMM, OP_BMM, OP_CONV2D = 0, 1, 2
ACT = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}

EXPORTS = ["gensor_hw_mi355x", "gensor_construct", "gensor_construct_trace", "gensor_predict_us",
           "gensor_num_instances", "gensor_instance_schedule", "gensor_gemm", "gensor_bmm", "gensor_conv2d",
           "gensor_workspace_bytes", "gensor_status_string", "gensor_gemm_static_scratch", "gensor_gemv", "gensor_avgpool2d"]
FUSED_EXPORTS = ["gensor_gemm_fused", "gensor_gemm_fused_workspace_bytes", "gensor_grouped_gemm", "gensor_grouped_wgrad",
                 "gensor_bias_grad", "gensor_bias_grad_workspace_bytes", "gensor_xent_forward", "gensor_xent_backward",
                 "gensor_xent_workspace_bytes"]          # include/gensor_fused.h
LM_EXPORTS = ["gensor_gated_gemm", "gensor_gated_act_grad", "gensor_logprobs", "gensor_logprobs_workspace_bytes", "gensor_distill_forward",
              "gensor_distill_backward", "gensor_distill_workspace_bytes"]               # include/gensor_lm.h
TOP_MAX, TEACHER_MAX = 64, 256


class Problem(C.Structure):
    _fields_ = [("op", C.c_int32), ("in_dtype", C.c_int32), ("out_dtype", C.c_int32),
                ("transA", C.c_int32), ("transB", C.c_int32),
                ("batch", C.c_int64), ("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64),
                ("n", C.c_int64), ("c", C.c_int64), ("h", C.c_int64), ("w", C.c_int64),
                ("k", C.c_int64), ("r", C.c_int64), ("s", C.c_int64),
                ("stride", C.c_int64), ("pad", C.c_int64)]


class Schedule(C.Structure):
    _fields_ = [("version", C.c_int32), ("kernel_id", C.c_int32),
                ("tile", (C.c_int32 * 3) * 3), ("vthread", C.c_int32 * 2),
                ("stages", C.c_int32), ("unroll", C.c_int32), ("vec_bytes", C.c_int32),
                ("direct_lds", C.c_int32), ("split_k", C.c_int32), ("wg_remap", C.c_int32),
                ("predicted_us", C.c_double), ("construct_s", C.c_double),
                ("iterations", C.c_int32), ("chains", C.c_int32), ("states_scored", C.c_int32),
                ("round_units", C.c_int32), ("seed", C.c_uint64)]

    def describe(self) -> dict:
        t = [[self.tile[d][l] for l in range(3)] for d in range(3)]
        return {"kernel_id": self.kernel_id, "tile_m": t[0], "tile_n": t[1], "tile_k": t[2],
                "vthread": [self.vthread[0], self.vthread[1]], "stages": self.stages, "unroll": self.unroll,
                "vec_bytes": self.vec_bytes, "direct_lds": self.direct_lds, "wg_remap": self.wg_remap,
                "predicted_us": self.predicted_us, "construct_s": self.construct_s,
                "iterations": self.iterations, "chains": self.chains, "states_scored": self.states_scored}


class Hw(C.Structure):
    _fields_ = [("compute_units", C.c_int32), ("simds_per_cu", C.c_int32), ("wave_size", C.c_int32),
                ("max_waves_per_wg", C.c_int32), ("lds_bytes_per_cu", C.c_int32), ("regs_per_lane", C.c_int32),
                ("lds_banks", C.c_int32), ("lds_bank_bytes", C.c_int32), ("clock_ghz", C.c_double),
                ("latency_ns", C.c_double * 3), ("bandwidth_gbs", C.c_double * 3),
                ("l2_bandwidth_gbs", C.c_double), ("mfma_tflops_16bit", C.c_double),
                ("mfma_tflops_f32", C.c_double), ("launch_us", C.c_double)]


class ConstructOpts(C.Structure):
    _fields_ = [("T0", C.c_double), ("threshold", C.c_double), ("chains", C.c_int32),
                ("keep_policy", C.c_int32), ("tiling_benefit", C.c_int32), ("no_vthread", C.c_int32),
                ("no_split_k", C.c_int32), ("greedy", C.c_int32)]


class Epilogue(C.Structure):
    _fields_ = [("act", C.c_int32), ("grad", C.c_int32), ("bias", C.c_void_p), ("preact", C.c_void_p), ("ld_preact", C.c_int64),
                ("residual", C.c_void_p), ("ld_residual", C.c_int64)]


class GensorError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({status_string(status)})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2502_11407_amd.csrc.build` "
                          "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    P, S = C.POINTER(Problem), C.POINTER(Schedule)
    vp, i64, f32, i32 = C.c_void_p, C.c_int64, C.c_float, C.c_int32
    L.gensor_status_string.restype = C.c_char_p
    L.gensor_status_string.argtypes = [i32]
    L.gensor_num_instances.restype = i32
    L.gensor_instance_schedule.restype = i32
    L.gensor_instance_schedule.argtypes = [i32, P, S]
    L.gensor_hw_mi355x.restype = C.POINTER(Hw)
    L.gensor_construct.restype = i32
    L.gensor_construct.argtypes = [P, C.POINTER(Hw), C.POINTER(ConstructOpts), C.c_uint64, S]
    L.gensor_construct_trace.restype = i32
    L.gensor_construct_trace.argtypes = [P, C.POINTER(Hw), C.POINTER(ConstructOpts), C.c_uint64, i32,
                                         C.POINTER(i32), C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
    L.gensor_predict_us.restype = C.c_double
    L.gensor_predict_us.argtypes = [S, P, C.POINTER(Hw)]
    L.gensor_gemm.restype = i32
    L.gensor_gemm.argtypes = [S, P, f32, vp, i64, vp, i64, f32, vp, i64, vp, C.c_size_t, vp]
    L.gensor_gemm_static_scratch.restype = i32
    L.gensor_gemm_static_scratch.argtypes = [S, P, f32, vp, i64, vp, i64, f32, vp, i64, vp]
    L.gensor_bmm.restype = i32
    L.gensor_bmm.argtypes = [S, P, f32, vp, i64, i64, vp, i64, i64, f32, vp, i64, i64, vp, C.c_size_t, vp]
    L.gensor_conv2d.restype = i32
    L.gensor_conv2d.argtypes = [S, P, vp, vp, vp, vp, C.c_size_t, vp]
    L.gensor_workspace_bytes.restype = C.c_size_t
    L.gensor_workspace_bytes.argtypes = [S, P]
    L.gensor_gemv.restype = i32
    L.gensor_gemv.argtypes = [i32, i64, i64, f32, vp, i64, vp, f32, vp, vp]
    L.gensor_avgpool2d.restype = i32
    L.gensor_avgpool2d.argtypes = [i32, i32, i64, i64, i64, i64, i64, i64, vp, vp, vp]
    E, sz = C.POINTER(Epilogue), C.c_size_t
    L.gensor_gemm_fused.restype = i32
    L.gensor_gemm_fused.argtypes = [P, E, f32, vp, i64, vp, i64, vp, i64, vp, sz, vp]
    L.gensor_gemm_fused_workspace_bytes.restype = sz
    L.gensor_gemm_fused_workspace_bytes.argtypes = [P]
    L.gensor_grouped_gemm.restype = i32
    L.gensor_grouped_gemm.argtypes = [P, vp, E, f32, vp, i64, vp, i64, i64, vp, i64, vp]
    L.gensor_grouped_wgrad.restype = i32
    L.gensor_grouped_wgrad.argtypes = [P, vp, vp, i64, vp, i64, vp, i64, i64, vp]
    L.gensor_bias_grad.restype = i32
    L.gensor_bias_grad.argtypes = [i32, i32, i64, i64, i64, vp, i64, vp, vp, vp, sz, vp]
    L.gensor_bias_grad_workspace_bytes.restype = sz
    L.gensor_bias_grad_workspace_bytes.argtypes = [i32, i64, i64, i64]
    L.gensor_xent_forward.restype = i32
    L.gensor_xent_forward.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, sz, vp]
    L.gensor_xent_backward.restype = i32
    L.gensor_xent_backward.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    L.gensor_xent_workspace_bytes.restype = sz
    L.gensor_xent_workspace_bytes.argtypes = [i32, i64, i64, i64, i32]
    L.gensor_gated_gemm.restype = i32
    L.gensor_gated_gemm.argtypes = [P, i32, f32, vp, i64, vp, i64, i64, vp, vp, i64, vp, i64, i64, vp]
    L.gensor_gated_act_grad.restype = i32
    L.gensor_gated_act_grad.argtypes = [P, i32, f32, vp, i64, vp, i64, vp, i64, i64, vp, i64, i64, vp, i64, vp]
    L.gensor_logprobs.restype = i32
    L.gensor_logprobs.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, f32, vp, i64, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    L.gensor_logprobs_workspace_bytes.restype = sz
    L.gensor_logprobs_workspace_bytes.argtypes = [i32, i64, i64, i64, i32]
    L.gensor_distill_forward.restype = i32
    L.gensor_distill_forward.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, f32, i32, vp, vp, i32, vp, vp, vp, sz, vp]
    L.gensor_distill_backward.restype = i32
    L.gensor_distill_backward.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, f32, i32, vp, vp, i32, vp, vp, vp, i64, vp, i64, vp, sz, vp]
    L.gensor_distill_workspace_bytes.restype = sz
    L.gensor_distill_workspace_bytes.argtypes = [i32, i64, i64, i64, i32, i32]
    return L


lib = _load()


def status_string(st: int) -> str:
    return lib.gensor_status_string(int(st)).decode()


def _check(st: int, where: str):
    if st != GENSOR_OK:
        raise GensorError(st, where)


def gemm_problem(dtype: str, M: int, N: int, K: int, transA: int = 0, transB: int = 0, batch: int = 1,
                 out_dtype: str = "f32") -> Problem:
    p = Problem()
    p.op = OP_BMM if batch > 1 else OP_GEMM
    p.in_dtype, p.out_dtype = DTYPE[dtype], DTYPE[out_dtype]
    p.transA, p.transB = transA, transB
    p.batch, p.M, p.N, p.K = batch, M, N, K
    return p


def conv_problem(dtype: str, n, c, h, w, k, r, s, stride, pad, out_dtype: str = "f32") -> Problem:
    p = Problem()
    p.op = OP_CONV2D
    p.in_dtype, p.out_dtype = DTYPE[dtype], DTYPE[out_dtype]
    p.n, p.c, p.h, p.w, p.k, p.r, p.s, p.stride, p.pad = n, c, h, w, k, r, s, stride, pad
    return p


def num_instances() -> int:
    return int(lib.gensor_num_instances())


def instance_schedule(idx: int, p: Problem) -> Optional[Schedule]:
    """Schedule describing compiled instance `idx`, or None if it does not serve `p`."""
    s = Schedule()
    st = lib.gensor_instance_schedule(idx, C.byref(p), C.byref(s))
    if st == 2:
        return None
    _check(st, "gensor_instance_schedule")
    return s


def hw_mi355x() -> Hw:
    return lib.gensor_hw_mi355x().contents


def construct(p: Problem, seed: int = 0, opts: Optional[ConstructOpts] = None, hw: Optional[Hw] = None) -> Schedule:
    s = Schedule()
    st = lib.gensor_construct(C.byref(p), C.byref(hw) if hw is not None else None,
                              C.byref(opts) if opts is not None else None, seed, C.byref(s))
    _check(st, "gensor_construct")
    return s


def construct_trace(p: Problem, seed: int = 0, opts: Optional[ConstructOpts] = None, hw: Optional[Hw] = None,
                    capacity: int = 4096):
    """One walk: returns (actions, dims, states) as int32 arrays, states of shape [steps][12]."""
    steps = C.c_int32(0)
    actions = np.zeros(capacity, dtype=np.int32)
    dims = np.zeros(capacity, dtype=np.int32)
    states = np.zeros((capacity, 12), dtype=np.int32)
    ip = C.POINTER(C.c_int32)
    st = lib.gensor_construct_trace(C.byref(p), C.byref(hw) if hw is not None else None,
                                    C.byref(opts) if opts is not None else None, seed, capacity, C.byref(steps),
                                    actions.ctypes.data_as(ip), dims.ctypes.data_as(ip), states.ctypes.data_as(ip))
    _check(st, "gensor_construct_trace")
    n = steps.value
    return actions[:n], dims[:n], states[:n]


def predict_us(s: Schedule, p: Problem, hw: Optional[Hw] = None) -> float:
    return float(lib.gensor_predict_us(C.byref(s), C.byref(p), C.byref(hw) if hw is not None else None))


_current = None      # (current device, current raw stream of a device), once torch is imported


def _stream_ptr(stream=None):
    """The stream as a hipStream_t.  The current one is asked for by its handle: building torch's Stream object for it
    took 2.8 us of the 8.1 us that a small call spent on the host (5.2 us without; the launch itself is 4)."""
    global _current
    if stream is not None:
        return stream.cuda_stream
    if _current is None:
        import torch
        _current = (torch.cuda.current_device, torch._C._cuda_getCurrentRawStream)
    return _current[1](_current[0]())


def _sref(s):
    return C.byref(s) if s is not None else None


def _ws(workspace):
    """Address and bytes of a workspace, or of none.  The kernels write to it: memory of the host's, or a view with gaps, is refused."""
    if workspace is None:
        return None, 0
    if not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError(f"workspace: a contiguous device tensor is wanted, got strides {workspace.stride()} on {workspace.device}")
    return workspace.data_ptr(), workspace.nbytes


def gemm(p: Problem, A, B, Cout, alpha: float = 1.0, beta: float = 0.0, schedule: Optional[Schedule] = None,
         lda: Optional[int] = None, ldb: Optional[int] = None, ldc: Optional[int] = None, stream=None, workspace=None):
    """C = alpha op(A) op(B) + beta C on device tensors (2-D, row-major with unit inner stride).
    `workspace`: device tensor of at least workspace_bytes(p, schedule) bytes for a split-k schedule (or None)."""
    ws_ptr, ws_len = _ws(workspace)
    st = lib.gensor_gemm(_sref(schedule), C.byref(p), alpha, A.data_ptr(), lda if lda is not None else A.stride(0),
                         B.data_ptr(), ldb if ldb is not None else B.stride(0), beta,
                         Cout.data_ptr(), ldc if ldc is not None else Cout.stride(0), ws_ptr, ws_len, _stream_ptr(stream))
    _check(st, "gensor_gemm")


STATIC_SCRATCH_BYTES = 32 * 1024 * 1024 + 65536


def gemm_static_scratch(p: Problem, A, B, Cout, alpha: float = 1.0, beta: float = 0.0, schedule: Optional[Schedule] = None,
                        stream=None):
    """gemm() with the split-k workspace taken from the library's own device array (nothing is allocated)."""
    st = lib.gensor_gemm_static_scratch(_sref(schedule), C.byref(p), alpha, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0),
                                        beta, Cout.data_ptr(), Cout.stride(0), _stream_ptr(stream))
    _check(st, "gensor_gemm_static_scratch")


def bmm(p: Problem, A, B, Cout, alpha: float = 1.0, beta: float = 0.0, schedule: Optional[Schedule] = None,
        stream=None, workspace=None):
    """Batched: 3-D device tensors [batch][rows][cols]."""
    ws_ptr, ws_len = _ws(workspace)
    st = lib.gensor_bmm(_sref(schedule), C.byref(p), alpha, A.data_ptr(), A.stride(1), A.stride(0),
                        B.data_ptr(), B.stride(1), B.stride(0), beta,
                        Cout.data_ptr(), Cout.stride(1), Cout.stride(0), ws_ptr, ws_len, _stream_ptr(stream))
    _check(st, "gensor_bmm")


def workspace_bytes(p: Problem, schedule: Optional[Schedule] = None) -> int:
    return int(lib.gensor_workspace_bytes(_sref(schedule), C.byref(p)))


def conv2d(p: Problem, I, W, O, schedule: Optional[Schedule] = None, workspace=None, stream=None):
    """O = conv(I, W): contiguous NCHW input, KCRS filters, NKPQ output, all on the device.
    `workspace` is a device tensor of at least workspace_bytes(p, schedule) bytes (or None)."""
    ws_ptr, ws_len = _ws(workspace)
    st = lib.gensor_conv2d(_sref(schedule), C.byref(p), I.data_ptr(), W.data_ptr(), O.data_ptr(), ws_ptr, ws_len,
                           _stream_ptr(stream))
    _check(st, "gensor_conv2d")


# ---- device memory helpers (plumbing): stored bits <-> torch tensors
def to_device(arr: np.ndarray, dtype: str):
    import torch
    if dtype == "bf16":
        return torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(arr)).cuda()


def gemv(dtype: str, A, x, y, alpha: float = 1.0, beta: float = 0.0, lda: Optional[int] = None, stream=None):
    """y = alpha A x + beta y: A [M][N] row-major and x [N] of `dtype`, y [M] fp32, all on the device."""
    M, N = A.shape
    st = lib.gensor_gemv(DTYPE[dtype], M, N, alpha, A.data_ptr(), lda if lda is not None else A.stride(0), x.data_ptr(),
                         beta, y.data_ptr(), _stream_ptr(stream))
    _check(st, "gensor_gemv")


def avgpool2d(dtype: str, I, O, f: int, stride: int, out_dtype: str = "f32", stream=None):
    """O = f x f average pooling at `stride` of a contiguous NCHW device tensor."""
    n, c, h, w = I.shape
    st = lib.gensor_avgpool2d(DTYPE[dtype], DTYPE[out_dtype], n, c, h, w, f, stride, I.data_ptr(), O.data_ptr(),
                              _stream_ptr(stream))
    _check(st, "gensor_avgpool2d")


def gemm_workspace(p: Problem, schedule: Schedule):
    """Device buffer for gensor_gemm / gensor_bmm on `p` with a split-k `schedule`, or None if it needs none (plumbing)."""
    import torch
    n = workspace_bytes(p, schedule)
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def conv_workspace(p: Problem, schedule: Optional[Schedule] = None):
    """Device buffer large enough for gensor_conv2d on `p` with `schedule` (plumbing)."""
    import torch
    return torch.empty(max(16, workspace_bytes(p, schedule)), dtype=torch.uint8, device="cuda")


def empty_device(shape, dtype: str = "f32"):
    import torch
    td = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    return torch.empty(shape, dtype=td, device="cuda")


def to_host_f64(t) -> np.ndarray:
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


# ---- products that are consumed where they are produced.  Shapes and types are checked here against the problem, because the library
# sees addresses only.
_TORCH = None        # torch's type of a gensor_dtype, and the other way round, once torch is imported
_CODE = None


def _torch_types():
    global _TORCH, _CODE
    import torch
    _TORCH = (torch.float32, torch.float16, torch.bfloat16)
    _CODE = {t: i for i, t in enumerate(_TORCH)}


def _code(t, what: str) -> int:
    """The gensor_dtype of a tensor."""
    if _CODE is None:
        _torch_types()
    code = _CODE.get(t.dtype)
    if code is None:
        raise ValueError(f"{what}: f32, f16 and bf16 are served, got {t.dtype}")
    return code


def _matrix(t, rows: int, cols: int, dtype, what: str) -> int:
    """Checks a device matrix with unit inner stride against what the problem says it is; its leading dimension."""
    if t.shape == (rows, cols) and t.dtype is dtype and t.is_cuda:
        ld, inner = t.stride()
        if inner == 1 and ld >= cols:
            return ld
        if (cols == 1 or inner == 1) and (rows == 1 or ld >= cols):
            return ld if rows > 1 else cols
        raise ValueError(f"{what}: contiguous rows that do not overlap are wanted, got strides {t.stride()}")
    raise ValueError(f"{what}: a device matrix of {rows} x {cols} {dtype} is wanted, got {tuple(t.shape)} {t.dtype} on {t.device}")


def _vector(t, n: int, dtype: str, what: str) -> int:
    if t.shape != (n,) or not t.is_contiguous() or not t.is_cuda or str(t.dtype) != dtype:
        raise ValueError(f"{what}: a contiguous device vector of {n} {dtype} is wanted, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _stack(t, groups: int, rows: int, cols: int, dtype, what: str):
    """The same for a stack of matrices: (leading dimension, distance between matrices)."""
    if t.shape == (groups, rows, cols) and t.dtype is dtype and t.is_cuda:
        far, ld, inner = t.stride()
        if (cols == 1 or inner == 1) and (rows == 1 or ld >= cols):
            return ld if rows > 1 else cols, far if groups > 1 else 0
        raise ValueError(f"{what}: contiguous rows that do not overlap are wanted, got strides {t.stride()}")
    raise ValueError(f"{what}: a device stack of {groups} matrices of {rows} x {cols} {dtype} is wanted, got {tuple(t.shape)} {t.dtype} on {t.device}")


def _epilogue(rows: int, N: int, bias_shape, dtype, out, bias, act: str, preact, residual, grad: int):
    """The epilogue's structure, or None for the plain product."""
    code = ACT.get(act)
    if code is None:
        raise ValueError(f"act: one of {sorted(ACT)} is wanted, got {act!r}")
    if bias is None and preact is None and residual is None and code == 0 and not grad:
        return None
    e = Epilogue(code, grad)
    if bias is not None:
        if bias.shape != bias_shape or not bias.is_contiguous() or bias.dtype is not dtype or not bias.is_cuda:
            raise ValueError(f"bias: a contiguous device tensor of {bias_shape} {dtype} is wanted, got {tuple(bias.shape)} {bias.dtype} on {bias.device}")
        e.bias = bias.data_ptr()
    if preact is not None:
        e.ld_preact = _matrix(preact, rows, N, out, "preact")
        e.preact = preact.data_ptr()
    if residual is not None:
        e.ld_residual = _matrix(residual, rows, N, out, "residual")
        e.residual = residual.data_ptr()
    return C.byref(e)


def gemm_fused_workspace_bytes(p: Problem) -> int:
    return int(lib.gensor_gemm_fused_workspace_bytes(C.byref(p)))


def _gemm_fused(p, A, B, Cout, bias, act, preact, residual, grad, alpha, workspace, stream):
    if _TORCH is None:
        _torch_types()
    M, N, K, dtype, out = p.M, p.N, p.K, _TORCH[p.in_dtype], _TORCH[p.out_dtype]
    e = _epilogue(M, N, (N,), dtype, out, bias, act, preact, residual, grad)
    lda = _matrix(A, K, M, dtype, "A") if p.transA else _matrix(A, M, K, dtype, "A")
    ldb = _matrix(B, N, K, dtype, "B") if p.transB else _matrix(B, K, N, dtype, "B")
    ldc = _matrix(Cout, M, N, out, "C")
    ws_ptr, ws_len = _ws(workspace)
    st = lib.gensor_gemm_fused(C.byref(p), e, alpha, A.data_ptr(), lda, B.data_ptr(), ldb, Cout.data_ptr(), ldc, ws_ptr, ws_len, _stream_ptr(stream))
    if st:
        _check(st, "gensor_gemm_fused")


def gemm_fused(p: Problem, A, B, Cout, bias=None, act: str = "none", preact=None, residual=None, alpha: float = 1.0, stream=None, workspace=None):
    """C = act(Z) + residual with Z = alpha op(A) op(B) + bias; `preact`, if given, receives Z.  act: none, relu, gelu (tanh form), silu.
    `workspace`: device tensor of gemm_fused_workspace_bytes(p) bytes, or less, or None."""
    _gemm_fused(p, A, B, Cout, bias, act, preact, residual, 0, alpha, workspace, stream)


def gemm_act_grad(p: Problem, A, B, preact, Cout, act: str, alpha: float = 1.0, stream=None, workspace=None):
    """C = (alpha op(A) op(B)) * act'(preact): the gradient that reaches an activation's input, from the product behind it."""
    _gemm_fused(p, A, B, Cout, None, act, preact, None, 1, alpha, workspace, stream)


def grouped_problem(dtype: str, groups: int, rows: int, N: int, K: int, transB: int = 0, out_dtype: str = "f32") -> Problem:
    """Products grouped by expert: `rows` rows of all groups together, each group with its own K x N (transB: N x K) matrix."""
    p = gemm_problem(dtype, rows, N, K, 0, transB, groups, out_dtype)
    p.op = OP_BMM
    return p


def _grouped_gemm(p, offsets, A, B, Cout, bias, act, preact, residual, grad, alpha, stream):
    if _TORCH is None:
        _torch_types()
    G, M, N, K, dtype, out = p.batch, p.M, p.N, p.K, _TORCH[p.in_dtype], _TORCH[p.out_dtype]
    off = _vector(offsets, G + 1, "torch.int32", "offsets")
    lda, ldc = _matrix(A, M, K, dtype, "A"), _matrix(Cout, M, N, out, "C")
    ldb, stride = _stack(B, G, N, K, dtype, "B") if p.transB else _stack(B, G, K, N, dtype, "B")
    e = _epilogue(M, N, (G, N), dtype, out, bias, act, preact, residual, grad)
    if M == 0:                                     # (nothing to do, and an empty tensor has no address)
        return
    st = lib.gensor_grouped_gemm(C.byref(p), off, e, alpha, A.data_ptr(), lda, B.data_ptr(), ldb, stride, Cout.data_ptr(), ldc, _stream_ptr(stream))
    if st:
        _check(st, "gensor_grouped_gemm")


def grouped_gemm(p: Problem, offsets, A, B, Cout, bias=None, act: str = "none", preact=None, residual=None, alpha: float = 1.0, stream=None):
    """Rows offsets[g] .. offsets[g+1] of C = act(alpha A B[g] + bias[g]) + residual.  offsets: groups + 1 int32 on the device."""
    _grouped_gemm(p, offsets, A, B, Cout, bias, act, preact, residual, 0, alpha, stream)


def grouped_act_grad(p: Problem, offsets, A, B, preact, Cout, act: str, alpha: float = 1.0, stream=None):
    """Rows offsets[g] .. offsets[g+1] of C = (alpha A B[g]) * act'(preact)."""
    _grouped_gemm(p, offsets, A, B, Cout, None, act, preact, None, 1, alpha, stream)


def grouped_wgrad(p: Problem, offsets, A, dY, dW, stream=None):
    """dW[g] = A_g^T dY_g over the rows of g, laid out like the B of `p`: the gradient of grouped_gemm's B for the same problem."""
    if _TORCH is None:
        _torch_types()
    G, M, N, K, dtype, out = p.batch, p.M, p.N, p.K, _TORCH[p.in_dtype], _TORCH[p.out_dtype]
    off = _vector(offsets, G + 1, "torch.int32", "offsets")
    lda, lddy = _matrix(A, M, K, dtype, "A"), _matrix(dY, M, N, dtype, "dY")
    lddw, stride = _stack(dW, G, N, K, out, "dW") if p.transB else _stack(dW, G, K, N, out, "dW")
    st = lib.gensor_grouped_wgrad(C.byref(p), off, A.data_ptr(), lda, dY.data_ptr(), lddy, dW.data_ptr(), lddw, stride, _stream_ptr(stream))
    if st:
        _check(st, "gensor_grouped_wgrad")


def bias_grad_workspace_bytes(groups: int, rows: int, N: int, dtype: str = "bf16") -> int:
    return int(lib.gensor_bias_grad_workspace_bytes(DTYPE[dtype], groups, rows, N))


def bias_grad(dY, db, offsets=None, stream=None, workspace=None):
    """db = column sums of dY [rows][N]; with offsets (groups + 1 int32 on the device) db[g] = column sums of the rows of g."""
    rows, N = dY.shape
    dt, out = _code(dY, "dY"), _code(db, "db")
    groups = 1 if offsets is None else offsets.shape[0] - 1
    off = None if offsets is None else _vector(offsets, groups + 1, "torch.int32", "offsets")
    if db.shape != ((N,) if offsets is None else (groups, N)) or not db.is_contiguous() or not db.is_cuda:
        raise ValueError(f"db: a contiguous device tensor of {(N,) if offsets is None else (groups, N)} is wanted, got {tuple(db.shape)} on {db.device}")
    ld = _matrix(dY, rows, N, dY.dtype, "dY")
    ws_ptr, ws_len = _ws(workspace)
    st = lib.gensor_bias_grad(dt, out, groups, rows, N, dY.data_ptr(), ld, off, db.data_ptr(), ws_ptr, ws_len, _stream_ptr(stream))
    if st:
        _check(st, "gensor_bias_grad")


def xent_workspace_bytes(dtype: str, T: int, V: int, D: int, backward: bool = False) -> int:
    return int(lib.gensor_xent_workspace_bytes(DTYPE[dtype], T, V, D, 1 if backward else 0))


def xent_forward(X, W, targets, loss, lse, ignore_index: int = -100, stream=None, workspace=None):
    """loss[t] = lse[t] - z[t][targets[t]] and lse[t] = log sum exp z[t] of the logits z = X W^T, which are never stored: X [T][D], W [V][D] of
    one type, targets [T] int64, loss and lse [T] fp32 (either may be None).  `workspace`: xent_workspace_bytes(...) bytes."""
    (T, D), (V, _) = X.shape, W.shape
    dt, dtype = _code(X, "X"), X.dtype
    ldx, ldw = _matrix(X, T, D, dtype, "X"), _matrix(W, V, D, dtype, "W")
    ws_ptr, ws_len = _ws(workspace)
    _check(lib.gensor_xent_forward(dt, T, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw,
                                   None if targets is None else _vector(targets, T, "torch.int64", "targets"), ignore_index,
                                   None if loss is None else _vector(loss, T, "torch.float32", "loss"),
                                   None if lse is None else _vector(lse, T, "torch.float32", "lse"), ws_ptr, ws_len, _stream_ptr(stream)), "gensor_xent_forward")


def xent_backward(X, W, targets, lse, dloss, dX, dW, ignore_index: int = -100, stream=None, workspace=None):
    """dX = G W and dW = G^T X with G[t][v] = dloss[t] (exp(z[t][v] - lse[t]) - (v == targets[t])); dX or dW may be None.
    `workspace`: xent_workspace_bytes(..., backward=True) bytes, or less for smaller pieces of the vocabulary."""
    (T, D), (V, _) = X.shape, W.shape
    dt, dtype = _code(X, "X"), X.dtype
    ldx, ldw = _matrix(X, T, D, dtype, "X"), _matrix(W, V, D, dtype, "W")
    ws_ptr, ws_len = _ws(workspace)
    _check(lib.gensor_xent_backward(dt, T, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw, _vector(targets, T, "torch.int64", "targets"), ignore_index,
                                    _vector(lse, T, "torch.float32", "lse"), _vector(dloss, T, "torch.float32", "dloss"),
                                    None if dX is None else dX.data_ptr(), 0 if dX is None else _matrix(dX, T, D, dtype, "dX"),
                                    None if dW is None else dW.data_ptr(), 0 if dW is None else _matrix(dW, V, D, dtype, "dW"),
                                    ws_ptr, ws_len, _stream_ptr(stream)), "gensor_xent_backward")


# ---- a language model's gated layers, the scores of its vocabulary, and learning from a teacher.  The launches go to the current device: tensors
# of another one are refused.
def _on_current_device(stream, **tensors):
    """The stream as a hipStream_t, once all tensors are found to be on its device."""
    if _current is None:
        _stream_ptr()
    here = _current[0]()
    if stream is not None and stream.device_index != here:
        raise ValueError(f"stream: one of the current device, {here}, is wanted, got device {stream.device_index}")
    for name, t in tensors.items():
        if t is not None and t.get_device() != here:
            raise ValueError(f"{name}: a tensor on the current device, {here}, is wanted, got {t.device}")
    return stream.cuda_stream if stream is not None else _current[1](here)


def _act(act: str) -> int:
    code = ACT.get(act)
    if code is None:
        raise ValueError(f"act: one of {sorted(ACT)} is wanted, got {act!r}")
    return code


def _two(t, rows: int, cols: int, dtype, what: str):
    """Two matrices as one tensor [2][rows][cols], wherever the second lies behind the first: (leading dimension, distance)."""
    if t.shape == (2, rows, cols) and t.dtype is dtype and t.is_cuda:
        far, ld, inner = t.stride()
        if (cols == 1 or inner == 1) and (rows == 1 or ld >= cols):
            return ld if rows > 1 else cols, far
        raise ValueError(f"{what}: contiguous rows that do not overlap are wanted, got strides {t.stride()}")
    raise ValueError(f"{what}: two device matrices of {rows} x {cols} {dtype} are wanted, got {tuple(t.shape)} {t.dtype} on {t.device}")


def gated_gemm(p: Problem, A, B, Cout, act: str = "silu", bias=None, preact=None, alpha: float = 1.0, stream=None):
    """C = act(G) * U of the products G = alpha A op(B[0]) + bias[0] and U = alpha A op(B[1]) + bias[1]: p is either product's, B [2][K][N] ([2][N][K] if
    p.transB) a tensor of both matrices, which may lie side by side in one: W.view(K, 2, N).transpose(0, 1).  bias [2][N]; preact [2][M][N] receives G
    and U in C's type (as the gradient needs them)."""
    if _TORCH is None:
        _torch_types()
    M, N, K, dtype, out = p.M, p.N, p.K, _TORCH[p.in_dtype], _TORCH[p.out_dtype]
    code = _act(act)
    lda, ldc = _matrix(A, M, K, dtype, "A"), _matrix(Cout, M, N, out, "C")
    ldb, far = _two(B, N, K, dtype, "B") if p.transB else _two(B, K, N, dtype, "B")
    ldz, far_z = (0, 0) if preact is None else _two(preact, M, N, out, "preact")
    if bias is not None and (bias.shape != (2, N) or not bias.is_contiguous() or bias.dtype is not dtype or not bias.is_cuda):
        raise ValueError(f"bias: a contiguous device tensor of {(2, N)} {dtype} is wanted, got {tuple(bias.shape)} {bias.dtype} on {bias.device}")
    st_ptr = _on_current_device(stream, A=A, B=B, C=Cout, bias=bias, preact=preact)
    st = lib.gensor_gated_gemm(C.byref(p), code, alpha, A.data_ptr(), lda, B.data_ptr(), ldb, far, None if bias is None else bias.data_ptr(), Cout.data_ptr(), ldc,
                               None if preact is None else preact.data_ptr(), ldz, far_z, st_ptr)
    if st:
        _check(st, "gensor_gated_gemm")


def gated_act_grad(p: Problem, A, B, preact, dpreact, act: str = "silu", H=None, alpha: float = 1.0, stream=None):
    """At the end of the product D = alpha A op(B), the gradient of a gated layer's result: dpreact[0] = D * U * act'(G) and dpreact[1] = D * act(G) of
    preact = (G, U), all [2][M][N]; dpreact may be preact.  H [M][N] receives act(G) * U again."""
    if _TORCH is None:
        _torch_types()
    M, N, K, dtype, out = p.M, p.N, p.K, _TORCH[p.in_dtype], _TORCH[p.out_dtype]
    code = _act(act)
    lda = _matrix(A, M, K, dtype, "A")
    ldb = _matrix(B, N, K, dtype, "B") if p.transB else _matrix(B, K, N, dtype, "B")
    ldz, far_z = _two(preact, M, N, out, "preact")
    ldd, far_d = _two(dpreact, M, N, out, "dpreact")
    ldh = 0 if H is None else _matrix(H, M, N, out, "H")
    st_ptr = _on_current_device(stream, A=A, B=B, preact=preact, dpreact=dpreact, H=H)
    st = lib.gensor_gated_act_grad(C.byref(p), code, alpha, A.data_ptr(), lda, B.data_ptr(), ldb, preact.data_ptr(), ldz, far_z, dpreact.data_ptr(), ldd, far_d,
                                   None if H is None else H.data_ptr(), ldh, st_ptr)
    if st:
        _check(st, "gensor_gated_act_grad")


def _table(t, shape, dtype: str, what: str) -> int:
    """The address of a contiguous device tensor."""
    if t.shape != shape or not t.is_contiguous() or not t.is_cuda or str(t.dtype) != dtype:
        raise ValueError(f"{what}: a contiguous device tensor of {shape} {dtype} is wanted, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def logprobs_workspace_bytes(dtype: str, T: int, V: int, D: int, top: int = 0) -> int:
    return int(lib.gensor_logprobs_workspace_bytes(DTYPE[dtype], T, V, D, top))


def logprobs(X, W, targets=None, logprob=None, lse=None, entropy=None, top_index=None, top_logprob=None, scale: float = 1.0, ignore_index: int = -100,
             stream=None, workspace=None):
    """Scores of the logits z = scale X W^T, which are not kept: X [T][D], W [V][D] of one type.  Into logprob [T] the log probabilities of `targets` [T]
    int64, into lse [T] log sum exp z, into entropy [T] the distributions' entropies, into top_index [T][k] int64 and top_logprob [T][k] the k most likely entries
    and their log probabilities, falling, of equal ones the lowest first; all fp32, each may be None.  `workspace`: logprobs_workspace_bytes(...) bytes, or
    less for smaller pieces of the vocabulary."""
    (T, D), (V, _) = X.shape, W.shape
    dt, dtype = _code(X, "X"), X.dtype
    ldx, ldw = _matrix(X, T, D, dtype, "X"), _matrix(W, V, D, dtype, "W")
    if (top_index is None) != (top_logprob is None):
        raise ValueError("top_index and top_logprob: both or neither are wanted")
    top = 0 if top_index is None else top_index.shape[-1]
    if top_index is not None and top == 0:
        raise ValueError("top_index: room for one alternative at least is wanted")
    ws_ptr, ws_len = _ws(workspace)
    st_ptr = _on_current_device(stream, X=X, W=W, targets=targets, logprob=logprob, lse=lse, entropy=entropy, top_index=top_index, top_logprob=top_logprob, workspace=workspace)
    _check(lib.gensor_logprobs(dt, T, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw, scale, None if targets is None else _vector(targets, T, "torch.int64", "targets"),
                               ignore_index, None if logprob is None else _vector(logprob, T, "torch.float32", "logprob"),
                               None if lse is None else _vector(lse, T, "torch.float32", "lse"), None if entropy is None else _vector(entropy, T, "torch.float32", "entropy"),
                               top, None if top == 0 else _table(top_index, (T, top), "torch.int64", "top_index"),
                               None if top == 0 else _table(top_logprob, (T, top), "torch.float32", "top_logprob"), ws_ptr, ws_len, st_ptr), "gensor_logprobs")


def distill_workspace_bytes(dtype: str, T: int, V: int, D: int, k: int, backward: bool = False) -> int:
    return int(lib.gensor_distill_workspace_bytes(DTYPE[dtype], T, V, D, k, 1 if backward else 0))


def _distill(X, W, index, teacher, stream, **tensors):
    (T, D), (V, _), k = X.shape, W.shape, index.shape[-1]
    dt, dtype = _code(X, "X"), X.dtype
    ldx, ldw = _matrix(X, T, D, dtype, "X"), _matrix(W, V, D, dtype, "W")
    at, q = _table(index, (T, k), "torch.int64", "index"), _table(teacher, (T, k), "torch.float32", "teacher")
    return dt, T, V, D, ldx, ldw, k, at, q, _on_current_device(stream, X=X, W=W, index=index, teacher=teacher, **tensors)


def distill_forward(X, W, index, teacher, loss, lse, scale: float = 1.0, normalize: bool = True, stream=None, workspace=None):
    """loss[t] = sum_j p_j (log p_j - z[index_j] + lse) of the logits z = scale X W^T, which are not kept, against a teacher's entries: index [T][k] int64 (-1: none)
    and their log probabilities teacher [T][k] fp32; p = softmax of scale * teacher over the token's entries, or exp(teacher) as it is.  loss and lse [T]
    fp32, either may be None.  `workspace`: distill_workspace_bytes(...) bytes."""
    dt, T, V, D, ldx, ldw, k, at, q, st_ptr = _distill(X, W, index, teacher, stream, loss=loss, lse=lse, workspace=workspace)
    ws_ptr, ws_len = _ws(workspace)
    _check(lib.gensor_distill_forward(dt, T, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw, scale, k, at, q, 1 if normalize else 0,
                                      None if loss is None else _vector(loss, T, "torch.float32", "loss"),
                                      None if lse is None else _vector(lse, T, "torch.float32", "lse"), ws_ptr, ws_len, st_ptr), "gensor_distill_forward")


def distill_backward(X, W, index, teacher, lse, dloss, dX, dW, scale: float = 1.0, normalize: bool = True, stream=None, workspace=None):
    """dX = G W and dW = G^T X with G[t][v] = dloss[t] scale (P exp(z[t][v] - lse[t]) - sum of p_j over index_j == v), P = sum_j p_j; dX or dW may be None.
    `workspace`: distill_workspace_bytes(..., backward=True) bytes, or less for smaller pieces of the vocabulary."""
    dt, T, V, D, ldx, ldw, k, at, q, st_ptr = _distill(X, W, index, teacher, stream, lse=lse, dloss=dloss, dX=dX, dW=dW, workspace=workspace)
    ws_ptr, ws_len = _ws(workspace)
    _check(lib.gensor_distill_backward(dt, T, V, D, X.data_ptr(), ldx, W.data_ptr(), ldw, scale, k, at, q, 1 if normalize else 0,
                                       _vector(lse, T, "torch.float32", "lse"), _vector(dloss, T, "torch.float32", "dloss"),
                                       None if dX is None else dX.data_ptr(), 0 if dX is None else _matrix(dX, T, D, X.dtype, "dX"),
                                       None if dW is None else dW.data_ptr(), 0 if dW is None else _matrix(dW, V, D, X.dtype, "dW"),
                                       ws_ptr, ws_len, st_ptr), "gensor_distill_backward")
