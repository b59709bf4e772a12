"""ctypes binding of libccl.so: the calls of include/ccl.h under the same names.

Argument marshalling only: every step runs in the HIP library. Device
buffers may be given as torch tensors (their data_ptr() is passed) or as
integer device addresses (what a call takes from a tensor beyond its address, a
type or a stride, is checked against what the call reads); `stream` may be a torch.cuda.Stream, an integer
hipStream_t, or None (torch's current stream when torch has initialised the
GPU, else the null stream). Errors raise CCLError with the library's status
and message. If libccl.so is not built, loading raises; there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import sys
from dataclasses import dataclass

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libccl.so")

CCL_A, CCL_B, CCL_C = 0, 1, 2
CCL_PLACE_RR, CCL_PLACE_COARSE, CCL_PLACE_CCL = 0, 1, 2
CCL_SCRATCH_BYTES = 64 << 20        # static split-K workspace of ccl_gemm_splitk_noalloc, per GPU
MAX_CHIPLETS = 64

STATUS_NAMES = {0: "CCL_OK", 1: "CCL_ERR_INVALID_ARG", 2: "CCL_ERR_UNALIGNED_PARTITION",
                3: "CCL_ERR_UNSUPPORTED", 4: "CCL_ERR_MISALIGNED_POINTER", 5: "CCL_ERR_HIP"}

# every symbol include/ccl.h declares
EXPORTED = ("ccl_plan", "ccl_plan_typed", "ccl_plan_destroy", "ccl_plan_grid", "ccl_plan_layout",
            "ccl_pack", "ccl_unpack", "ccl_gemm", "ccl_gemm_scaled", "ccl_gemm_splitk_workspace",
            "ccl_gemm_splitk", "ccl_gemm_splitk_noalloc", "ccl_gemm_rowmajor",
            "ccl_plan_matrix_layout", "ccl_gemm_fused_workspace", "ccl_gemm_fused", "ccl_gemm_fused_grad_workspace",
            "ccl_gemm_fused_grad", "ccl_moe_workspace", "ccl_moe_decode",
            "ccl_orthogonalize_workspace", "ccl_orthogonalize",
            "ccl_grouped_gemm_workspace", "ccl_grouped_gemm", "ccl_grouped_gemm_grad", "ccl_grouped_gemm_wgrad",
            "ccl_cross_entropy_workspace", "ccl_cross_entropy", "ccl_cross_entropy_grad",
            "ccl_adamw_step", "ccl_adamw_moments",
            "ccl_remote_bytes", "ccl_remote_bytes_l2", "ccl_status_string", "ccl_last_error",
            "ccl_debug_tile_of_wg", "ccl_debug_gemm_config", "ccl_debug_dispatch",
            "ccl_debug_gemm_timeline", "ccl_debug_launch", "ccl_debug_launch_tile_of_wg",
            "ccl_debug_launch_dispatch", "ccl_debug_launch_timeline")


class CCLError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        self.status_name = STATUS_NAMES.get(status, str(status))
        super().__init__(f"{self.status_name}: {message}")


class _Layout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "cols", "grid_r", "grid_c", "block_rows",
                                               "block_cols", "strip_bytes", "strip_stride_bytes",
                                               "total_bytes", "elem_bytes")]


class _Traffic(ctypes.Structure):
    _fields_ = [("accessed", ctypes.c_uint64 * 3), ("remote", ctypes.c_uint64 * 3),
                ("floor_bytes", ctypes.c_uint64), ("footprint", ctypes.c_uint64 * 3),
                ("remote_per_chiplet", ctypes.c_uint64 * MAX_CHIPLETS), ("chiplets", ctypes.c_int32)]


class _L2Config(ctypes.Structure):
    _fields_ = [("l2_bytes", ctypes.c_int64), ("ways", ctypes.c_int32), ("line_bytes", ctypes.c_int32),
                ("slots", ctypes.c_int32), ("k_step", ctypes.c_int32), ("traversal", ctypes.c_int32),
                ("threads", ctypes.c_int32), ("group_rows", ctypes.c_int32)]


class _L2Traffic(ctypes.Structure):
    _fields_ = [("accesses", ctypes.c_uint64 * 2), ("misses", ctypes.c_uint64 * 2),
                ("remote", ctypes.c_uint64 * 3),
                ("remote_per_chiplet", ctypes.c_uint64 * MAX_CHIPLETS), ("chiplets", ctypes.c_int32)]


class _Launch(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_char * 32), ("workgroups", ctypes.c_int64)] + \
               [(n, ctypes.c_int) for n in ("tile_rows", "tile_cols", "waves", "k_ranges", "ragged", "far", "stream_b", "c_nt")]


class _Epilogue(ctypes.Structure):
    _fields_ = [("activation", ctypes.c_int), ("gated", ctypes.c_int32), ("layout", ctypes.c_int),
                ("bias_type", ctypes.c_int), ("alpha", ctypes.c_float), ("beta", ctypes.c_float),
                ("rows", ctypes.c_int64), ("bias", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("preact", ctypes.c_void_p)]


class _EpilogueGrad(ctypes.Structure):
    _fields_ = [("activation", ctypes.c_int), ("gated", ctypes.c_int32), ("layout", ctypes.c_int),
                ("alpha", ctypes.c_float), ("rows", ctypes.c_int64), ("preact", ctypes.c_void_p),
                ("dbias", ctypes.c_void_p)]


class _Moe(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int64), ("ffn", ctypes.c_int64), ("experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("activation", ctypes.c_int), ("normalize", ctypes.c_int32),
                ("weight_type", ctypes.c_int)] + \
               [(n, ctypes.c_int64) for n in ("gate_up_ld", "gate_up_stride", "down_ld", "down_stride")]


class _Grouped(ctypes.Structure):
    _fields_ = [("in_features", ctypes.c_int64), ("out_features", ctypes.c_int64), ("experts", ctypes.c_int32),
                ("activation", ctypes.c_int), ("gated", ctypes.c_int32), ("w_ld", ctypes.c_int64),
                ("w_stride", ctypes.c_int64)]


class _Vocab(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("hidden", "vocab", "w_ld", "block")] + [("scale", ctypes.c_float)]


class _Adamw(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps")] + [("step", ctypes.c_int64)] + \
               [(n, ctypes.c_void_p) for n in ("step_ptr", "lr_ptr", "grad_scale")]


class _AdamwTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale",
                                               "exp_avg_sq_scale", "copy")] + \
               [("n", ctypes.c_int64), ("param_type", ctypes.c_int), ("grad_type", ctypes.c_int),
                ("moment_bits", ctypes.c_int32), ("weight_decay", ctypes.c_float)]


_lib = None


def library() -> ctypes.CDLL:
    """Load libccl.so once (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run __graft_entry__.build() "
                          "or python -m paper_2606_11718_amd.build")
    # libccl.so needs libamdhip64.so.7. torch ships its own copy of the HIP
    # runtime under that soname; loading torch first makes the dynamic loader
    # hand libccl.so that same runtime, so one HIP runtime serves both (two
    # runtimes in one process do not share devices, memory or streams).
    import torch  # noqa: F401
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    sig = {
        "ccl_plan": [i64, i64, i64, i32, i32, i64, ctypes.POINTER(vp)],
        "ccl_plan_typed": [i64, i64, i64, i32, i32, i64, i32, i32, ctypes.POINTER(vp)],
        "ccl_plan_destroy": [vp],
        "ccl_plan_grid": [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)],
        "ccl_plan_layout": [vp, i32, ctypes.POINTER(_Layout)],
        "ccl_pack": [vp, i32, vp, i64, i32, vp, vp],
        "ccl_unpack": [vp, i32, vp, vp, i64, vp],
        "ccl_gemm": [vp, vp, vp, vp, vp],
        "ccl_gemm_scaled": [vp, ctypes.c_float, vp, vp, ctypes.c_float, vp, vp],
        "ccl_gemm_splitk_workspace": [vp, ctypes.POINTER(i32), ctypes.POINTER(i64)],
        "ccl_gemm_splitk": [vp, ctypes.c_float, vp, vp, ctypes.c_float, vp, i32, vp, i64, vp],
        "ccl_gemm_splitk_noalloc": [vp, ctypes.c_float, vp, vp, ctypes.c_float, vp, i32, vp],
        "ccl_gemm_rowmajor": [vp, vp, vp, vp, i32, vp],
        "ccl_plan_matrix_layout": [vp, i64, ctypes.POINTER(_Layout)],
        "ccl_gemm_fused_workspace": [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(i64)],
        "ccl_gemm_fused": [vp, ctypes.POINTER(_Epilogue), vp, vp, vp, i32, vp, i64, vp],
        "ccl_gemm_fused_grad_workspace": [vp, i32, i32, i32, ctypes.POINTER(i64)],
        "ccl_gemm_fused_grad": [vp, ctypes.POINTER(_EpilogueGrad), vp, vp, vp, vp, i64, vp],
        "ccl_moe_workspace": [ctypes.POINTER(_Moe), i64, ctypes.POINTER(i64)],
        "ccl_moe_decode": [ctypes.POINTER(_Moe), i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp, i64, vp],
        "ccl_orthogonalize_workspace": [i64, i64, i64, ctypes.POINTER(i64)],
        "ccl_orthogonalize": [i64, i64, i64, vp, i32, i64, i64, i32, ctypes.POINTER(ctypes.c_float), ctypes.c_float,
                              vp, i64, i64, vp, i64, vp],
        "ccl_grouped_gemm_workspace": [ctypes.POINTER(_Grouped), i64, i32, ctypes.POINTER(i64)],
        "ccl_grouped_gemm": [ctypes.POINTER(_Grouped), i64, vp, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp],
        "ccl_grouped_gemm_grad": [ctypes.POINTER(_Grouped), i64, vp, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp],
        "ccl_grouped_gemm_wgrad": [ctypes.POINTER(_Grouped), i64, vp, vp, i64, vp, i64, vp, i32, i32, vp, i64, vp],
        "ccl_cross_entropy_workspace": [ctypes.POINTER(_Vocab), i64, i32, ctypes.POINTER(i64)],
        "ccl_cross_entropy": [ctypes.POINTER(_Vocab), i64, vp, i64, vp, vp, vp, vp, vp, i64, vp],
        "ccl_cross_entropy_grad": [ctypes.POINTER(_Vocab), i64, vp, i64, vp, vp, vp, ctypes.c_float, vp, vp, vp, i64, vp, i64,
                                   i32, i32, vp, i64, vp],
        "ccl_adamw_step": [ctypes.POINTER(_Adamw), ctypes.POINTER(_AdamwTensor), i64, vp],
        "ccl_adamw_moments": [i64, vp, vp, vp, vp, vp, vp, i32, vp],
        "ccl_remote_bytes": [vp, i32, i32, ctypes.POINTER(_Traffic)],
        "ccl_remote_bytes_l2": [vp, i32, i32, ctypes.POINTER(_L2Config), ctypes.POINTER(_L2Traffic)],
        "ccl_debug_tile_of_wg": [vp, i64, ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(i64)],
        "ccl_debug_gemm_config": [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i64)],
        "ccl_debug_dispatch": [vp, vp, vp],
        "ccl_debug_gemm_timeline": [vp, vp, vp, vp, vp, i64, vp],
        "ccl_debug_launch": [vp, i32, i32, i32, ctypes.POINTER(_Launch)],
        "ccl_debug_launch_tile_of_wg": [vp, i64, ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(i64)],
        "ccl_debug_launch_dispatch": [vp, vp, vp],
        "ccl_debug_launch_timeline": [vp, vp, vp, vp, vp, i64, vp],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    lib.ccl_status_string.argtypes = [ctypes.c_int]
    lib.ccl_status_string.restype = ctypes.c_char_p
    lib.ccl_last_error.argtypes = []
    lib.ccl_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int) -> None:
    if status != 0:
        raise CCLError(status, library().ccl_last_error().decode())


def _ptr(x) -> int:
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    return int(x.data_ptr())


def _refuse(name: str, why: str) -> None:
    raise CCLError(1, f"{name}: {why}")


def _whole(name: str, t, n: int, dtype) -> int:
    """Address of n elements side by side."""
    if t is None or isinstance(t, int):
        return t or 0
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        _refuse(name, f"not {n} elements of {dtype} without gaps")
    return t.data_ptr()


def _stream(s) -> int:
    if s is None:
        torch = sys.modules.get("torch")
        if torch is not None and torch.cuda.is_initialized():
            # The current device's current stream as its raw handle, without
            # building a torch.cuda.Stream: 0.5 against 3.4 us, of 8 us per call.
            raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
            if raw is not None:
                return raw(torch._C._cuda_getDevice())
            return int(torch.cuda.current_stream().cuda_stream)
        return 0
    if isinstance(s, int):
        return s
    return int(s.cuda_stream)


class Plan:
    """Owns a ccl_plan_t; destroyed with the object."""

    def __init__(self, handle: int, args: tuple):
        self.handle = handle
        self.args = args

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.ccl_plan_destroy(self.handle)
            self.handle = None

    @property
    def _as_parameter_(self):
        return ctypes.c_void_p(self.handle)


@dataclass
class Layout:
    rows: int
    cols: int
    grid_r: int
    grid_c: int
    block_rows: int
    block_cols: int
    strip_bytes: int
    strip_stride_bytes: int
    total_bytes: int
    elem_bytes: int


CCL_DT_BF16, CCL_DT_FP8_E4M3, CCL_DT_FP32 = 0, 1, 2


def ccl_plan(M: int, N: int, K: int, chiplets: int, grid_rows: int, page_bytes: int) -> Plan:
    h = ctypes.c_void_p()
    _check(library().ccl_plan(M, N, K, chiplets, grid_rows, page_bytes, ctypes.byref(h)))
    return Plan(h.value, (M, N, K, chiplets, grid_rows, page_bytes))


def ccl_plan_typed(M: int, N: int, K: int, chiplets: int, grid_rows: int, page_bytes: int,
                   ab_type: int, c_type: int) -> Plan:
    h = ctypes.c_void_p()
    _check(library().ccl_plan_typed(M, N, K, chiplets, grid_rows, page_bytes, ab_type, c_type,
                                    ctypes.byref(h)))
    return Plan(h.value, (M, N, K, chiplets, grid_rows, page_bytes, ab_type, c_type))


def ccl_plan_grid(plan: Plan) -> tuple[int, int]:
    r, c = ctypes.c_int(), ctypes.c_int()
    _check(library().ccl_plan_grid(plan, ctypes.byref(r), ctypes.byref(c)))
    return r.value, c.value


def ccl_plan_layout(plan: Plan, op: int) -> Layout:
    out = _Layout()
    _check(library().ccl_plan_layout(plan, op, ctypes.byref(out)))
    return Layout(*(getattr(out, f) for f, _ in _Layout._fields_))


def ccl_pack(plan: Plan, op: int, src, ld: int, src_trans: int, dst_ccl, stream=None) -> None:
    _check(library().ccl_pack(plan, op, _ptr(src), ld, src_trans, _ptr(dst_ccl), _stream(stream)))


def ccl_unpack(plan: Plan, op: int, src_ccl, dst, ld: int, stream=None) -> None:
    _check(library().ccl_unpack(plan, op, _ptr(src_ccl), _ptr(dst), ld, _stream(stream)))


def ccl_gemm(plan: Plan, A_ccl, B_ccl, C_ccl, stream=None) -> None:
    _check(library().ccl_gemm(plan, _ptr(A_ccl), _ptr(B_ccl), _ptr(C_ccl), _stream(stream)))


def ccl_gemm_scaled(plan: Plan, alpha: float, A_ccl, B_ccl, beta: float, C_ccl, stream=None) -> None:
    _check(library().ccl_gemm_scaled(plan, alpha, _ptr(A_ccl), _ptr(B_ccl), beta, _ptr(C_ccl),
                                     _stream(stream)))


def ccl_gemm_splitk_workspace(plan: Plan, splits: int = 0) -> tuple[int, int]:
    """(K ranges used, workspace bytes) for a requested split count (0: choose)."""
    s = ctypes.c_int(splits)
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_gemm_splitk_workspace(plan, ctypes.byref(s), ctypes.byref(nbytes)))
    return s.value, nbytes.value


def ccl_gemm_splitk(plan: Plan, alpha: float, A_ccl, B_ccl, beta: float, C_ccl, splits: int,
                    workspace, workspace_bytes: int, stream=None) -> None:
    _check(library().ccl_gemm_splitk(plan, alpha, _ptr(A_ccl), _ptr(B_ccl), beta, _ptr(C_ccl),
                                     splits, _ptr(workspace), workspace_bytes, _stream(stream)))


def ccl_gemm_splitk_noalloc(plan: Plan, alpha: float, A_ccl, B_ccl, beta: float, C_ccl,
                            splits: int, stream=None) -> None:
    _check(library().ccl_gemm_splitk_noalloc(plan, ctypes.c_float(alpha), _ptr(A_ccl),
                                             _ptr(B_ccl), ctypes.c_float(beta), _ptr(C_ccl),
                                             splits, _stream(stream)))


def ccl_gemm_rowmajor(plan: Plan, A, B, C, remap: int, stream=None) -> None:
    _check(library().ccl_gemm_rowmajor(plan, _ptr(A), _ptr(B), _ptr(C), remap, _stream(stream)))


CCL_ACT_NONE, CCL_ACT_RELU, CCL_ACT_GELU, CCL_ACT_SILU = 0, 1, 2, 3
CCL_LAYOUT_CCL, CCL_LAYOUT_ROWMAJOR = 0, 1


def ccl_plan_matrix_layout(plan: Plan, cols: int) -> Layout:
    """Layout of a bf16 M x cols matrix on the plan's grid."""
    out = _Layout()
    _check(library().ccl_plan_matrix_layout(plan, cols, ctypes.byref(out)))
    return Layout(*(getattr(out, f) for f, _ in _Layout._fields_))


def ccl_gemm_fused_workspace(plan: Plan, splits: int = 1, *, layout: int = CCL_LAYOUT_CCL) -> tuple[int, int]:
    """(K ranges used, workspace bytes) of ccl_gemm_fused for a requested split count (0: choose)."""
    s = ctypes.c_int(splits)
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_gemm_fused_workspace(plan, layout, ctypes.byref(s), ctypes.byref(nbytes)))
    return s.value, nbytes.value


def _bias(bias, bias_type, n: int) -> tuple[int, int]:
    """Address and element type of a bias of n columns: the type as given, else a tensor's own (CCL_DT_FP32 for an
    address). A tensor has to hold n of them side by side."""
    if bias is None or isinstance(bias, int):
        return bias or 0, CCL_DT_FP32 if bias_type is None else bias_type
    own = {"torch.float32": CCL_DT_FP32, "torch.bfloat16": CCL_DT_BF16}.get(str(bias.dtype))
    if bias_type is None:
        bias_type = own
    size = {CCL_DT_FP32: 4, CCL_DT_BF16: 2}.get(bias_type)
    if size is None or (bias.dtype.is_floating_point and own != bias_type):
        _refuse("bias", f"a tensor of {bias.dtype}; the bias must be fp32 or bf16")
    if not bias.is_contiguous() or bias.nbytes < n * size:
        _refuse("bias", f"not {n} elements without gaps")
    return bias.data_ptr(), bias_type


def ccl_gemm_fused(plan: Plan, A, B, C, *, activation: int = CCL_ACT_NONE, gated: bool = False, bias=None,
                   bias_type: int | None = None, residual=None, beta: float = 1.0, preact=None, alpha: float = 1.0,
                   rows: int | None = None, layout: int = CCL_LAYOUT_CCL, splits: int = 1, workspace=None,
                   workspace_bytes: int = 0, stream=None) -> None:
    """C = act(alpha A B + bias) + beta residual, gated or not; preact takes alpha A B + bias."""
    bias, bias_type = _bias(bias, bias_type, plan.args[1])
    e = _Epilogue(activation, int(gated), layout, bias_type, alpha, beta, plan.args[0] if rows is None else rows, bias,
                  _ptr(residual), _ptr(preact))
    _check(library().ccl_gemm_fused(plan, ctypes.byref(e), _ptr(A), _ptr(B), _ptr(C), splits, _ptr(workspace),
                                    workspace_bytes, _stream(stream)))


def ccl_gemm_fused_grad_workspace(plan: Plan, *, gated: bool = False, dbias: bool = False,
                                  layout: int = CCL_LAYOUT_CCL) -> int:
    """Workspace bytes of ccl_gemm_fused_grad."""
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_gemm_fused_grad_workspace(plan, layout, int(gated), int(dbias), ctypes.byref(nbytes)))
    return nbytes.value


def ccl_gemm_fused_grad(plan: Plan, A, B, preact, dZ, *, activation: int = CCL_ACT_NONE, gated: bool = False,
                        dbias=None, alpha: float = 1.0, rows: int | None = None, layout: int = CCL_LAYOUT_CCL,
                        workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """dZ = (alpha A B) * act'(preact), gated or not; dbias takes its column sums."""
    if dbias is not None:
        import torch
        dbias = _whole("dbias", dbias, plan.args[1] * (2 if gated else 1), torch.float32)
    e = _EpilogueGrad(activation, int(gated), layout, alpha, plan.args[0] if rows is None else rows, _ptr(preact), dbias)
    _check(library().ccl_gemm_fused_grad(plan, ctypes.byref(e), _ptr(A), _ptr(B), _ptr(dZ), _ptr(workspace),
                                         workspace_bytes, _stream(stream)))


CCL_MOE_MAX_TOKENS = 64


def ccl_moe(*, hidden: int, ffn: int, experts: int, top_k: int, activation: int = CCL_ACT_SILU,
            normalize: bool = True, weight_type: int = CCL_DT_BF16, gate_up_ld: int = 0, gate_up_stride: int = 0,
            down_ld: int = 0, down_stride: int = 0) -> _Moe:
    """Description of a mixture-of-experts FFN layer for ccl_moe_decode."""
    return _Moe(hidden, ffn, experts, top_k, activation, int(normalize), weight_type, gate_up_ld, gate_up_stride,
                down_ld, down_stride)


def ccl_moe_workspace(moe: _Moe, tokens: int) -> int:
    """Workspace bytes of ccl_moe_decode for up to `tokens` tokens."""
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_moe_workspace(ctypes.byref(moe), tokens, ctypes.byref(nbytes)))
    return nbytes.value


def _rows(name: str, t, ld, rows: int, width: int, dtype, bits=None) -> tuple[int, int]:
    """Address of a rows x width operand and the elements between its rows: as given, else a tensor's own (its row
    length for an address or a flat tensor). A tensor has to be of dtype (or bits, an integer type that holds it)
    and to have its rows whole and as many as the call takes."""
    if t is None or isinstance(t, int):
        return t or 0, width if ld is None else ld
    if t.dtype is not dtype and (bits is None or t.dtype is not bits):
        _refuse(name, f"a tensor of {t.dtype}, not {dtype}")
    if ld is not None:
        return t.data_ptr(), ld
    shape, stride = t.shape, t.stride()
    if len(shape) > 2:
        try:
            flat = t.view(-1, shape[-1])
        except RuntimeError:
            _refuse(name, "rows that are not one stride apart")
        shape, stride = flat.shape, flat.stride()
    if len(shape) < 2:
        if not t.is_contiguous() or t.numel() < rows * width:
            _refuse(name, f"a flat tensor has to hold {rows} x {width} elements without gaps")
        return t.data_ptr(), width
    n, w = shape
    ld, step = stride
    if n < rows or w < width or (step != 1 and w > 1):
        _refuse(name, f"a tensor of {n} x {w} with columns {step} apart, not {rows} x {width} with columns side by side")
    return t.data_ptr(), ld if rows > 1 else width      # one row: a stride that means nothing


def _expert_weights(name: str, t, experts: int, rows: int, cols: int, ld: int, stride: int, dtype) -> int:
    """Address of a layer's weights, (experts, rows, cols) or raw memory of as many bytes."""
    if t is None or isinstance(t, int):
        return t or 0
    ld = ld or cols
    stride = stride or rows * ld
    if t.dtype is dtype:
        shape = t.shape
        if len(shape) == 3:
            steps = t.stride()
            apart = steps == (stride, ld, 1) or (experts == 1 and steps[1:] == (ld, 1))
            if shape[0] < experts or shape[1] < rows or shape[2] < cols or not apart:
                _refuse(name, f"{tuple(shape)} with strides {steps}, not {(experts, rows, cols)} with {(stride, ld, 1)}")
            return t.data_ptr()
    elif t.dtype.is_floating_point:
        _refuse(name, f"a tensor of {t.dtype}, not {dtype}")
    if not t.is_contiguous() or t.nbytes < ((experts - 1) * stride + (rows - 1) * ld + cols) * dtype.itemsize:
        _refuse(name, "smaller than the layer's weights, or with gaps")
    return t.data_ptr()


def ccl_moe_decode(moe: _Moe, tokens: int, x, logits, gate_up, down, y, *, ids=None, probs=None, gate_up_scale=None,
                   down_scale=None, workspace=None, workspace_bytes: int = 0, x_ld: int | None = None,
                   logits_ld: int | None = None, y_ld: int | None = None, stream=None) -> None:
    """y = the layer on `tokens` rows of x, routed by logits; ids and probs take the choice."""
    call = library().ccl_moe_decode
    import torch
    bf16, f32, bits = torch.bfloat16, torch.float32, torch.int16
    D, F, E = moe.hidden, moe.ffn, moe.experts
    w = torch.float8_e4m3fn if moe.weight_type == CCL_DT_FP8_E4M3 else bf16
    x, x_ld = _rows("x", x, x_ld, tokens, D, bf16, bits)
    logits, logits_ld = _rows("logits", logits, logits_ld, tokens, E, f32)
    y, y_ld = _rows("y", y, y_ld, tokens, D, bf16, bits)
    if ids is not None:
        ids = _whole("ids", ids, tokens * moe.top_k, torch.int32)
    if probs is not None:
        probs = _whole("probs", probs, tokens * moe.top_k, f32)
    if gate_up_scale is not None:
        gate_up_scale = _whole("gate_up_scale", gate_up_scale, E, f32)
    if down_scale is not None:
        down_scale = _whole("down_scale", down_scale, E, f32)
    gate_up = _expert_weights("gate_up", gate_up, E, 2 * F, D, moe.gate_up_ld, moe.gate_up_stride, w)
    down = _expert_weights("down", down, E, D, F, moe.down_ld, moe.down_stride, w)
    _check(call(ctypes.byref(moe), tokens, x, x_ld, logits, logits_ld, gate_up, gate_up_scale, down, down_scale, y, y_ld,
                ids, probs, _ptr(workspace), workspace_bytes, _stream(stream)))


def ccl_orthogonalize_workspace(batch: int, rows: int, cols: int) -> int:
    """Workspace bytes of ccl_orthogonalize."""
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_orthogonalize_workspace(batch, rows, cols, ctypes.byref(nbytes)))
    return nbytes.value


def ccl_orthogonalize(batch: int, rows: int, cols: int, G, g_type: int, ld: int, stride: int, O, *,
                      o_ld: int | None = None, o_stride: int | None = None, steps: int = 5, coeffs=None,
                      eps: float = 1e-7, workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """O = the Newton-Schulz orthogonalisation of each of the batch's matrices (O without gaps by default)."""
    c = None if coeffs is None else (ctypes.c_float * 3)(*coeffs)
    o_ld = cols if o_ld is None else o_ld
    _check(library().ccl_orthogonalize(batch, rows, cols, _ptr(G), g_type, ld, stride, steps, c, eps, _ptr(O), o_ld,
                                       rows * o_ld if o_stride is None else o_stride, _ptr(workspace), workspace_bytes,
                                       _stream(stream)))


def _here(**tensors) -> None:
    """Tensors of a call have to be on the current device, whose kernels read them."""
    at = None
    for name, t in tensors.items():
        if t is None or isinstance(t, int):
            continue
        if at is None:
            import torch
            at = torch.cuda.current_device() if t.is_cuda else 0
        if t.get_device() != at:
            _refuse(name, f"a tensor on {t.device}, not on the current GPU")


def _room(workspace, nbytes: int):
    """The address of a workspace of that many bytes, which a tensor has to hold."""
    if workspace is not None and not isinstance(workspace, int):
        if not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < nbytes:
            _refuse("workspace", f"a tensor that does not hold {nbytes} contiguous bytes")
    return _ptr(workspace)


CCL_GROUPED_FORWARD, CCL_GROUPED_GRAD, CCL_GROUPED_WGRAD = 0, 1, 2


def ccl_grouped(*, in_features: int, out_features: int, experts: int, activation: int = CCL_ACT_NONE, gated: bool = False,
                w_ld: int = 0, w_stride: int = 0) -> _Grouped:
    """Description of experts' products on sorted rows for the ccl_grouped_gemm calls."""
    return _Grouped(in_features, out_features, experts, activation, int(gated), w_ld, w_stride)


def ccl_grouped_gemm_workspace(grouped: _Grouped, rows: int, direction: int) -> int:
    """Workspace bytes of ccl_grouped_gemm, _grad or _wgrad for `rows` rows."""
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_grouped_gemm_workspace(ctypes.byref(grouped), rows, direction, ctypes.byref(nbytes)))
    return nbytes.value


def ccl_grouped_gemm(grouped: _Grouped, rows: int, ends, X, W, Y, *, preact=None, x_ld: int | None = None,
                     y_ld: int | None = None, z_ld: int | None = None, workspace=None, workspace_bytes: int = 0,
                     stream=None) -> None:
    """Y = act(X W_e^T), gated or not, on rows sorted by expert; preact takes X W_e^T."""
    call = library().ccl_grouped_gemm
    import torch
    bf16, bits = torch.bfloat16, torch.int16
    K, N, E = grouped.in_features, grouped.out_features, grouped.experts
    _here(ends=ends, X=X, W=W, Y=Y, preact=preact, workspace=workspace)
    X, x_ld = _rows("X", X, x_ld, rows, K, bf16, bits)
    Y, y_ld = _rows("Y", Y, y_ld, rows, N // 2 if grouped.gated else N, bf16, bits)
    preact, z_ld = _rows("preact", preact, z_ld, rows, N, bf16, bits)
    W = _expert_weights("W", W, E, N, K, grouped.w_ld, grouped.w_stride, bf16)
    _check(call(ctypes.byref(grouped), rows, _whole("ends", ends, E, torch.int32), X, x_ld, W, Y, y_ld, preact, z_ld,
                _room(workspace, workspace_bytes), workspace_bytes, _stream(stream)))


def ccl_grouped_gemm_grad(grouped: _Grouped, rows: int, ends, dY, W, dX, *, preact=None, dy_ld: int | None = None,
                          dx_ld: int | None = None, z_ld: int | None = None, workspace=None, workspace_bytes: int = 0,
                          stream=None) -> None:
    """dX = dY W_e on rows sorted by expert, or with an activation dZ = (dY W_e) * act'(preact), gated or not."""
    call = library().ccl_grouped_gemm_grad
    import torch
    bf16, bits = torch.bfloat16, torch.int16
    K, N, E = grouped.in_features, grouped.out_features, grouped.experts
    wide = 2 * K if grouped.gated else K
    _here(ends=ends, dY=dY, W=W, dX=dX, preact=preact, workspace=workspace)
    dY, dy_ld = _rows("dY", dY, dy_ld, rows, N, bf16, bits)
    dX, dx_ld = _rows("dX", dX, dx_ld, rows, wide, bf16, bits)
    preact, z_ld = _rows("preact", preact, z_ld, rows, wide, bf16, bits)
    W = _expert_weights("W", W, E, N, K, grouped.w_ld, grouped.w_stride, bf16)
    _check(call(ctypes.byref(grouped), rows, _whole("ends", ends, E, torch.int32), dY, dy_ld, W, dX, dx_ld, preact, z_ld,
                _room(workspace, workspace_bytes), workspace_bytes, _stream(stream)))


def ccl_grouped_gemm_wgrad(grouped: _Grouped, rows: int, ends, dY, X, dW, *, dw_type: int | None = None,
                           accumulate: bool = False, dy_ld: int | None = None, x_ld: int | None = None, workspace=None,
                           workspace_bytes: int = 0, stream=None) -> None:
    """dW_e = dY_e^T X_e (+ dW_e) over each expert's rows; dW's type is a tensor's own (bf16 for an address)."""
    call = library().ccl_grouped_gemm_wgrad
    import torch
    bf16, bits = torch.bfloat16, torch.int16
    K, N, E = grouped.in_features, grouped.out_features, grouped.experts
    _here(ends=ends, dY=dY, X=X, dW=dW, workspace=workspace)
    dY, dy_ld = _rows("dY", dY, dy_ld, rows, N, bf16, bits)
    X, x_ld = _rows("X", X, x_ld, rows, K, bf16, bits)
    if dw_type is None:
        dw_type = CCL_DT_FP32 if getattr(dW, "dtype", None) is torch.float32 else CCL_DT_BF16
    dW = _expert_weights("dW", dW, E, N, K, grouped.w_ld, grouped.w_stride,
                         torch.float32 if dw_type == CCL_DT_FP32 else bf16)
    _check(call(ctypes.byref(grouped), rows, _whole("ends", ends, E, torch.int32), dY, dy_ld, X, x_ld, dW, dw_type,
                int(accumulate), _room(workspace, workspace_bytes), workspace_bytes, _stream(stream)))


def ccl_vocab(*, hidden: int, vocab: int, scale: float = 1.0, w_ld: int = 0, block: int = 0) -> _Vocab:
    """Description of an output matrix and its loss for the ccl_cross_entropy calls."""
    return _Vocab(hidden, vocab, w_ld, block, scale)


def ccl_cross_entropy_workspace(vocab: _Vocab, tokens: int, *, grad: bool = False) -> int:
    """Workspace bytes of ccl_cross_entropy, or with grad of ccl_cross_entropy_grad."""
    nbytes = ctypes.c_int64(0)
    _check(library().ccl_cross_entropy_workspace(ctypes.byref(vocab), tokens, int(grad), ctypes.byref(nbytes)))
    return nbytes.value


def _vocab_weight(vocab: _Vocab, W, bf16) -> int:
    """Address of W, vocab x hidden with its rows as the description says."""
    if W is None or isinstance(W, int):
        return W or 0
    W, ld = _rows("W", W, None, vocab.vocab, vocab.hidden, bf16)
    if vocab.vocab > 1 and ld != (vocab.w_ld or vocab.hidden):
        _refuse("W", f"rows {ld} apart, not {vocab.w_ld or vocab.hidden}")
    return W


def ccl_cross_entropy(vocab: _Vocab, tokens: int, X, W, targets, loss, *, lse=None, x_ld: int | None = None,
                      workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """loss = log sum exp(scale X W^T) - the target's logit, one fp32 a token (0 without a target); lse takes the first term."""
    call = library().ccl_cross_entropy
    import torch
    bf16, f32 = torch.bfloat16, torch.float32
    _here(X=X, W=W, targets=targets, loss=loss, lse=lse, workspace=workspace)
    X, x_ld = _rows("X", X, x_ld, tokens, vocab.hidden, bf16, torch.int16)
    _check(call(ctypes.byref(vocab), tokens, X, x_ld, _vocab_weight(vocab, W, bf16),
                _whole("targets", targets, tokens, torch.int64), _whole("loss", loss, tokens, f32),
                _whole("lse", lse, tokens, f32), _room(workspace, workspace_bytes), workspace_bytes, _stream(stream)))


def ccl_cross_entropy_grad(vocab: _Vocab, tokens: int, X, W, targets, loss, dX, dW, *, lse=None, dloss=None,
                           dloss_scale: float = 1.0, dw_type: int | None = None, accumulate: bool = False,
                           x_ld: int | None = None, dx_ld: int | None = None, dw_ld: int | None = None, workspace=None,
                           workspace_bytes: int = 0, stream=None) -> None:
    """The loss and its gradients for token weights dloss * dloss_scale, dX and dW (either may be None); dW's type is a
    tensor's own (bf16 for an address)."""
    call = library().ccl_cross_entropy_grad
    import torch
    bf16, f32 = torch.bfloat16, torch.float32
    if dw_type is None:
        dw_type = CCL_DT_FP32 if getattr(dW, "dtype", None) is f32 else CCL_DT_BF16
    D = vocab.hidden
    _here(X=X, W=W, targets=targets, loss=loss, dX=dX, dW=dW, lse=lse, dloss=dloss, workspace=workspace)
    X, x_ld = _rows("X", X, x_ld, tokens, D, bf16, torch.int16)
    dX, dx_ld = _rows("dX", dX, dx_ld, tokens, D, bf16, torch.int16)
    dW, dw_ld = _rows("dW", dW, dw_ld, vocab.vocab, D, f32 if dw_type == CCL_DT_FP32 else bf16)
    _check(call(ctypes.byref(vocab), tokens, X, x_ld, _vocab_weight(vocab, W, bf16),
                _whole("targets", targets, tokens, torch.int64), _whole("dloss", dloss, tokens, f32), dloss_scale,
                _whole("loss", loss, tokens, f32), _whole("lse", lse, tokens, f32), dX, dx_ld, dW, dw_ld, dw_type,
                int(accumulate), _room(workspace, workspace_bytes), workspace_bytes, _stream(stream)))


CCL_ADAMW_BLOCK = 128               # elements of 8-bit moments that share a scale


def _adamw_types() -> dict:
    import torch
    return {torch.float32: CCL_DT_FP32, torch.bfloat16: CCL_DT_BF16}


def ccl_adamw_tensor(param, grad, exp_avg, exp_avg_sq, *, exp_avg_scale=None, exp_avg_sq_scale=None, copy=None,
                     weight_decay: float = 0.0) -> tuple[_AdamwTensor, tuple]:
    """One tensor of a ccl_adamw set: contiguous tensors of as many elements; uint8 moments (with their scales, one byte
    for every 128) are 8-bit ones. The set keeps the tensors alive and steps with these, whatever param.grad becomes."""
    import torch
    types = _adamw_types()
    n = param.numel()
    at = param.get_device()
    for name, t in (("grad", grad), ("exp_avg", exp_avg), ("exp_avg_sq", exp_avg_sq), ("exp_avg_scale", exp_avg_scale),
                    ("exp_avg_sq_scale", exp_avg_sq_scale), ("copy", copy)):
        if t is not None and t.get_device() != at:
            _refuse(name, f"a tensor on {t.device}, the param on {param.device}")
    for name, t in (("param", param), ("grad", grad)):
        if t.dtype not in types:
            _refuse(name, f"a tensor of {t.dtype}, not fp32 or bf16")
    bits = 8 if exp_avg.dtype is torch.uint8 else 32
    moment = torch.uint8 if bits == 8 else torch.float32
    blocks = -(-n // CCL_ADAMW_BLOCK)

    def exact(name, t, count, dtype):
        if t is not None and t.numel() != count:
            _refuse(name, f"{t.numel()} elements, not {count}")
        return _whole(name, t, count, dtype)
    scales = (exact("exp_avg_scale", exp_avg_scale, blocks, torch.uint8),
              exact("exp_avg_sq_scale", exp_avg_sq_scale, blocks, torch.uint8)) if bits == 8 else (0, 0)
    t = _AdamwTensor(exact("param", param, n, param.dtype), exact("grad", grad, n, grad.dtype),
                     exact("exp_avg", exp_avg, n, moment), exact("exp_avg_sq", exp_avg_sq, n, moment), *scales,
                     exact("copy", copy, n, torch.bfloat16), n, types[param.dtype], types[grad.dtype], bits, weight_decay)
    return t, (param, grad, exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale, copy)


class AdamwSet:
    """Tensors for ccl_adamw_step, held while it lives. A step reads them where they lay when they were given: gradients
    that have other storage since (as behind torch's zero_grad(), which drops them) are given anew with grads()."""

    def __init__(self, tensors):
        tensors = list(tensors)
        self.device = {held[0].get_device() for t, held in tensors if held and t.n}
        self.tensors = (_AdamwTensor * len(tensors))(*(t for t, _ in tensors))
        self.kept = [held for _, held in tensors]

    def grads(self, grads) -> "AdamwSet":
        """Other gradients for the tensors, one each in their order, for the steps from here on (a captured step keeps
        those it was captured with)."""
        grads, new, types = list(grads), [], _adamw_types()
        if len(grads) != len(self.tensors):
            _refuse("grads", f"{len(grads)} gradients for {len(self.tensors)} tensors")
        for t, held, g in zip(self.tensors, self.kept, grads):
            if g is None or g.dtype not in types or g.numel() != t.n:
                _refuse("grads", f"not {t.n} elements of fp32 or bf16")
            if held and g.device != held[0].device:
                _refuse("grads", f"a tensor on {g.device}, the param on {held[0].device}")
            new.append(_whole("grads", g, t.n, g.dtype))
        for i, (t, g, address) in enumerate(zip(self.tensors, grads, new)):
            t.grad, t.grad_type = address, types[g.dtype]
            held = self.kept[i]
            self.kept[i] = (*held[:1], g, *held[2:])
        return self


def ccl_adamw(tensors) -> AdamwSet:
    """A set of ccl_adamw_tensor to step together; set.grads(...) replaces its gradients."""
    return AdamwSet(tensors)


def ccl_adamw_step(tensors: AdamwSet, *, lr: float, step: int = 0, beta1: float = 0.9, beta2: float = 0.999,
                   eps: float = 1e-8, step_ptr=None, lr_ptr=None, grad_scale=None, stream=None) -> None:
    """One AdamW step of the set; step counts from 1. step_ptr (int64), lr_ptr and grad_scale (fp32): one element on the
    device, read when the step runs."""
    call = library().ccl_adamw_step
    import torch
    if tensors.device:
        at = torch.cuda.current_device() if torch.cuda.is_initialized() else -1
        if tensors.device != {at} or at < 0:
            _refuse("tensors", "not all on the current GPU")
    _here(step_ptr=step_ptr, lr_ptr=lr_ptr, grad_scale=grad_scale)
    a = _Adamw(lr, beta1, beta2, eps, step, _whole("step_ptr", step_ptr, 1, torch.int64),
               _whole("lr_ptr", lr_ptr, 1, torch.float32), _whole("grad_scale", grad_scale, 1, torch.float32))
    _check(call(ctypes.byref(a), tensors.tensors, len(tensors.tensors), _stream(stream)))


def ccl_adamw_moments(n: int, exp_avg, exp_avg_scale, exp_avg_sq, exp_avg_sq_scale, m, v, *, stream=None) -> None:
    """The values of n 8-bit moments, to m and v (fp32 or bf16 tensors of one type; either may be None). With exp_avg, v
    is what a step reads: not 0 where exp_avg is not."""
    call = library().ccl_adamw_moments
    import torch
    u8, blocks = torch.uint8, -(-n // CCL_ADAMW_BLOCK)
    dtype = next((t.dtype for t in (m, v) if t is not None), torch.float32)
    if dtype not in (torch.float32, torch.bfloat16):
        _refuse("m and v", f"tensors of {dtype}, not fp32 or bf16")
    _here(exp_avg=exp_avg, exp_avg_scale=exp_avg_scale, exp_avg_sq=exp_avg_sq, exp_avg_sq_scale=exp_avg_sq_scale, m=m, v=v)
    _check(call(n, _whole("exp_avg", exp_avg, n, u8), _whole("exp_avg_scale", exp_avg_scale, blocks, u8),
                _whole("exp_avg_sq", exp_avg_sq, n, u8), _whole("exp_avg_sq_scale", exp_avg_sq_scale, blocks, u8),
                _whole("m", m, n, dtype), _whole("v", v, n, dtype), CCL_DT_BF16 if dtype is torch.bfloat16 else CCL_DT_FP32,
                _stream(stream)))


CCL_TRAFFIC_A_TRANS, CCL_TRAFFIC_B_TRANS, CCL_TRAFFIC_C_READ = 1, 2, 4


def ccl_remote_bytes(plan: Plan, placement: int, flags: int) -> dict:
    t = _Traffic()
    _check(library().ccl_remote_bytes(plan, placement, flags, ctypes.byref(t)))
    return {
        "accessed": list(t.accessed),
        "remote": list(t.remote),
        "remote_per_chiplet": list(t.remote_per_chiplet[:t.chiplets]),
        "floor": int(t.floor_bytes),
        "footprint": list(t.footprint),
    }


def ccl_remote_bytes_l2(plan: Plan, placement: int, flags: int, *, l2_bytes: int,
                        slots: int, ways: int = 16, line_bytes: int = 128, k_step: int = 64,
                        traversal: int = 0, threads: int = 0, group_rows: int = 0) -> dict:
    cfg = _L2Config(l2_bytes, ways, line_bytes, slots, k_step, traversal, threads, group_rows)
    t = _L2Traffic()
    _check(library().ccl_remote_bytes_l2(plan, placement, flags, ctypes.byref(cfg),
                                         ctypes.byref(t)))
    return {
        "accesses": list(t.accesses),
        "misses": list(t.misses),
        "remote": list(t.remote),
        "remote_per_chiplet": list(t.remote_per_chiplet[:t.chiplets]),
    }


def ccl_status_string(status: int) -> str:
    return library().ccl_status_string(status).decode()


def ccl_last_error() -> str:
    return library().ccl_last_error().decode()


def ccl_debug_tile_of_wg(plan: Plan, wg: int) -> tuple[int, int, int]:
    x, tm, tn = ctypes.c_int(), ctypes.c_int64(), ctypes.c_int64()
    _check(library().ccl_debug_tile_of_wg(plan, wg, ctypes.byref(x), ctypes.byref(tm), ctypes.byref(tn)))
    return x.value, tm.value, tn.value


def ccl_debug_gemm_config(plan: Plan) -> tuple[int, int, int]:
    r, c, w = ctypes.c_int(), ctypes.c_int(), ctypes.c_int64()
    _check(library().ccl_debug_gemm_config(plan, ctypes.byref(r), ctypes.byref(c), ctypes.byref(w)))
    return r.value, c.value, w.value


def ccl_debug_dispatch(plan: Plan, out, stream=None) -> None:
    _check(library().ccl_debug_dispatch(plan, _ptr(out), _stream(stream)))


def ccl_debug_gemm_timeline(plan: Plan, A_ccl, B_ccl, C_ccl, timeline, timeline_bytes: int,
                            stream=None) -> None:
    _check(library().ccl_debug_gemm_timeline(plan, _ptr(A_ccl), _ptr(B_ccl), _ptr(C_ccl),
                                             _ptr(timeline), timeline_bytes, _stream(stream)))


@dataclass
class Launch:
    kernel: str
    workgroups: int
    tile_rows: int
    tile_cols: int
    waves: int
    k_ranges: int
    ragged: bool
    far: bool
    stream_b: bool
    c_nt: bool


def ccl_debug_launch(plan: Plan, splits: int = 1, operands: int = 0, reads_c: int = 0) -> Launch:
    out = _Launch()
    _check(library().ccl_debug_launch(plan, splits, operands, reads_c, ctypes.byref(out)))
    return Launch(out.kernel.decode(), out.workgroups, out.tile_rows, out.tile_cols, out.waves, out.k_ranges,
                  bool(out.ragged), bool(out.far), bool(out.stream_b), bool(out.c_nt))


def ccl_debug_launch_tile_of_wg(plan: Plan, wg: int) -> tuple[int, int, int]:
    x, tm, tn = ctypes.c_int(), ctypes.c_int64(), ctypes.c_int64()
    _check(library().ccl_debug_launch_tile_of_wg(plan, wg, ctypes.byref(x), ctypes.byref(tm), ctypes.byref(tn)))
    return x.value, tm.value, tn.value


def ccl_debug_launch_dispatch(plan: Plan, out, stream=None) -> None:
    _check(library().ccl_debug_launch_dispatch(plan, _ptr(out), _stream(stream)))


def ccl_debug_launch_timeline(plan: Plan, A_ccl, B_ccl, C_ccl, timeline, timeline_bytes: int,
                              stream=None) -> None:
    _check(library().ccl_debug_launch_timeline(plan, _ptr(A_ccl), _ptr(B_ccl), _ptr(C_ccl),
                                               _ptr(timeline), timeline_bytes, _stream(stream)))
