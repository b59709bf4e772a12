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
            "ccl_orthogonalize_workspace", "ccl_orthogonalize", "ccl_remote_bytes", "ccl_remote_bytes_l2", "ccl_status_string", "ccl_last_error",
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
