"""Thin Python binding of the C ABI in include/vlut.h (argument marshalling only).

Device buffers are torch tensors on a ROCm device; this module passes their raw
pointers and the current HIP stream to libvlut.so.  Every step of the path runs
inside the library's kernels; there is no fallback: if the library is missing or
a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import sys
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvlut.so")
NATIVE_PATH = os.path.join(_HERE, "_vlut_torch.so")

VLUT_OK = 0
VLUT_ERR_NULL, VLUT_ERR_SHAPE, VLUT_ERR_SMALL_BUFFER = -1, -2, -3
VLUT_ERR_VALUE, VLUT_ERR_DEVICE, VLUT_ERR_UNSUPPORTED = -4, -5, -6

EXPORTS = [
    "vlut_status_string", "vlut_version", "vlut_packed_weight_bytes", "vlut_packed_offset", "vlut_act_bytes",
    "vlut_lut_bytes",
    "vlut_workspace_bytes", "vlut_pack_weights", "vlut_quantize_act", "vlut_build_lut", "vlut_mpgemm",
    "vlut_mpgemm_rows", "vlut_mpgemm_mfma", "vlut_mfma_workspace_bytes", "vlut_set_plan", "vlut_query_plan",
    "vlut_packed_weight_bytes_g5", "vlut_packed_offset_g5", "vlut_workspace_bytes_g5", "vlut_pack_weights_g5",
    "vlut_mpgemm_g5", "vlut_set_plan_g5", "vlut_query_plan_g5",
    "vlut_workspace_bytes_f32", "vlut_query_plan_f32", "vlut_mpgemm_f32",
    "vlut_build_lut_token_outer", "vlut_mpgemm_token_outer",
    "vlut_mixed_k5", "vlut_packed_weight_bytes_mixed", "vlut_workspace_bytes_mixed", "vlut_pack_weights_mixed",
    "vlut_mpgemm_mixed", "vlut_static_scratch_bytes", "vlut_mpgemm_static", "vlut_query_lookup_waves",
    "vlut_query_kernel", "vlut_query_matrix_plan", "vlut_workspace_used", "vlut_workspace_used_g5", "vlut_workspace_used_mixed",
    "vlut_mpgemm_lean", "vlut_mpgemm_g5_lean", "vlut_mpgemm_mixed_lean",
    "vlut_norm_rope", "vlut_append_kv", "vlut_shared_prefix_attention", "vlut_shared_prefix_attention_bytes",
    "vlut_query_shared_prefix_attention",
    "vlut_chunk_attention", "vlut_chunk_attention_bytes", "vlut_query_chunk_attention",
    "vlut_residual_norm", "vlut_gated_norm", "vlut_token_logprobs", "vlut_token_logprobs_bytes",
]

_lib = None


class _Heads(ctypes.Structure):          # vlut_heads
    _fields_ = [("data", ctypes.c_void_p), ("weight", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("weight_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("type", ctypes.c_int32)]


class _Rotation(ctypes.Structure):       # vlut_rotation
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("features", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class _Cache(ctypes.Structure):          # vlut_cache
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("k_page", ctypes.c_int64), ("k_head", ctypes.c_int64), ("k_token", ctypes.c_int64),
                ("v_page", ctypes.c_int64), ("v_head", ctypes.c_int64), ("v_token", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("type", ctypes.c_int32)]


class _Rows(ctypes.Structure):           # vlut_rows
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("type", ctypes.c_int32)]


class VlutError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def lib() -> ctypes.CDLL:
    """Loads libvlut.so; building it is the job of __graft_entry__.build() / paper_2512_06443_amd.build."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_06443_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        i64, sz, p, ci, cf = ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
        L.vlut_status_string.argtypes, L.vlut_status_string.restype = [ci], ctypes.c_char_p
        L.vlut_version.argtypes, L.vlut_version.restype = [], ci
        L.vlut_packed_weight_bytes.argtypes, L.vlut_packed_weight_bytes.restype = [i64, i64], sz
        L.vlut_packed_offset.argtypes, L.vlut_packed_offset.restype = [i64, i64, i64, i64], sz
        L.vlut_act_bytes.argtypes, L.vlut_act_bytes.restype = [i64, i64], sz
        L.vlut_lut_bytes.argtypes, L.vlut_lut_bytes.restype = [i64, i64], sz
        L.vlut_workspace_bytes.argtypes, L.vlut_workspace_bytes.restype = [i64, i64, i64], sz
        L.vlut_mfma_workspace_bytes.argtypes, L.vlut_mfma_workspace_bytes.restype = [i64, i64, i64], sz
        L.vlut_pack_weights.argtypes, L.vlut_pack_weights.restype = [p, i64, i64, p, sz, p], ci
        L.vlut_quantize_act.argtypes, L.vlut_quantize_act.restype = [p, i64, i64, i64, p, p, p], ci
        L.vlut_build_lut.argtypes, L.vlut_build_lut.restype = [p, i64, i64, p, sz, p], ci
        gemm_args = [p, cf, p, p, p, i64, i64, i64, p, i64, p, p, sz, p]
        L.vlut_mpgemm.argtypes, L.vlut_mpgemm.restype = gemm_args, ci
        L.vlut_mpgemm_mfma.argtypes, L.vlut_mpgemm_mfma.restype = gemm_args, ci
        L.vlut_mpgemm_lean.argtypes, L.vlut_mpgemm_lean.restype = gemm_args, ci
        for f in (L.vlut_workspace_used, L.vlut_workspace_used_g5, L.vlut_workspace_used_mixed):
            f.argtypes, f.restype = [i64, i64, i64], sz
        for f in (L.vlut_mpgemm_g5_lean, L.vlut_mpgemm_mixed_lean):
            f.argtypes, f.restype = [p, cf, p, p, i64, i64, i64, p, i64, p, p, sz, p], ci
        L.vlut_mpgemm_rows.argtypes, L.vlut_mpgemm_rows.restype = [p, p] + list(gemm_args[2:]), ci
        L.vlut_packed_weight_bytes_g5.argtypes, L.vlut_packed_weight_bytes_g5.restype = [i64, i64], sz
        L.vlut_packed_offset_g5.argtypes, L.vlut_packed_offset_g5.restype = [i64, i64, i64, i64], sz
        L.vlut_workspace_bytes_g5.argtypes, L.vlut_workspace_bytes_g5.restype = [i64, i64, i64], sz
        L.vlut_pack_weights_g5.argtypes, L.vlut_pack_weights_g5.restype = [p, i64, i64, p, sz, p], ci
        L.vlut_mpgemm_g5.argtypes, L.vlut_mpgemm_g5.restype = [p, cf, p, p, i64, i64, i64, p, i64, p, p, sz, p], ci
        L.vlut_set_plan_g5.argtypes, L.vlut_set_plan_g5.restype = [ci, ci], ci
        L.vlut_query_plan_g5.argtypes, L.vlut_query_plan_g5.restype = [i64, i64, i64, ctypes.POINTER(ci)], ci
        L.vlut_mixed_k5.argtypes, L.vlut_mixed_k5.restype = [i64], i64
        L.vlut_packed_weight_bytes_mixed.argtypes, L.vlut_packed_weight_bytes_mixed.restype = [i64, i64], sz
        L.vlut_workspace_bytes_mixed.argtypes, L.vlut_workspace_bytes_mixed.restype = [i64, i64, i64], sz
        L.vlut_pack_weights_mixed.argtypes, L.vlut_pack_weights_mixed.restype = [p, i64, i64, p, sz, p], ci
        L.vlut_mpgemm_mixed.argtypes, L.vlut_mpgemm_mixed.restype = [p, cf, p, p, i64, i64, i64, p, i64, p, p, sz, p], ci
        L.vlut_build_lut_token_outer.argtypes, L.vlut_build_lut_token_outer.restype = [p, i64, i64, p, sz, p], ci
        L.vlut_mpgemm_token_outer.argtypes = [p, cf, p, p, i64, i64, i64, p, i64, p, p]
        L.vlut_mpgemm_token_outer.restype = ci
        L.vlut_workspace_bytes_f32.argtypes, L.vlut_workspace_bytes_f32.restype = [i64, i64, i64], sz
        L.vlut_query_plan_f32.argtypes, L.vlut_query_plan_f32.restype = [i64, i64, i64, ctypes.POINTER(ci)], ci
        L.vlut_mpgemm_f32.argtypes = [p, cf, p, p, i64, i64, i64, i64, p, i64, p, p, p, sz, p]
        L.vlut_mpgemm_f32.restype = ci
        L.vlut_query_lookup_waves.argtypes, L.vlut_query_lookup_waves.restype = [i64, i64, i64], ci
        L.vlut_query_kernel.argtypes, L.vlut_query_kernel.restype = [ci, i64, i64, i64], ci
        L.vlut_query_matrix_plan.argtypes, L.vlut_query_matrix_plan.restype = [ci, i64, i64, i64, ctypes.POINTER(ci)], ci
        L.vlut_static_scratch_bytes.argtypes, L.vlut_static_scratch_bytes.restype = [], sz
        L.vlut_mpgemm_static.argtypes, L.vlut_mpgemm_static.restype = [p, cf, p, p, i64, i64, i64, p, i64, p, p], ci
        heads, rotation, cache = (ctypes.POINTER(s) for s in (_Heads, _Rotation, _Cache))
        L.vlut_norm_rope.argtypes, L.vlut_norm_rope.restype = [heads, heads, cf, rotation, i64, i64, heads, heads, p], ci
        L.vlut_append_kv.argtypes, L.vlut_append_kv.restype = [heads, heads, heads, cf, rotation, p, i64, i64, cache, heads, p], ci
        L.vlut_shared_prefix_attention_bytes.argtypes, L.vlut_shared_prefix_attention_bytes.restype = [i64] * 7, sz
        L.vlut_query_shared_prefix_attention.argtypes = [i64] * 7 + [ctypes.POINTER(ci)]
        L.vlut_query_shared_prefix_attention.restype = ci
        L.vlut_shared_prefix_attention.argtypes = [heads, i64, cache, p, i64, p, i64, p, i64, p, i64, i64, i64, cf, heads, i64, p, p, sz, p]
        L.vlut_shared_prefix_attention.restype = ci
        L.vlut_chunk_attention_bytes.argtypes, L.vlut_chunk_attention_bytes.restype = [i64] * 8, sz
        L.vlut_query_chunk_attention.argtypes, L.vlut_query_chunk_attention.restype = [i64] * 8 + [ctypes.POINTER(ci)], ci
        L.vlut_chunk_attention.argtypes = [heads, cache, p, i64, p, p, i64, i64, i64, i64, i64, i64, cf, heads, p, p, sz, p]
        L.vlut_chunk_attention.restype = ci
        rows = ctypes.POINTER(_Rows)
        L.vlut_residual_norm.argtypes, L.vlut_residual_norm.restype = [rows, p, rows, ci, cf, rows, p, cf, i64, i64, rows, rows, p], ci
        L.vlut_gated_norm.argtypes, L.vlut_gated_norm.restype = [rows, rows, ci, p, cf, i64, i64, rows, p], ci
        L.vlut_token_logprobs_bytes.argtypes, L.vlut_token_logprobs_bytes.restype = [i64, i64, ci], sz
        L.vlut_token_logprobs.argtypes, L.vlut_token_logprobs.restype = [rows, p, cf, ci, i64, i64, p, p, p, p, p, sz, p], ci
        L.vlut_set_plan.argtypes, L.vlut_set_plan.restype = [ci, ci, ci, ci], ci
        L.vlut_query_plan.argtypes, L.vlut_query_plan.restype = [i64, i64, i64, ctypes.POINTER(ci)], ci
        _load_native(L)
        _lib = L
    return _lib


# The frequent calls as native code (csrc/torch_calls.cpp): the same arguments, outputs and library call without ctypes and without
# torch's Python layer.  Each returns None for arguments it leaves to the Python form below it (which also raises every
# error), an int status or the tuple of outputs.  None here: not built, or built for another torch; the Python form serves then.
# The products take the lean form of the call: no workspace is allocated where the kernel leaves it alone (0.75 us each).
# Host time of a call, Python / native form, us (640 x 2560, four tokens; the launch alone is 2.2): quantize_act 7.9 / 4.9,
# mpgemm 7.6 / 4.4, with y and workspace given 5.5 / 3.4, mpgemm_g5 and mpgemm_mixed 4.5, mpgemm_f32 7.6 / 4.4; with a workspace for
# each call, a launch by <<< >>> and the rules worked out anew 5.3, 4.6, 3.6, 5.9 and 4.5 (hosts differ: the native forms 4.5, 3.8, 2.9, 3.9
# and 3.8 on another; with a layer's four matrices in turn within 0.2 of that).
_native = None
_NATIVE_ORDER = ("vlut_quantize_act", "vlut_mpgemm_lean", "vlut_workspace_used", "vlut_mpgemm_f32", "vlut_workspace_bytes_f32", "vlut_mpgemm_g5_lean",
                 "vlut_workspace_used_g5", "vlut_mpgemm_mixed_lean", "vlut_workspace_used_mixed", "vlut_pack_weights",
                 "vlut_packed_weight_bytes", "vlut_pack_weights_g5", "vlut_packed_weight_bytes_g5", "vlut_pack_weights_mixed",
                 "vlut_packed_weight_bytes_mixed")

_NATIVE_ATTENTION_ORDER = ("vlut_norm_rope", "vlut_append_kv", "vlut_shared_prefix_attention", "vlut_shared_prefix_attention_bytes")
_NATIVE_LAYER_ORDER = ("vlut_chunk_attention", "vlut_chunk_attention_bytes", "vlut_residual_norm", "vlut_gated_norm", "vlut_token_logprobs", "vlut_token_logprobs_bytes")


def built_for() -> str:
    """What NATIVE_PATH is compiled against: it holds layouts and key numbers of torch's headers, and a file for others may load all the same."""
    return f"torch {torch.__version__} {getattr(torch.version, 'git_version', '')} python {sys.version_info[0]}.{sys.version_info[1]}"


def _load_native(L: ctypes.CDLL) -> None:
    global _native
    if not os.path.exists(NATIVE_PATH) or not hasattr(torch._C, "_cuda_getCurrentRawStream"):
        return
    try:
        spec = importlib.util.spec_from_file_location("_vlut_torch", NATIVE_PATH)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
    except ImportError:                 # built for another torch
        return
    if getattr(mod, "built_for", None) != built_for():      # (whose symbols are all here)
        return
    for bind, order in ((mod.bind, _NATIVE_ORDER), (mod.bind_attention, _NATIVE_ATTENTION_ORDER), (mod.bind_layer, _NATIVE_LAYER_ORDER)):
        bind(*[ctypes.cast(getattr(L, f), ctypes.c_void_p).value for f in order])
    _native = mod


def status_string(status: int) -> str:
    return lib().vlut_status_string(status).decode()


def _check(status: int, where: str) -> None:
    if status != VLUT_OK:
        raise VlutError(status, where)


# The raw handle of the current device's current stream.  torch.cuda.current_stream() builds a Stream object around the same
# handle, 2.7 us of a call that takes 8.7; asking for the handle itself takes 0.1.  The two functions are private names of torch:
# where a build does not have them (one without a GPU, on which the size helpers still work) the public call serves.
if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
    _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

    def _stream() -> int:
        return _raw_stream(_device())
else:
    def _stream() -> int:
        return torch.cuda.current_stream().cuda_stream


def _outputs(r, where: str):
    """What a native call returned: the outputs, or the status of a call that was refused."""
    if type(r) is tuple:
        return r
    raise VlutError(r, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def packed_weight_bytes(M: int, K: int) -> int:
    return lib().vlut_packed_weight_bytes(M, K)


def packed_offset(M: int, K: int, m: int, kg: int) -> int:
    return lib().vlut_packed_offset(M, K, m, kg)


def act_bytes(K: int, N: int) -> int:
    return lib().vlut_act_bytes(K, N)


def act_chunked_to_kn(a_q: torch.Tensor, N: int) -> torch.Tensor:
    """View helper for checks: token-chunked int8 [ceil(N/8)][K][8] -> plain [K][N] (a copy)."""
    C, K, _ = a_q.shape
    return a_q.permute(1, 0, 2).reshape(K, C * 8)[:, :N].contiguous()


def lut_bytes(K: int, N: int) -> int:
    return lib().vlut_lut_bytes(K, N)


def _workspace(t: Optional[torch.Tensor]) -> None:
    """A caller's workspace, of which kernels write as many bytes as its elements have, from its address on."""
    if t is not None and not (t.is_cuda and t.is_contiguous()):
        raise ValueError("workspace: a contiguous GPU tensor is wanted")


def workspace_bytes(M: int, K: int, N: int) -> int:
    return lib().vlut_workspace_bytes(M, K, N)


def set_plan(J: int = 0, R: int = 0, waves: int = 0, split_k: int = 0) -> None:
    _check(lib().vlut_set_plan(J, R, waves, split_k), "vlut_set_plan")


def query_plan(M: int, K: int, N: int) -> Tuple[int, int, int, int]:
    out = (ctypes.c_int * 4)()
    _check(lib().vlut_query_plan(M, K, N, out), "vlut_query_plan")
    return out[0], out[1], out[2], out[3]


def pack_weights(w_ternary: torch.Tensor) -> torch.Tensor:
    """int8 [M][K] on the GPU -> packed uint8 blob (opaque tile layout) on the GPU."""
    if _native is not None:
        r = _native.pack_weights(w_ternary)
        if r is not None:
            return _outputs(r, "vlut_pack_weights")[0]
    assert w_ternary.is_cuda and w_ternary.dtype == torch.int8 and w_ternary.is_contiguous()
    M, K = w_ternary.shape
    nbytes = packed_weight_bytes(M, K)
    if nbytes == 0:
        raise VlutError(VLUT_ERR_SHAPE, "vlut_packed_weight_bytes")
    packed = torch.empty(nbytes, dtype=torch.uint8, device=w_ternary.device)
    _check(lib().vlut_pack_weights(_ptr(w_ternary), M, K, _ptr(packed), nbytes, _stream()), "vlut_pack_weights")
    return packed


def quantize_act(x: torch.Tensor, a_q: Optional[torch.Tensor] = None, a_scale: Optional[torch.Tensor] = None):
    """fp32 [N][K] (row stride >= K) -> (int8 token-chunked [ceil(N/8)][K][8], fp32 [N])."""
    if _native is not None:
        r = _native.quantize_act(x, a_q, a_scale)
        if r is not None:
            return _outputs(r, "vlut_quantize_act")
    assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    N, K = x.shape
    if a_q is None:
        a_q = torch.empty(((N + 7) // 8, K, 8), dtype=torch.int8, device=x.device)
    if a_scale is None:
        a_scale = torch.empty(N, dtype=torch.float32, device=x.device)
    _check(lib().vlut_quantize_act(_ptr(x), N, K, x.stride(0), _ptr(a_q), _ptr(a_scale), _stream()), "vlut_quantize_act")
    return a_q, a_scale


def build_lut(a_q: torch.Tensor, N: int, lut: Optional[torch.Tensor] = None) -> torch.Tensor:
    assert a_q.is_cuda and a_q.dtype == torch.int8 and a_q.is_contiguous() and a_q.dim() == 3
    K = a_q.shape[1]
    assert a_q.shape[0] == (N + 7) // 8
    if lut is None:
        lut = torch.empty((K // 4, 81, N), dtype=torch.int16, device=a_q.device)
    _check(lib().vlut_build_lut(_ptr(a_q), K, N, _ptr(lut), lut.numel() * 2, _stream()), "vlut_build_lut")
    return lut


def mpgemm(packed: torch.Tensor, w_scale: float, a_q: torch.Tensor, a_scale: torch.Tensor, M: int,
           y: Optional[torch.Tensor] = None, acc: Optional[torch.Tensor] = None, lut: Optional[torch.Tensor] = None,
           workspace: Optional[torch.Tensor] = None, want_acc: bool = False, mfma: bool = False):
    """Runs vlut_mpgemm (or the MFMA comparison path).  Returns (y fp32 [N][M], acc int32 [M][N] or None)."""
    if _native is not None and lut is None and not mfma:
        r = _native.mpgemm(packed, w_scale, a_q, a_scale, M, y, acc, want_acc, workspace)
        if r is not None:
            return _outputs(r, "vlut_mpgemm")
    K, N = a_q.shape[1], a_scale.shape[0]
    dev = a_q.device
    if y is None:
        y = torch.empty((N, M), dtype=torch.float32, device=dev)
    if acc is None and want_acc:
        acc = torch.empty((M, N), dtype=torch.int32, device=dev)
    _workspace(workspace)
    ws_bytes = lib().vlut_mfma_workspace_bytes(M, K, N) if mfma else workspace_bytes(M, K, N)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    fn = lib().vlut_mpgemm_mfma if mfma else lib().vlut_mpgemm
    rc = fn(_ptr(packed), float(w_scale), _ptr(a_q), _ptr(a_scale), _ptr(lut), M, K, N, _ptr(y), y.stride(0),
            _ptr(acc), _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
            _stream())
    _check(rc, "vlut_mpgemm_mfma" if mfma else "vlut_mpgemm")
    return y, acc


def query_lookup_waves(M: int, K: int, N: int) -> int:
    """Lookup waves per workgroup (12 or 14) of the plan query_plan reports; 0 for the few-token kernel."""
    w = lib().vlut_query_lookup_waves(M, K, N)
    if w < 0:
        raise VlutError(w, "vlut_query_lookup_waves")
    return w


_FORMS = {"codes": 0, "f32": 1, "g5": 2, "mixed": 3}
_KERNELS = {1: "lookup", 2: "few_tokens", 3: "matrix", 4: "matrix_few_tokens"}


def query_kernel(form: str, M: int, K: int, N: int) -> str:
    """The kernel that computes the product of `mpgemm` ("codes"), `mpgemm_f32` ("f32"), `mpgemm_g5` ("g5") or
    `mpgemm_mixed` ("mixed"): "lookup", "few_tokens", "matrix" or "matrix_few_tokens" (VLUT_KERNEL_* of the header).
    From INT8 codes both "few_tokens" and "matrix" can be the matrix-core kernel for a few tokens: query_matrix_plan tells."""
    k = lib().vlut_query_kernel(_FORMS[form], M, K, N)
    if k < 0:
        raise VlutError(k, "vlut_query_kernel")
    return _KERNELS[k]


def query_matrix_plan(form: str, M: int, K: int, N: int) -> Optional[Tuple[int, int, int, int]]:
    """(rows, tokens, parts of K) of a workgroup and the number of workgroups of the matrix-core kernel that computes the
    product of such a call; up to 16 tokens: a kernel for a few tokens.  None where a kernel that looks up tables runs."""
    out = (ctypes.c_int * 4)()
    rc = lib().vlut_query_matrix_plan(_FORMS[form], M, K, N, out)
    if rc == VLUT_ERR_UNSUPPORTED and lib().vlut_query_kernel(_FORMS[form], M, K, N) > 0:
        return None
    _check(rc, "vlut_query_matrix_plan")
    return out[0], out[1], out[2], out[3]


def static_scratch_bytes() -> int:
    return lib().vlut_static_scratch_bytes()


def mpgemm_static(packed: torch.Tensor, w_scale: float, a_q: torch.Tensor, a_scale: torch.Tensor, M: int,
                  y: torch.Tensor, acc: Optional[torch.Tensor] = None):
    """Runs vlut_mpgemm_static: the caller passes inputs and outputs only, the split-K scratch is the library's own
    static device array; neither this wrapper nor the call allocates anything."""
    K, N = a_q.shape[1], a_scale.shape[0]
    rc = lib().vlut_mpgemm_static(_ptr(packed), float(w_scale), _ptr(a_q), _ptr(a_scale), M, K, N, _ptr(y), y.stride(0),
                                  _ptr(acc), _stream())
    _check(rc, "vlut_mpgemm_static")
    return y, acc


def mpgemm_rows(packed: torch.Tensor, w_scale_rows: torch.Tensor, a_q: torch.Tensor, a_scale: torch.Tensor, M: int,
                y: Optional[torch.Tensor] = None, want_acc: bool = False, workspace: Optional[torch.Tensor] = None):
    """Runs vlut_mpgemm_rows: stacked weight matrices, one weight scale per output row (fp32 [M] on the GPU)."""
    assert w_scale_rows.is_cuda and w_scale_rows.dtype == torch.float32 and w_scale_rows.numel() == M
    K, N = a_q.shape[1], a_scale.shape[0]
    dev = a_q.device
    if y is None:
        y = torch.empty((N, M), dtype=torch.float32, device=dev)
    acc = torch.empty((M, N), dtype=torch.int32, device=dev) if want_acc else None
    _workspace(workspace)
    ws_bytes = workspace_bytes(M, K, N)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    rc = lib().vlut_mpgemm_rows(_ptr(packed), _ptr(w_scale_rows), _ptr(a_q), _ptr(a_scale), None, M, K, N, _ptr(y),
                                y.stride(0), _ptr(acc), _ptr(workspace),
                                0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    _check(rc, "vlut_mpgemm_rows")
    return y, acc


def build_lut_token_outer(a_q: torch.Tensor, N: int) -> torch.Tensor:
    """The table with the token index outermost, int16 [N][K/4][81] (layout ablation)."""
    assert a_q.is_cuda and a_q.dtype == torch.int8 and a_q.is_contiguous() and a_q.dim() == 3
    K = a_q.shape[1]
    lut = torch.empty((N, K // 4, 81), dtype=torch.int16, device=a_q.device)
    _check(lib().vlut_build_lut_token_outer(_ptr(a_q), K, N, _ptr(lut), lut.numel() * 2, _stream()),
           "vlut_build_lut_token_outer")
    return lut


def mpgemm_token_outer(packed: torch.Tensor, w_scale: float, a_scale: torch.Tensor, lut: torch.Tensor, M: int,
                       want_acc: bool = False):
    """Runs vlut_mpgemm_token_outer on a table from build_lut_token_outer.  Returns (y [N][M], acc or None)."""
    N, G, _ = lut.shape
    y = torch.empty((N, M), dtype=torch.float32, device=lut.device)
    acc = torch.empty((M, N), dtype=torch.int32, device=lut.device) if want_acc else None
    _check(lib().vlut_mpgemm_token_outer(_ptr(packed), float(w_scale), _ptr(a_scale), _ptr(lut), M, 4 * G, N, _ptr(y),
                                         y.stride(0), _ptr(acc), _stream()), "vlut_mpgemm_token_outer")
    return y, acc


def query_plan_f32(M: int, K: int, N: int) -> Tuple[int, int, int, int, bool]:
    """(J, R, split_k, workgroups, one launch) of vlut_mpgemm_f32 for this shape; query_kernel names the kernel."""
    out = (ctypes.c_int * 5)()
    _check(lib().vlut_query_plan_f32(M, K, N, out), "vlut_query_plan_f32")
    return out[0], out[1], out[2], out[3], bool(out[4])


def mpgemm_f32(packed: torch.Tensor, w_scale, x: torch.Tensor, M: int, y: Optional[torch.Tensor] = None,
               want_acc: bool = False, want_scales: bool = False, workspace: Optional[torch.Tensor] = None):
    """Runs vlut_mpgemm_f32 on fp32 activations x [N][K] (row stride >= K).  w_scale: a float, or an fp32 [M]
    tensor on the GPU with one weight scale per output row.  Returns (y [N][M], acc or None, a_scale or None)."""
    if _native is not None:
        r = _native.mpgemm_f32(packed, w_scale, x, M, y, want_acc, want_scales, workspace)
        if r is not None:
            return _outputs(r, "vlut_mpgemm_f32")
    assert x.is_cuda and x.dtype == torch.float32 and x.dim() == 2 and x.stride(1) == 1
    L = _lib or lib()
    N, K = x.shape
    rows = w_scale if isinstance(w_scale, torch.Tensor) else None
    if rows is not None:
        assert rows.is_cuda and rows.dtype == torch.float32 and rows.numel() == M
    if y is None:
        y = torch.empty((N, M), dtype=torch.float32, device=x.device)
    acc = torch.empty((M, N), dtype=torch.int32, device=x.device) if want_acc else None
    scales = torch.empty(N, dtype=torch.float32, device=x.device) if want_scales else None
    _workspace(workspace)
    if workspace is None:
        ws_bytes = L.vlut_workspace_bytes_f32(M, K, N)
        if ws_bytes:
            workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=x.device)
    else:
        ws_bytes = workspace.numel() * workspace.element_size()
    rc = L.vlut_mpgemm_f32(_ptr(packed), 1.0 if rows is not None else float(w_scale), _ptr(rows), x.data_ptr(), x.stride(0),
                           M, K, N, y.data_ptr(), y.stride(0), _ptr(acc), _ptr(scales), _ptr(workspace), ws_bytes, _stream())
    if rc != VLUT_OK:
        raise VlutError(rc, "vlut_mpgemm_f32")
    return y, acc, scales


# ---- 1.60-bit packing (g = 5)
def pack_weights_g5(w_ternary: torch.Tensor) -> torch.Tensor:
    """int8 [M][K] (K % 5 == 0) on the GPU -> 1.60-bit packed blob on the GPU."""
    if _native is not None:
        r = _native.pack_weights_g5(w_ternary)
        if r is not None:
            return _outputs(r, "vlut_pack_weights_g5")[0]
    assert w_ternary.is_cuda and w_ternary.dtype == torch.int8 and w_ternary.is_contiguous()
    M, K = w_ternary.shape
    nbytes = lib().vlut_packed_weight_bytes_g5(M, K)
    if nbytes == 0:
        raise VlutError(VLUT_ERR_SHAPE, "vlut_packed_weight_bytes_g5")
    packed = torch.empty(nbytes, dtype=torch.uint8, device=w_ternary.device)
    _check(lib().vlut_pack_weights_g5(_ptr(w_ternary), M, K, _ptr(packed), nbytes, _stream()), "vlut_pack_weights_g5")
    return packed


def pack_weights_mixed(w_ternary: torch.Tensor) -> torch.Tensor:
    """int8 [M][K] (K % 4 == 0) on the GPU -> blob of the mixed 1.60-bit / 2-bit packing on the GPU."""
    if _native is not None:
        r = _native.pack_weights_mixed(w_ternary)
        if r is not None:
            return _outputs(r, "vlut_pack_weights_mixed")[0]
    assert w_ternary.is_cuda and w_ternary.dtype == torch.int8 and w_ternary.is_contiguous()
    M, K = w_ternary.shape
    nbytes = lib().vlut_packed_weight_bytes_mixed(M, K)
    if nbytes == 0:
        raise VlutError(VLUT_ERR_SHAPE, "vlut_packed_weight_bytes_mixed")
    packed = torch.empty(nbytes, dtype=torch.uint8, device=w_ternary.device)
    _check(lib().vlut_pack_weights_mixed(_ptr(w_ternary), M, K, _ptr(packed), nbytes, _stream()), "vlut_pack_weights_mixed")
    return packed


def mpgemm_mixed(packed: torch.Tensor, w_scale: float, a_q: torch.Tensor, a_scale: torch.Tensor, M: int,
                 y: Optional[torch.Tensor] = None, want_acc: bool = False):
    """Runs vlut_mpgemm_mixed on a blob from pack_weights_mixed.  Returns (y [N][M], acc or None)."""
    if _native is not None:
        r = _native.mpgemm_mixed(packed, w_scale, a_q, a_scale, M, y, None, want_acc, None)
        if r is not None:
            return _outputs(r, "vlut_mpgemm_mixed")
    K, N = a_q.shape[1], a_scale.shape[0]
    dev = a_q.device
    if y is None:
        y = torch.empty((N, M), dtype=torch.float32, device=dev)
    acc = torch.empty((M, N), dtype=torch.int32, device=dev) if want_acc else None
    ws = torch.empty(max(lib().vlut_workspace_bytes_mixed(M, K, N), 16), dtype=torch.uint8, device=dev)
    _check(lib().vlut_mpgemm_mixed(_ptr(packed), float(w_scale), _ptr(a_q), _ptr(a_scale), M, K, N, _ptr(y), y.stride(0),
                                   _ptr(acc), _ptr(ws), ws.numel(), _stream()), "vlut_mpgemm_mixed")
    return y, acc


def set_plan_g5(R: int = 0, split_k: int = 0) -> None:
    _check(lib().vlut_set_plan_g5(R, split_k), "vlut_set_plan_g5")


def query_plan_g5(M: int, K: int, N: int) -> Tuple[int, int, int]:
    out = (ctypes.c_int * 3)()
    _check(lib().vlut_query_plan_g5(M, K, N, out), "vlut_query_plan_g5")
    return out[0], out[1], out[2]


def mpgemm_g5(packed: torch.Tensor, w_scale: float, a_q: torch.Tensor, a_scale: torch.Tensor, M: int,
              y: Optional[torch.Tensor] = None, want_acc: bool = False, workspace: Optional[torch.Tensor] = None):
    """Runs vlut_mpgemm_g5.  Returns (y fp32 [N][M], acc int32 [M][N] or None)."""
    if _native is not None:
        r = _native.mpgemm_g5(packed, w_scale, a_q, a_scale, M, y, None, want_acc, workspace)
        if r is not None:
            return _outputs(r, "vlut_mpgemm_g5")
    K, N = a_q.shape[1], a_scale.shape[0]
    dev = a_q.device
    if y is None:
        y = torch.empty((N, M), dtype=torch.float32, device=dev)
    acc = torch.empty((M, N), dtype=torch.int32, device=dev) if want_acc else None
    _workspace(workspace)
    ws_bytes = lib().vlut_workspace_bytes_g5(M, K, N)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    rc = lib().vlut_mpgemm_g5(_ptr(packed), float(w_scale), _ptr(a_q), _ptr(a_scale), M, K, N, _ptr(y), y.stride(0),
                              _ptr(acc), _ptr(workspace),
                              0 if workspace is None else workspace.numel() * workspace.element_size(), _stream())
    _check(rc, "vlut_mpgemm_g5")
    return y, acc


# ---- between the projections: heads, paged cache, attention over a shared prefix
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _on_gpu(t: torch.Tensor, dim: int, what: str) -> None:
    """A tensor whose features (its last dimension) are contiguous."""
    if not t.is_cuda or t.dim() != dim or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{what}: a GPU tensor of {dim} dimensions with contiguous features is wanted")
    if t.dtype not in _TYPES:
        raise ValueError(f"{what}: fp32, bf16 or fp16 is wanted, not {t.dtype}")


def _indices(t: torch.Tensor, dtype: torch.dtype, size: int, what: str) -> None:
    if not t.is_cuda or t.dtype != dtype or t.dim() != 1 or not t.is_contiguous() or t.numel() < size:
        raise ValueError(f"{what}: a contiguous {dtype} GPU tensor of {size} values is wanted")


def _heads(t: Optional[torch.Tensor], weight: Optional[torch.Tensor] = None, what: str = "heads") -> Optional[_Heads]:
    """[N][heads][D] and the norm's weight, fp32 [D] or [heads][D]."""
    if t is None:
        return None
    _on_gpu(t, 3, what)
    if weight is not None and not (weight.is_cuda and weight.dtype == torch.float32 and tuple(weight.shape) in ((t.shape[2],), tuple(t.shape[1:]))
                                   and (weight.shape[-1] == 1 or weight.stride(-1) == 1)):
        raise ValueError(f"{what}: the norm's weight is an fp32 GPU tensor [D] or [heads][D]")
    return _Heads(t.data_ptr(), _ptr(weight), t.stride(0), t.stride(1), weight.stride(0) if weight is not None and weight.dim() == 2 else 0,
                  t.shape[1], _TYPES[t.dtype])


def _rotation(positions, cos, sin, interleaved: bool, N: int) -> Optional[_Rotation]:
    if cos is None and sin is None and positions is None:
        return None
    if cos is None or sin is None or positions is None:
        raise ValueError("the rotation takes positions, cos and sin, or none of them")
    for t, what in ((cos, "cos"), (sin, "sin")):
        if not t.is_cuda or t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous() or t.shape != cos.shape:
            raise ValueError(f"{what}: a contiguous fp32 GPU tensor [positions][features / 2] is wanted")
    _indices(positions, torch.int64, N, "positions")
    return _Rotation(cos.data_ptr(), sin.data_ptr(), positions.data_ptr(), cos.shape[0], 2 * cos.shape[1], bool(interleaved))


def _cache(k_cache: torch.Tensor, v_cache: torch.Tensor, D: int) -> _Cache:
    """[pages][heads][page_size][D] twice, in any order of the first three in memory."""
    _on_gpu(k_cache, 4, "k_cache")
    _on_gpu(v_cache, 4, "v_cache")
    if k_cache.shape != v_cache.shape or k_cache.dtype != v_cache.dtype or k_cache.shape[3] != D:
        raise ValueError("k_cache and v_cache: one shape [pages][heads][page_size][D] and one type are wanted")
    return _Cache(k_cache.data_ptr(), v_cache.data_ptr(), k_cache.shape[0], k_cache.shape[2], k_cache.stride(0), k_cache.stride(1), k_cache.stride(2),
                  v_cache.stride(0), v_cache.stride(1), v_cache.stride(2), k_cache.shape[1], _TYPES[k_cache.dtype])


def _ref(s):
    return None if s is None else ctypes.byref(s)


def norm_rope(q: torch.Tensor, k: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, cos: Optional[torch.Tensor] = None,
              sin: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
              eps: float = 1e-6, interleaved: bool = False, dtype: Optional[torch.dtype] = None, q_out: Optional[torch.Tensor] = None,
              k_out: Optional[torch.Tensor] = None):
    """Runs vlut_norm_rope: the RMS norm of every head of q [N][heads][D] and k (where a weight is given: fp32 [D] or [heads][D]), then the
    rotation by the tokens' int64 `positions` with the tables cos and sin, fp32 [rows][features / 2] (where they are given), in one pass.
    The tensors may be views of a stacked projection's rows.  Returns (q_out, k_out or None) of type `dtype` (default: q's); an output may
    be the input."""
    if _native is not None:
        r = _native.norm_rope(q, k, positions, cos, sin, q_weight, k_weight, eps, interleaved, dtype, q_out, k_out)
        if r is not None:
            return _outputs(r, "vlut_norm_rope")
    _on_gpu(q, 3, "q")
    N, _, D = q.shape
    if dtype is None:
        dtype = q.dtype if q_out is None else q_out.dtype
    if k is not None and (k.dim() != 3 or k.shape[0] != N or k.shape[2] != D):
        raise ValueError("k: [N][heads][D] of q's tokens and features is wanted")
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
    if k is not None and k_out is None:
        k_out = torch.empty(k.shape, dtype=dtype, device=q.device)
    for out, x, what in ((q_out, q, "q_out"), (k_out, k, "k_out")):
        if (out is None) != (x is None) or (out is not None and out.shape != x.shape):
            raise ValueError(f"{what}: a tensor of the input's shape is wanted")
    _check(lib().vlut_norm_rope(_ref(_heads(q, q_weight, "q")), _ref(_heads(k, k_weight, "k")), eps, _ref(_rotation(positions, cos, sin, interleaved, N)),
                                N, D, _ref(_heads(q_out, what="q_out")), _ref(_heads(k_out, what="k_out")), _stream()), "vlut_norm_rope")
    return q_out, k_out


def append_kv(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
              positions: Optional[torch.Tensor] = None, cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None,
              k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False, q: Optional[torch.Tensor] = None,
              q_weight: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None):
    """Runs vlut_append_kv: keys (normed and rotated as in `norm_rope`) and values, [N][heads][D], to the int64 `slots` (page * page_size +
    token in the page; negative: left out) of the caches [pages][heads][page_size][D] (bf16 or fp16).  With q the queries are normed and
    rotated in the same launch: returns q_out, of the cache's type (None without q)."""
    if _native is not None:
        r = _native.append_kv(k, v, slots, k_cache, v_cache, positions, cos, sin, k_weight, eps, interleaved, q, q_weight, q_out)
        if r is not None:
            return _outputs(r, "vlut_append_kv")[0]
    _on_gpu(k, 3, "k")
    N, _, D = k.shape
    if tuple(v.shape) != tuple(k.shape) or (q is not None and (q.dim() != 3 or q.shape[0] != N or q.shape[2] != D)):
        raise ValueError("q, k and v: [N][heads][D] of the same tokens and features are wanted")
    _indices(slots, torch.int64, N, "slots")
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=k_cache.dtype, device=q.device)
    if (q is None) != (q_out is None) or (q is not None and q_out.shape != q.shape):
        raise ValueError("q_out: a tensor of q's shape is wanted")
    _check(lib().vlut_append_kv(_ref(_heads(k, k_weight, "k")), _ref(_heads(v, what="v")), _ref(_heads(q, q_weight, "q")), eps,
                                _ref(_rotation(positions, cos, sin, interleaved, N)), slots.data_ptr(), N, D, _ref(_cache(k_cache, v_cache, D)),
                                _ref(_heads(q_out, what="q_out")), _stream()), "vlut_append_kv")
    return q_out


def shared_prefix_attention_bytes(B: int, n: int, q_heads: int, k_heads: int, D: int, prefix_len: int, max_own_len: int) -> int:
    return lib().vlut_shared_prefix_attention_bytes(B, n, q_heads, k_heads, D, prefix_len, max_own_len)


def query_shared_prefix_attention(B: int, n: int, q_heads: int, k_heads: int, D: int, prefix_len: int, max_own_len: int) -> Tuple[int, int, int, int]:
    """(query rows per workgroup, parts of the prefix, parts of an own sequence, workgroups) of such a call."""
    out = (ctypes.c_int * 4)()
    _check(lib().vlut_query_shared_prefix_attention(B, n, q_heads, k_heads, D, prefix_len, max_own_len, out), "vlut_query_shared_prefix_attention")
    return out[0], out[1], out[2], out[3]


def shared_prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, prefix_pages: Optional[torch.Tensor], prefix_len: int,
                            page_table: Optional[torch.Tensor], own_lens: torch.Tensor, query_lens: Optional[torch.Tensor] = None,
                            max_own_len: Optional[int] = None, scale: Optional[float] = None, dtype: Optional[torch.dtype] = None,
                            out: Optional[torch.Tensor] = None, want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """Runs vlut_shared_prefix_attention: q [B][n][heads][D] (the cache's type) over the first `prefix_len` tokens of `prefix_pages` (int32), which
    all sequences share, and over each sequence's own `own_lens[b]` tokens (int32 [B]) in the pages of its row of `page_table` (int32
    [B][pages]); its last `query_lens[b]` (default n) own tokens are the queries', each of which sees up to itself.
    max_own_len: an upper bound of own_lens (default: what the table's rows hold).  scale: default D ** -0.5.  dtype: fp32 or the
    cache's (default).  Returns (out [B][n][heads][D], lse fp32 [B][n][heads] or None)."""
    if _native is not None:
        r = _native.shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, own_lens, query_lens, max_own_len, scale, dtype,
                                            out, want_lse, workspace)
        if r is not None:
            return _outputs(r, "vlut_shared_prefix_attention")
    _on_gpu(q, 4, "q")
    B, n, Hq, D = q.shape
    cache = _cache(k_cache, v_cache, D)
    page_size, Hk = k_cache.shape[2], k_cache.shape[1]
    table_stride = 0
    if page_table is not None:
        if not page_table.is_cuda or page_table.dtype != torch.int32 or page_table.dim() != 2 or page_table.shape[0] != B or (
                page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table: an int32 GPU tensor [B][pages] is wanted")
        table_stride = page_table.stride(0)
    room = 0 if page_table is None else page_table.shape[1] * page_size
    if max_own_len is None:
        max_own_len = room
    if max_own_len > room:
        raise ValueError("max_own_len: more tokens than the rows of page_table hold")
    if prefix_len > 0:
        if prefix_pages is None:
            raise ValueError("prefix_pages: the pages of the prefix are wanted")
        _indices(prefix_pages, torch.int32, -(-prefix_len // page_size), "prefix_pages")
    _indices(own_lens, torch.int32, B, "own_lens")
    if query_lens is not None:
        _indices(query_lens, torch.int32, B, "query_lens")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype if dtype is None else dtype, device=q.device)
    _on_gpu(out, 4, "out")
    if out.shape != q.shape:
        raise ValueError("out: a tensor of q's shape is wanted")
    lse = torch.empty((B, n, Hq), dtype=torch.float32, device=q.device) if want_lse else None
    _workspace(workspace)
    if workspace is None:
        nbytes = shared_prefix_attention_bytes(B, n, Hq, Hk, D, prefix_len, max_own_len)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    rows = [_Heads(t.data_ptr(), None, t.stride(1), t.stride(2), 0, Hq, _TYPES[t.dtype]) for t in (q, out)]
    _check(lib().vlut_shared_prefix_attention(
        ctypes.byref(rows[0]), q.stride(0), ctypes.byref(cache), _ptr(prefix_pages), prefix_len, _ptr(page_table), table_stride, own_lens.data_ptr(),
        max_own_len, _ptr(query_lens), B, n, D, D ** -0.5 if scale is None else scale, ctypes.byref(rows[1]), out.stride(0), _ptr(lse),
        _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()), "vlut_shared_prefix_attention")
    return out, lse


# ---- chunks of new tokens over a paged cache
def _here(*tensors: Optional[torch.Tensor]) -> None:
    """The tensors are on the current device, whose current stream the call is given."""
    for t in tensors:
        if t is not None and t.is_cuda and t.device.index != torch.cuda.current_device():
            raise ValueError(f"a tensor on {t.device}: the current device is wanted")


def chunk_attention_bytes(N: int, B: int, q_heads: int, k_heads: int, D: int, max_queries: int, max_len: int, window: int = 0) -> int:
    return lib().vlut_chunk_attention_bytes(N, B, q_heads, k_heads, D, max_queries, max_len, window)


def query_chunk_attention(N: int, B: int, q_heads: int, k_heads: int, D: int, max_queries: int, max_len: int, window: int = 0) -> Tuple[int, int, int, int, int, int]:
    """(rows of a key head up to which a sequence is worked on as one of few, parts of its keys at most, keys of a part; rows of a tile of the others, parts,
    keys) of such a call."""
    out = (ctypes.c_int * 6)()
    _check(lib().vlut_query_chunk_attention(N, B, q_heads, k_heads, D, max_queries, max_len, window, out), "vlut_query_chunk_attention")
    return tuple(out)


def chunk_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, page_table: torch.Tensor, query_starts: torch.Tensor, lens: torch.Tensor,
                    max_queries: Optional[int] = None, max_len: Optional[int] = None, window: int = 0, scale: Optional[float] = None,
                    dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, want_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """Runs vlut_chunk_attention: q [N][heads][D] (the cache's type) holds the new tokens of B sequences one behind the other, sequence b's from row
    query_starts[b] to query_starts[b + 1] (int32 [B + 1]); they are the last of its lens[b] tokens (int32 [B]), whose keys and values the pages of
    its row of `page_table` (int32 [B][pages]) hold.  Each sees the tokens up to itself, the last `window` of them where that is not 0.
    max_queries, max_len: upper bounds, which size the launches (default: N, and what the table's rows hold).  scale: default D ** -0.5.  dtype: fp32 or the cache's
    (default).  Returns (out [N][heads][D], lse fp32 [N][heads] or None); rows of no sequence are left as they are."""
    if _native is not None:
        r = _native.chunk_attention(q, k_cache, v_cache, page_table, query_starts, lens, max_queries, max_len, window, scale, dtype, out, want_lse, workspace)
        if r is not None:
            return _outputs(r, "vlut_chunk_attention")
    _on_gpu(q, 3, "q")
    N, Hq, D = q.shape
    cache = _cache(k_cache, v_cache, D)
    page_size, Hk = k_cache.shape[2], k_cache.shape[1]
    if not page_table.is_cuda or page_table.dtype != torch.int32 or page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table: an int32 GPU tensor [B][pages] is wanted")
    B, room = page_table.shape[0], page_table.shape[1] * page_size
    if not (query_starts.is_cuda and query_starts.dtype == torch.int32 and query_starts.is_contiguous() and tuple(query_starts.shape) == (B + 1,)):
        raise ValueError(f"query_starts: a contiguous int32 GPU tensor [{B + 1}] is wanted")
    _indices(lens, torch.int32, B, "lens")
    max_len = room if max_len is None else max_len
    max_queries = N if max_queries is None else max_queries
    if max_len > room:
        raise ValueError("max_len: more tokens than the rows of page_table hold")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype if dtype is None else dtype, device=q.device)
    _on_gpu(out, 3, "out")
    if out.shape != q.shape:
        raise ValueError("out: a tensor of q's shape is wanted")
    _here(q, k_cache, v_cache, page_table, query_starts, lens, out, workspace)
    lse = torch.empty((N, Hq), dtype=torch.float32, device=q.device) if want_lse else None
    _workspace(workspace)
    if workspace is None:
        nbytes = chunk_attention_bytes(N, B, Hq, Hk, D, max_queries, max_len, window)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    _check(lib().vlut_chunk_attention(_ref(_heads(q, what="q")), _ref(cache), _ptr(page_table), page_table.stride(0), query_starts.data_ptr(), lens.data_ptr(), N, B, D,
                                      max_queries, max_len, window, D ** -0.5 if scale is None else scale, _ref(_heads(out, what="out")), _ptr(lse), _ptr(workspace),
                                      0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()), "vlut_chunk_attention")
    return out, lse


# ---- around a block: norms, gate, residual; behind the last product: log probabilities
_ACTIVATIONS = {None: 0, "none": 0, "sigmoid": 1, "silu": 2, "relu2": 3, "gelu": 4}


def _rows(t: Optional[torch.Tensor], shape, what: str) -> Optional[_Rows]:
    """[N][K], features contiguous."""
    if t is None:
        return None
    _on_gpu(t, 2, what)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: a tensor of {tuple(shape)} is wanted, not {tuple(t.shape)}")
    return _Rows(t.data_ptr(), t.stride(0), _TYPES[t.dtype])


def _weight(t: Optional[torch.Tensor], K: int, what: str) -> Optional[torch.Tensor]:
    if t is not None and not (t.is_cuda and t.dtype == torch.float32 and tuple(t.shape) == (K,) and t.is_contiguous()):
        raise ValueError(f"{what}: a contiguous fp32 GPU tensor [{K}] is wanted")
    return t


def _gate(gate: Optional[torch.Tensor], y: torch.Tensor) -> Optional[torch.Tensor]:
    """One for all tokens as rows that lie on each other."""
    return gate.expand(y.shape) if gate is not None and gate.dim() == 1 and y.dim() == 2 and gate.shape[0] == y.shape[1] else gate


def _activation(name: Optional[str]) -> int:
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation: one of {sorted(k for k in _ACTIVATIONS if k)} is wanted, not {name!r}")
    return _ACTIVATIONS[name]


def residual_norm(y: torch.Tensor, residual: torch.Tensor, weight: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                  activation: Optional[str] = None, scale: float = 1.0, next_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, next_out: Optional[torch.Tensor] = None):
    """Runs vlut_residual_norm behind a block with output y [N][K]: h = residual + scale * act(gate) * norm(y), and the next block's input
    x = norm(h) where `next_weight` is given, in one pass.  weight, next_weight: fp32 [K] of RMS norms (weight None: no norm after the block).  gate: [N][K], or
    [K] for all tokens, of y's type or fp32; activation: None, "sigmoid", "silu", "relu2" or "gelu" of it.  Returns (h of the residual's type, x or
    None of type `dtype`, default y's); `out` and `next_out` may be an input itself (the residual, say)."""
    if _native is not None:
        r = _native.residual_norm(y, residual, weight, gate, activation, scale, next_weight, eps, dtype, out, next_out)
        if r is not None:
            return _outputs(r, "vlut_residual_norm")
    _on_gpu(y, 2, "y")
    N, K = y.shape
    code, gate = _activation(activation), _gate(gate, y)
    if residual.dtype not in _TYPES or (next_out is not None and next_weight is None):
        raise ValueError("next_out: a next_weight is wanted" if residual.dtype in _TYPES else f"residual: fp32, bf16 or fp16 is wanted, not {residual.dtype}")
    if out is None:
        out = torch.empty((N, K), dtype=residual.dtype, device=y.device)
    if next_out is None and next_weight is not None:
        next_out = torch.empty((N, K), dtype=y.dtype if dtype is None else dtype, device=y.device)
    _here(y, residual, weight, gate, next_weight, out, next_out)
    rows = [_rows(t, (N, K), what) for t, what in ((y, "y"), (gate, "gate"), (residual, "residual"), (out, "out"), (next_out, "next_out"))]
    _check(lib().vlut_residual_norm(_ref(rows[0]), _ptr(_weight(weight, K, "weight")), _ref(rows[1]), code, scale, _ref(rows[2]),
                                    _ptr(_weight(next_weight, K, "next_weight")), eps, N, K, _ref(rows[3]), _ref(rows[4]), _stream()), "vlut_residual_norm")
    return out, next_out


def gated_norm(x: torch.Tensor, gate: Optional[torch.Tensor] = None, activation: Optional[str] = "silu", weight: Optional[torch.Tensor] = None,
               eps: float = 1e-6, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Runs vlut_gated_norm inside a block: act(gate) * x (act(x) without a gate), x [N][K], and its RMS norm where `weight` (fp32 [K]) is given.  x and gate may be
    views of a stacked gate|up projection's rows.  Returns out of type `dtype` (default: x's)."""
    if _native is not None:
        r = _native.gated_norm(x, gate, activation, weight, eps, dtype, out)
        if r is not None:
            return _outputs(r, "vlut_gated_norm")[0]
    _on_gpu(x, 2, "x")
    N, K = x.shape
    code, gate = _activation(activation), _gate(gate, x)
    if out is None:
        out = torch.empty((N, K), dtype=x.dtype if dtype is None else dtype, device=x.device)
    _here(x, gate, weight, out)
    rows = [_rows(t, (N, K), what) for t, what in ((x, "x"), (gate, "gate"), (out, "out"))]
    _check(lib().vlut_gated_norm(_ref(rows[0]), _ref(rows[1]), code, _ptr(_weight(weight, K, "weight")), eps, N, K, _ref(rows[2]), _stream()), "vlut_gated_norm")
    return out


def token_logprobs_bytes(N: int, V: int, top: int = 0) -> int:
    return lib().vlut_token_logprobs_bytes(N, V, top)


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0, temperature: float = 1.0, want_entropy: bool = True,
                   workspace: Optional[torch.Tensor] = None):
    """Runs vlut_token_logprobs on logits [N][V] (fp32, bf16 or fp16; -inf: not allowed): (log probabilities of the int64 `tokens` [N] or None, entropies or
    None, int64 ids [N][top] of the largest logits or None, their log probabilities or None); fp32, of softmax(logits / temperature)."""
    if _native is not None:
        r = _native.token_logprobs(logits, tokens, top, temperature, want_entropy, workspace)
        if r is not None:
            return _outputs(r, "vlut_token_logprobs")
    _on_gpu(logits, 2, "logits")
    N, V = logits.shape
    if tokens is not None:
        _indices(tokens, torch.int64, N, "tokens")
    new = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device=logits.device)  # noqa: E731
    _here(logits, tokens, workspace)
    logprob = None if tokens is None else new(torch.float32, N)
    entropy = new(torch.float32, N) if want_entropy else None
    ids, logprobs = (new(torch.int64, N, top), new(torch.float32, N, top)) if top > 0 else (None, None)
    _workspace(workspace)
    if workspace is None:
        nbytes = token_logprobs_bytes(N, V, top)
        if nbytes:
            workspace = new(torch.uint8, nbytes)
    _check(lib().vlut_token_logprobs(_ref(_rows(logits, (N, V), "logits")), _ptr(tokens), temperature, top, N, V, _ptr(logprob), _ptr(entropy), _ptr(ids),
                                     _ptr(logprobs), _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()),
           "vlut_token_logprobs")
    return logprob, entropy, ids, logprobs
