"""Thin ctypes binding of libqadc.so: argument marshalling only.

Every function has the name of the C entry point it calls (include/qadc.h) and
takes torch tensors that live on the GPU; torch is used for device memory and
for the current HIP stream, nothing else.  There is no fallback: if the HIP
library is missing or a call fails, an exception is raised.
"""

from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "libqadc.so")

QADC_OK, QADC_EINVAL, QADC_ENOMEM, QADC_EHIP = 0, -1, -2, -3
QADC_MAX_R = 1024
QADC_MAX_INIT = 8192
QADC_QMIN_PER_TABLE, QADC_QMIN_GLOBAL = 0, 1
QADC_U8_4BIT, QADC_F32_4BIT, QADC_F32_8BIT, QADC_U8_8BIT, QADC_U8_6BIT = 0, 1, 2, 3, 4
QADC_WS_SCAN_TOPK, QADC_WS_SCAN_F32_4BIT, QADC_WS_SCAN_F32_8BIT, QADC_WS_SEARCH, QADC_WS_SCAN_U8_8BIT = 0, 1, 2, 3, 4
QADC_WS_SCAN_U8_6BIT = 5
(QADC_PROF_SCAN, QADC_PROF_MERGE, QADC_PROF_SEED, QADC_PROF_IVF_INDEX, QADC_PROF_IVF_TABLES,
 QADC_PROF_TABLES, QADC_PROF_QUANTIZE, QADC_PROF_PREPARE, QADC_PROF_ROTATE, QADC_PROF_IVF_SHARED,
 QADC_PROF_NORM, QADC_PROF_LINEAR4, QADC_PROF_LOGPROBS, QADC_PROF_MIX,
 QADC_PROF_RMS, QADC_PROF_ADJUST, QADC_PROF_DISTILL, QADC_PROF_ADAPTERS) = range(18)
QADC_LAYOUT_STANDARD, QADC_LAYOUT_TRANSPOSED = 0, 1
QADC_TYPE_F32, QADC_TYPE_F16, QADC_TYPE_BF16, QADC_TYPE_E4M3 = 0, 1, 2, 3
QADC_MAX_ALTERNATIVES = 128
QADC_MAX_HISTORY = 1 << 24
QADC_MAX_RANK = 128

EXPORTS = (
    "qadc_layer_norm", "qadc_layer_norm_backward", "qadc_layer_norm_workspace_bytes",
    "qadc_rms_norm", "qadc_rms_norm_backward", "qadc_rms_norm_workspace_bytes",
    "qadc_weights4_bytes", "qadc_pack_weights4", "qadc_linear4",
    "qadc_token_logprobs", "qadc_token_logprobs_workspace_bytes", "qadc_token_logprobs_backward", "qadc_neighbour_mix",
    "qadc_add_adapters", "qadc_adapters_workspace_bytes",
    "qadc_adjust_logits", "qadc_distill", "qadc_distill_workspace_bytes", "qadc_distill_backward", "qadc_distill_step",
    "qadc_build_luts", "qadc_quantize_luts", "qadc_quantize_luts_8bit", "qadc_quantize_luts_6bit", "qadc_scan_topk", "qadc_search", "qadc_ivf_search",
    "qadc_ivf_workspace_bytes", "qadc_pq_encode", "qadc_pq_train", "qadc_rotate",
    "qadc_profile_enable", "qadc_profile_only", "qadc_profile_read", "qadc_workspace_bytes", "qadc_workspace_init",
    "qadc_last_error", "qadc_version", "qadc_packed_bytes", "qadc_pack_codes", "qadc_unpack_codes",
    "qadc_ivf_assign", "qadc_ivf_group_workspace_bytes", "qadc_ivf_group", "qadc_ivf_encode",
    "qadc_multi_index_cells", "qadc_multi_index_assign", "qadc_multi_index_workspace_bytes",
    "qadc_multi_index_probes", "qadc_multi_index_group_workspace_bytes", "qadc_multi_index_group",
    "qadc_multi_index_encode", "qadc_multi_index_slots", "qadc_search_static", "qadc_static_scratch_bytes",
)

_lib = None


class qadc_ivf_index(ctypes.Structure):
    """Mirror of the C struct: device pointers + shapes (include/qadc.h)."""
    _fields_ = [("coarse", ctypes.c_void_p), ("list_off", ctypes.c_void_p), ("codes", ctypes.c_void_p),
                ("ids", ctypes.c_void_p), ("codebooks", ctypes.c_void_p), ("d", ctypes.c_int),
                ("m", ctypes.c_int), ("K", ctypes.c_int), ("n", ctypes.c_int64),
                ("halves", ctypes.c_void_p), ("cell_ids", ctypes.c_void_p), ("Kh", ctypes.c_int)]


class qadc_weights4(ctypes.Structure):
    """Mirror of the C struct (include/qadc.h); `tensor` keeps the packed weights alive."""
    _fields_ = [("packed", ctypes.c_void_p), ("N", ctypes.c_int64), ("K", ctypes.c_int), ("group", ctypes.c_int),
                ("stype", ctypes.c_int), ("has_zeros", ctypes.c_int)]


class qadc_adapters(ctypes.Structure):
    """Mirror of the C struct (include/qadc.h), made of a pool: a [count][rank][K] and b [count][N][rank] (f32, f16 or bf16), scales
    f32 [count] | None, ranks i32 [count] | None; `tensors` keeps them alive."""
    _fields_ = [("a", ctypes.c_void_p), ("b", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("ranks", ctypes.c_void_p),
                ("N", ctypes.c_int64), ("K", ctypes.c_int), ("rank", ctypes.c_int), ("count", ctypes.c_int), ("type", ctypes.c_int)]

    def __init__(self, a, b, scales=None, ranks=None):
        if a.dim() != 3 or b.dim() != 3 or (b.shape[0], b.shape[2]) != (a.shape[0], a.shape[1]):
            raise ValueError("expected a [count][rank][K] and b [count][N][rank]")
        count, rank, K = a.shape
        device = a.get_device()
        super().__init__(_ptr(a), _ptr(b, a.dtype, device), _vector(scales, count, torch.float32, device),
                         _vector(ranks, count, torch.int32, device), b.shape[1], K, rank, count, _type(a))
        self.dtype, self.device, self.tensors = a.dtype, device, (a, b, scales, ranks)


class QadcError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"qadc error {code}: {msg}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Loads libqadc.so (built in-tree by paper_1704_07355_amd/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_SO):
            raise ImportError(f"{_SO} not found: run `python -m paper_1704_07355_amd.build` first")
        L = ctypes.CDLL(_SO)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        L.qadc_build_luts.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp, vp]
        L.qadc_build_luts.restype = i32
        L.qadc_quantize_luts.argtypes = [vp, i32, i32, i32, vp, i64, vp, i32, i32, i32,
                                         vp, vp, vp, vp, vp]
        L.qadc_quantize_luts.restype = i32
        L.qadc_quantize_luts_8bit.argtypes = L.qadc_quantize_luts.argtypes
        L.qadc_quantize_luts_8bit.restype = i32
        L.qadc_quantize_luts_6bit.argtypes = L.qadc_quantize_luts.argtypes
        L.qadc_quantize_luts_6bit.restype = i32
        L.qadc_scan_topk.argtypes = [i32, vp, i64, i32, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        L.qadc_scan_topk.restype = i32
        L.qadc_search.argtypes = [vp, i32, i32, vp, i32, vp, i64, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        L.qadc_search.restype = i32
        L.qadc_search_static.argtypes = [vp, i32, i32, vp, i32, vp, i64, i32, i32, i32, i32, vp, vp, vp, vp]
        L.qadc_search_static.restype = i32
        L.qadc_static_scratch_bytes.argtypes = []
        L.qadc_static_scratch_bytes.restype = sz
        L.qadc_ivf_search.argtypes = [ctypes.POINTER(qadc_ivf_index), vp, i32, i32, i32, i32, i32, i32,
                                      vp, vp, vp, vp, vp, vp, sz, vp]
        L.qadc_ivf_search.restype = i32
        L.qadc_ivf_workspace_bytes.argtypes = [ctypes.POINTER(qadc_ivf_index), i32, i32, i32]
        L.qadc_ivf_workspace_bytes.restype = sz
        L.qadc_pq_encode.argtypes = [vp, i32, i32, i32, vp, i64, vp, vp]
        L.qadc_pq_encode.restype = i32
        L.qadc_rotate.argtypes = [vp, i32, vp, i64, vp, vp]
        L.qadc_rotate.restype = i32
        L.qadc_pq_train.argtypes = [vp, i64, i32, i32, i32, vp, i32, vp, vp, sz, vp]
        L.qadc_pq_train.restype = i32
        L.qadc_profile_only.argtypes = [i32]
        L.qadc_profile_only.restype = i32
        L.qadc_profile_enable.argtypes = [i32]
        L.qadc_profile_enable.restype = i32
        L.qadc_profile_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
        L.qadc_profile_read.restype = i32
        L.qadc_workspace_bytes.argtypes = [i32, i64, i32, i32, i32]
        L.qadc_workspace_bytes.restype = sz
        L.qadc_workspace_init.argtypes = [vp, sz, vp]
        L.qadc_workspace_init.restype = i32
        L.qadc_packed_bytes.argtypes = [i64, i32, i32]
        L.qadc_packed_bytes.restype = sz
        L.qadc_pack_codes.argtypes = [vp, i64, i32, i32, vp, vp]
        L.qadc_pack_codes.restype = i32
        L.qadc_unpack_codes.argtypes = [vp, i64, i32, i32, vp, vp]
        L.qadc_unpack_codes.restype = i32
        L.qadc_ivf_assign.argtypes = [vp, i32, i32, vp, i64, vp, vp]
        L.qadc_ivf_assign.restype = i32
        L.qadc_ivf_group_workspace_bytes.argtypes = [i64, i32]
        L.qadc_ivf_group_workspace_bytes.restype = sz
        L.qadc_ivf_group.argtypes = [vp, i64, i32, vp, vp, vp, sz, vp]
        L.qadc_ivf_group.restype = i32
        L.qadc_ivf_encode.argtypes = [vp, i32, vp, i32, i32, vp, i64, vp, vp, i64, vp, vp]
        L.qadc_ivf_encode.restype = i32
        L.qadc_multi_index_cells.argtypes = [vp, i32, i32, vp, vp]
        L.qadc_multi_index_cells.restype = i32
        L.qadc_multi_index_assign.argtypes = [vp, i32, i32, vp, i64, vp, vp]
        L.qadc_multi_index_assign.restype = i32
        L.qadc_multi_index_workspace_bytes.argtypes = [i32, i32, i32]
        L.qadc_multi_index_workspace_bytes.restype = sz
        L.qadc_multi_index_probes.argtypes = [vp, i32, i32, vp, i32, i32, vp, vp, sz, vp]
        L.qadc_multi_index_probes.restype = i32
        L.qadc_multi_index_group_workspace_bytes.argtypes = [i64, i32]
        L.qadc_multi_index_group_workspace_bytes.restype = sz
        L.qadc_multi_index_group.argtypes = [vp, i64, i32, i64, vp, vp, vp, vp, vp, sz, vp]
        L.qadc_multi_index_group.restype = i32
        L.qadc_multi_index_encode.argtypes = [vp, i32, vp, i32, i32, vp, i64, vp, vp, i64, vp, vp]
        L.qadc_multi_index_encode.restype = i32
        L.qadc_multi_index_slots.argtypes = [vp, i64, vp, i64, vp, vp]
        L.qadc_multi_index_slots.restype = i32
        f32 = ctypes.c_float
        L.qadc_layer_norm.argtypes = [vp, i64, i32, vp, vp, i32, i64, i32, f32, vp, vp, vp, vp]
        L.qadc_layer_norm.restype = i32
        L.qadc_layer_norm_backward.argtypes = [vp, i64, vp, i64, i32, vp, i32, vp, vp, i64, i32, vp, vp, vp, vp, sz, vp]
        L.qadc_layer_norm_backward.restype = i32
        L.qadc_layer_norm_workspace_bytes.argtypes = [i64, i32]
        L.qadc_layer_norm_workspace_bytes.restype = sz
        L.qadc_rms_norm.argtypes = [vp, i64, vp, i64, i32, vp, i32, i64, i32, f32, vp, i64, vp, i32, vp, vp, vp]
        L.qadc_rms_norm.restype = i32
        L.qadc_rms_norm_backward.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, i32, vp, i64, i32, vp, vp, vp, sz, vp]
        L.qadc_rms_norm_backward.restype = i32
        L.qadc_rms_norm_workspace_bytes.argtypes = [i64, i32]
        L.qadc_rms_norm_workspace_bytes.restype = sz
        L.qadc_weights4_bytes.argtypes = [i64, i32, i32, i32]
        L.qadc_weights4_bytes.restype = sz
        L.qadc_pack_weights4.argtypes = [vp, vp, i32, vp, i64, i32, i32, vp, vp]
        L.qadc_pack_weights4.restype = i32
        L.qadc_linear4.argtypes = [ctypes.POINTER(qadc_weights4), vp, i64, i32, i64, vp, vp, i64, vp]
        L.qadc_linear4.restype = i32
        L.qadc_token_logprobs.argtypes = [vp, i64, i32, i64, i32, f32, vp, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.qadc_token_logprobs.restype = i32
        L.qadc_token_logprobs_workspace_bytes.argtypes = [i64, i32, i32]
        L.qadc_token_logprobs_workspace_bytes.restype = sz
        L.qadc_token_logprobs_backward.argtypes = [vp, i64, i32, i64, i32, f32, vp, i32, vp, vp, vp, vp, vp, i64, vp]
        L.qadc_token_logprobs_backward.restype = i32
        L.qadc_neighbour_mix.argtypes = [vp, vp, i32, vp, i64, i32, vp, i64, f32, vp, i32, vp, f32, vp, vp, vp]
        L.qadc_neighbour_mix.restype = i32
        L.qadc_adjust_logits.argtypes = [vp, i64, i32, i64, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp, i32, vp, i64, i32, vp, vp, i64, vp]
        L.qadc_adjust_logits.restype = i32
        L.qadc_distill.argtypes = [vp, i64, i32, i64, i32, f32, vp, vp, i32, i32, vp, vp, vp, vp, sz, vp]
        L.qadc_distill.restype = i32
        L.qadc_distill_workspace_bytes.argtypes = [i64, i32]
        L.qadc_distill_workspace_bytes.restype = sz
        L.qadc_distill_backward.argtypes = [vp, i64, i32, i64, i32, f32, vp, vp, i32, i32, vp, vp, vp, vp, i64, vp]
        L.qadc_distill_backward.restype = i32
        L.qadc_distill_step.argtypes = [vp, i64, i32, i64, i32, f32, vp, vp, i32, i32, vp, vp, vp, i64, vp, sz, vp]
        L.qadc_distill_step.restype = i32
        L.qadc_add_adapters.argtypes = [ctypes.POINTER(qadc_adapters), vp, vp, i64, i64, vp, i64, vp, i64, vp, sz, vp]
        L.qadc_add_adapters.restype = i32
        L.qadc_adapters_workspace_bytes.argtypes = [ctypes.POINTER(qadc_adapters), i64]
        L.qadc_adapters_workspace_bytes.restype = sz
        L.qadc_last_error.restype = ctypes.c_char_p
        L.qadc_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


# `device`, of the helpers that look at a tensor: the GPU that it has to be on, in calls that say so (its number costs what is_cuda
# does).
def _refusal(t, device, what):
    if device is not None and t.is_cuda and t.get_device() != device:
        what = f"tensors of one call on cuda:{device} and cuda:{t.get_device()}"
    return ValueError(what)


def _ptr(t, dtype=None, device=None):
    if t is None:
        return None
    if not (t.is_cuda if device is None else t.get_device() == device) or not t.is_contiguous():
        raise _refusal(t, device, "tensor must be a contiguous GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


# The current device's current stream as a raw handle, where torch gives it: the Stream object costs 2.7 us a call.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _stream_on(device):
    """The current stream, for a call on tensors of GPU number `device`, which has to be the current one."""
    current = torch.cuda.current_device()
    if device != current:
        raise ValueError(f"tensors on cuda:{device}, the current device is cuda:{current}")
    if _raw_stream is not None:
        return _raw_stream(device)
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(rc: int):
    if rc != QADC_OK:
        raise QadcError(rc, lib().qadc_last_error().decode())


def qadc_version() -> str:
    return lib().qadc_version().decode()


def qadc_last_error() -> str:
    return lib().qadc_last_error().decode()


def qadc_workspace_bytes(call: int, n: int, m: int, nq: int, R: int) -> int:
    return int(lib().qadc_workspace_bytes(call, n, m, nq, R))


def qadc_workspace_init(workspace):
    """Clears a workspace tensor before its first use; returns it."""
    _check(lib().qadc_workspace_init(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream()))
    return workspace


def qadc_build_luts(codebooks, queries, base=None, out=None):
    """codebooks f32 [m][ksub][dsub], queries f32 [nq][d], base f32 [nq][d] | None -> f32 [nq][m][ksub]."""
    m, ksub, dsub = codebooks.shape
    nq, d = queries.shape
    if out is None:
        out = torch.empty((nq, m, ksub), dtype=torch.float32, device=queries.device)
    _check(lib().qadc_build_luts(_ptr(codebooks, torch.float32), d, m, ksub,
                                 _ptr(queries, torch.float32), _ptr(base, torch.float32), nq,
                                 _ptr(out, torch.float32), _stream()))
    return out


def qadc_quantize_luts(luts, init_codes, R, nbins=255, qmin_mode=QADC_QMIN_PER_TABLE, qmax_in=None):
    """luts f32 [nq][m][k] or [nq][ngroup][m][k], k = 16 (init_codes u8 [n_init][m/2] | None) or
    k = 256 (8-bit components, init_codes u8 [n_init][m] | None: qadc_quantize_luts_8bit) or k = 64
    (6-bit components, init_codes u8 [n_init][3m/4] | None: qadc_quantize_luts_6bit).

    Returns (qluts u8 like luts, bias f32 [nq][m], delta f32 [nq], qmax f32 [nq]).
    """
    if luts.dim() == 3:
        nq, m, k = luts.shape
        ngroup = 1
    else:
        nq, ngroup, m, k = luts.shape
    if k not in (16, 64, 256):
        raise ValueError("tables of 16, 64 or 256 entries expected")
    fn = {16: lib().qadc_quantize_luts, 64: lib().qadc_quantize_luts_6bit, 256: lib().qadc_quantize_luts_8bit}[k]
    dev = luts.device
    qluts = torch.empty(luts.shape, dtype=torch.uint8, device=dev)
    bias = torch.empty((nq, m), dtype=torch.float32, device=dev)
    delta = torch.empty((nq,), dtype=torch.float32, device=dev)
    qmax = torch.empty((nq,), dtype=torch.float32, device=dev)
    n_init = 0 if init_codes is None else init_codes.shape[0]
    _check(fn(_ptr(luts, torch.float32), nq, ngroup, m, _ptr(init_codes, torch.uint8), n_init,
              _ptr(qmax_in, torch.float32), R, nbins, qmin_mode,
              _ptr(qluts), _ptr(bias), _ptr(delta), _ptr(qmax), _stream()))
    return qluts, bias, delta, qmax


def qadc_quantize_luts_8bit(luts, init_codes, R, nbins=255, qmin_mode=QADC_QMIN_PER_TABLE, qmax_in=None):
    """qadc_quantize_luts for 256-entry tables: luts f32 [nq][m][256] or [nq][ngroup][m][256], init_codes
    u8 [n_init][m] | None."""
    if luts.shape[-1] != 256:
        raise ValueError("tables of 256 entries expected")
    return qadc_quantize_luts(luts, init_codes, R, nbins, qmin_mode, qmax_in)


def qadc_quantize_luts_6bit(luts, init_codes, R, nbins=255, qmin_mode=QADC_QMIN_PER_TABLE, qmax_in=None):
    """qadc_quantize_luts for 64-entry tables: luts f32 [nq][m][64] or [nq][ngroup][m][64], init_codes
    u8 [n_init][3m/4] | None."""
    if luts.shape[-1] != 64:
        raise ValueError("tables of 64 entries expected")
    return qadc_quantize_luts(luts, init_codes, R, nbins, qmin_mode, qmax_in)


def qadc_scan_topk(variant, codes, luts, R, nbins=255, workspace=None, out_idx=None, out_dist=None,
                   n=None):
    """codes u8 [n][row]; luts [nq][m][ksub] (u8 or f32 by variant) -> (idx i64-viewable u32 [nq][R], dist)."""
    nq, m, ksub = luts.shape
    if n is None:
        n = codes.shape[0]
    dev = luts.device
    want = torch.uint8 if variant in (QADC_U8_4BIT, QADC_U8_8BIT, QADC_U8_6BIT) else torch.float32
    if luts.dtype != want:
        raise ValueError(f"variant {variant} needs {want} tables")
    if out_idx is None:
        out_idx = torch.empty((nq, R), dtype=torch.int32, device=dev)  # bit pattern of uint32
    if out_dist is None:
        out_dist = torch.empty((nq, R), dtype=want, device=dev)
    need = qadc_workspace_bytes({QADC_U8_4BIT: QADC_WS_SCAN_TOPK, QADC_F32_4BIT: QADC_WS_SCAN_F32_4BIT,
                                 QADC_F32_8BIT: QADC_WS_SCAN_F32_8BIT,
                                 QADC_U8_8BIT: QADC_WS_SCAN_U8_8BIT,
                                 QADC_U8_6BIT: QADC_WS_SCAN_U8_6BIT}[variant], n, m, nq, R)
    if workspace is None:
        workspace = qadc_workspace_init(torch.empty((max(need, 256),), dtype=torch.uint8, device=dev))
    _check(lib().qadc_scan_topk(variant, _ptr(codes, torch.uint8), n, m, _ptr(luts), nq, R, nbins,
                                _ptr(out_idx), _ptr(out_dist), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream()))
    return out_idx, out_dist


def qadc_pq_encode(codebooks, x, out=None):
    """codebooks f32 [m][ksub][dsub], x f32 [n][d] -> codes u8 [n][m/2] (ksub 16), [n][3m/4] (ksub 64)
    or [n][m] (ksub 256)."""
    m, ksub, dsub = codebooks.shape
    n, d = x.shape
    row = m // 2 if ksub == 16 else 3 * m // 4 if ksub == 64 else m
    if out is None:
        out = torch.empty((n, row), dtype=torch.uint8, device=x.device)
    _check(lib().qadc_pq_encode(_ptr(codebooks, torch.float32), d, m, ksub, _ptr(x, torch.float32),
                                n, _ptr(out, torch.uint8), _stream()))
    return out


def qadc_rotate(rot, x, out=None):
    """rot f32 [d][d], x f32 [n][d] -> y f32 [n][d], y[i] = rot @ x[i]."""
    n, d = x.shape
    assert rot.shape == (d, d)
    if out is None:
        out = torch.empty((n, d), dtype=torch.float32, device=x.device)
    _check(lib().qadc_rotate(_ptr(rot, torch.float32), d, _ptr(x, torch.float32), n, _ptr(out, torch.float32),
                             _stream()))
    return out


def qadc_packed_bytes(n: int, m: int, layout: int) -> int:
    return int(lib().qadc_packed_bytes(n, m, layout))


def qadc_pack_codes(std_codes, layout, out=None):
    """std_codes u8 [n][m/2] -> the list in `layout`, flat u8 [qadc_packed_bytes(n, m, layout)]."""
    n, half = std_codes.shape
    if out is None:
        out = torch.empty((qadc_packed_bytes(n, 2 * half, layout),), dtype=torch.uint8, device=std_codes.device)
    _check(lib().qadc_pack_codes(_ptr(std_codes, torch.uint8), n, 2 * half, layout, _ptr(out, torch.uint8),
                                 _stream()))
    return out


def qadc_unpack_codes(packed, n, m, layout, out=None):
    """packed flat u8 (n codes in `layout`) -> std codes u8 [n][m/2]."""
    if out is None:
        out = torch.empty((n, m // 2), dtype=torch.uint8, device=packed.device)
    _check(lib().qadc_unpack_codes(_ptr(packed, torch.uint8), n, m, layout, _ptr(out, torch.uint8), _stream()))
    return out


def qadc_ivf_assign(coarse, x, out=None):
    """coarse f32 [K][d], x f32 [n][d] -> cells i32 [n]."""
    K, d = coarse.shape
    n = x.shape[0]
    assert x.shape[1] == d
    if out is None:
        out = torch.empty((n,), dtype=torch.int32, device=x.device)
    _check(lib().qadc_ivf_assign(_ptr(coarse, torch.float32), K, d, _ptr(x, torch.float32), n,
                                 _ptr(out, torch.int32), _stream()))
    return out


def qadc_multi_index_cells(halves, out=None):
    """halves f32 [2][K][d/2] -> the K*K cell centroids f32 [K*K][d], cell id = i*K + j."""
    _, K, dh = halves.shape
    if out is None:
        out = torch.empty((K * K, 2 * dh), dtype=torch.float32, device=halves.device)
    _check(lib().qadc_multi_index_cells(_ptr(halves, torch.float32), K, 2 * dh, _ptr(out, torch.float32),
                                        _stream()))
    return out


def qadc_multi_index_assign(halves, x, out=None):
    """halves f32 [2][K][d/2], x f32 [n][d] -> cells i32 [n]."""
    _, K, dh = halves.shape
    n = x.shape[0]
    assert x.shape[1] == 2 * dh
    if out is None:
        out = torch.empty((n,), dtype=torch.int32, device=x.device)
    _check(lib().qadc_multi_index_assign(_ptr(halves, torch.float32), K, 2 * dh, _ptr(x, torch.float32), n,
                                         _ptr(out, torch.int32), _stream()))
    return out


def qadc_multi_index_workspace_bytes(K: int, nq: int, nprobe: int) -> int:
    return int(lib().qadc_multi_index_workspace_bytes(K, nq, nprobe))


def qadc_multi_index_probes(halves, queries, nprobe, workspace=None, out=None):
    """halves f32 [2][K][d/2], queries f32 [nq][d] -> probes i32 [nq][nprobe]."""
    _, K, dh = halves.shape
    nq = queries.shape[0]
    assert queries.shape[1] == 2 * dh
    if workspace is None:
        workspace = torch.empty((max(16, qadc_multi_index_workspace_bytes(K, nq, nprobe)),), dtype=torch.uint8,
                                device=queries.device)
    if out is None:
        out = torch.empty((nq, nprobe), dtype=torch.int32, device=queries.device)
    _check(lib().qadc_multi_index_probes(_ptr(halves, torch.float32), K, 2 * dh, _ptr(queries, torch.float32), nq,
                                         nprobe, _ptr(out, torch.int32), _ptr(workspace, torch.uint8),
                                         workspace.numel(), _stream()))
    return out


def qadc_multi_index_group_workspace_bytes(n: int, K: int) -> int:
    return int(lib().qadc_multi_index_group_workspace_bytes(n, K))


def qadc_multi_index_group(cells, K, workspace=None):
    """cells i32 [n] (product cells of K half-centroids per half) -> (cell_ids u32-bits [L], list_off i64 [L+1],
    ids u32-bits [n_placed]): the lists of the occupied cells, ascending.  Reads L back from the device."""
    n = cells.shape[0]
    cap = min(n, K * K)
    dev = cells.device
    if workspace is None:
        workspace = torch.empty((max(16, qadc_multi_index_group_workspace_bytes(n, K)),), dtype=torch.uint8, device=dev)
    cell_ids = torch.zeros((max(cap, 1),), dtype=torch.int32, device=dev)
    list_off = torch.zeros((cap + 1,), dtype=torch.int64, device=dev)
    ids = torch.zeros((max(n, 1),), dtype=torch.int32, device=dev)
    n_lists = torch.zeros((1,), dtype=torch.int64, device=dev)
    _check(lib().qadc_multi_index_group(_ptr(cells, torch.int32), n, K, cap, _ptr(cell_ids, torch.int32),
                                        _ptr(list_off, torch.int64), _ptr(ids, torch.int32),
                                        _ptr(n_lists, torch.int64), _ptr(workspace, torch.uint8),
                                        workspace.numel(), _stream()))
    L = int(n_lists.item())
    list_off = list_off[:L + 1].clone()
    placed = int(list_off[L].item())
    return cell_ids[:L].clone(), list_off, ids[:placed].clone()


def qadc_multi_index_encode(halves, codebooks, x, cells, ids, out=None):
    """Residual codes in list order against the half-centroids: row p = enc(x[ids[p]] - (halves[0][c // K],
    halves[1][c % K])), c = cells[ids[p]]; u8 [len(ids)][m/2]."""
    _, K, dh = halves.shape
    m = codebooks.shape[0]
    n = x.shape[0]
    n_list = ids.shape[0]
    assert x.shape[1] == 2 * dh
    if out is None:
        out = torch.empty((n_list, m // 2), dtype=torch.uint8, device=x.device)
    _check(lib().qadc_multi_index_encode(_ptr(halves, torch.float32), K, _ptr(codebooks, torch.float32), 2 * dh, m,
                                         _ptr(x, torch.float32), n, _ptr(cells, torch.int32),
                                         _ptr(ids, torch.int32), n_list, _ptr(out, torch.uint8), _stream()))
    return out


def qadc_multi_index_slots(cell_ids, cells, out=None):
    """cell_ids u32-bits [L] ascending, cells i32 [...] -> list numbers i32 [...], -1 for cells without a list."""
    if out is None:
        out = torch.empty_like(cells)
    _check(lib().qadc_multi_index_slots(_ptr(cell_ids, torch.int32), cell_ids.numel(), _ptr(cells, torch.int32),
                                        cells.numel(), _ptr(out, torch.int32), _stream()))
    return out


def qadc_ivf_group_workspace_bytes(n: int, K: int) -> int:
    return int(lib().qadc_ivf_group_workspace_bytes(n, K))


def qadc_ivf_group(cells, K, workspace=None):
    """cells i32 [n] -> (list_off i64 [K+1], ids u32 [n]) as torch int64 / int32-typed-as-uint32 tensors.

    ids is returned as an int32 tensor holding the uint32 bit patterns (torch has no uint32 arithmetic).
    """
    n = cells.shape[0]
    if workspace is None:
        workspace = torch.empty((max(16, qadc_ivf_group_workspace_bytes(n, K)),), dtype=torch.uint8,
                                device=cells.device)
    list_off = torch.empty((K + 1,), dtype=torch.int64, device=cells.device)
    ids = torch.zeros((n,), dtype=torch.int32, device=cells.device)
    _check(lib().qadc_ivf_group(_ptr(cells, torch.int32), n, K, _ptr(list_off, torch.int64),
                                _ptr(ids, torch.int32), _ptr(workspace, torch.uint8), workspace.numel(),
                                _stream()))
    return list_off, ids


def qadc_ivf_encode(coarse, codebooks, x, cells, ids, out=None):
    """Residual codes in list order: row p = enc(x[ids[p]] - coarse[cells[ids[p]]]); u8 [len(ids)][m/2]."""
    K, d = coarse.shape
    m = codebooks.shape[0]
    n = x.shape[0]
    n_list = ids.shape[0]
    if out is None:
        out = torch.empty((n_list, m // 2), dtype=torch.uint8, device=x.device)
    _check(lib().qadc_ivf_encode(_ptr(coarse, torch.float32), K, _ptr(codebooks, torch.float32), d, m,
                                 _ptr(x, torch.float32), n, _ptr(cells, torch.int32), _ptr(ids, torch.int32),
                                 n_list, _ptr(out, torch.uint8), _stream()))
    return out


def qadc_profile_enable(on: bool) -> None:
    _check(lib().qadc_profile_enable(1 if on else 0))


def qadc_profile_only(which: int) -> None:
    """Profiling on for the kernels of one slot only; qadc_profile_enable(False) ends it."""
    _check(lib().qadc_profile_only(which))


def qadc_profile_read(which: int):
    """-> (total milliseconds, launches) of the named kernel since profiling was enabled."""
    ms, cnt = ctypes.c_double(0), ctypes.c_int64(0)
    _check(lib().qadc_profile_read(which, ctypes.byref(ms), ctypes.byref(cnt)))
    return ms.value, cnt.value


class IvfIndex:
    """Holds the tensors of an inverted index on the GPU and the C struct that points at them.

    coarse f32 [K][d], or None for a multi-index over its occupied cells: then `halves` f32 [2][Kh][d/2]
    and `cell_ids` u32-bits [K] (ascending product cell of every list) stand in for the centroids.
    """

    def __init__(self, coarse, list_off, codes, ids, codebooks, halves=None, cell_ids=None):
        m = codebooks.shape[0]
        if coarse is not None:
            K, d = coarse.shape
            hp, cp, Kh = None, None, 0
        else:
            assert halves is not None and cell_ids is not None
            _, Kh, dh = halves.shape
            K, d = cell_ids.numel(), 2 * dh
            hp, cp = _ptr(halves, torch.float32).value, _ptr(cell_ids, torch.int32).value
        assert codebooks.shape[1] == 16 and codes.shape[1] == m // 2
        assert list_off.dtype == torch.int64 and list_off.numel() == K + 1
        assert ids.dtype == torch.int32 or ids.dtype == torch.uint32
        self.tensors = (coarse, list_off, codes, ids, codebooks)  # keep alive
        self.half_tensors = (halves, cell_ids)
        self.c = qadc_ivf_index(_ptr(coarse, torch.float32).value if coarse is not None else None,
                                _ptr(list_off).value, _ptr(codes, torch.uint8).value, _ptr(ids).value,
                                _ptr(codebooks, torch.float32).value, d, m, K, codes.shape[0], hp, cp, Kh)
        self.d, self.m, self.K, self.n = d, m, K, codes.shape[0]


def qadc_ivf_workspace_bytes(index: IvfIndex, nq: int, nprobe: int, R: int) -> int:
    return int(lib().qadc_ivf_workspace_bytes(ctypes.byref(index.c), nq, nprobe, R))


def qadc_ivf_search(index: IvfIndex, queries, nprobe, R, init, nbins=255,
                    qmin_mode=QADC_QMIN_PER_TABLE, probes_in=None, workspace=None, debug=False):
    """-> (ids i32-bits-of-u32 [nq][R], dist u8 [nq][R][, probes i32 [nq][nprobe], qluts u8 [nq][nprobe][m][16]])."""
    nq = queries.shape[0]
    dev = queries.device
    out_ids = torch.empty((nq, R), dtype=torch.int32, device=dev)
    out_dist = torch.empty((nq, R), dtype=torch.uint8, device=dev)
    dbg_p = torch.empty((nq, nprobe), dtype=torch.int32, device=dev) if debug else None
    dbg_q = torch.empty((nq, nprobe, index.m, 16), dtype=torch.uint8, device=dev) if debug else None
    need = qadc_ivf_workspace_bytes(index, nq, nprobe, R)
    if workspace is None:
        workspace = qadc_workspace_init(torch.empty((max(need, 256),), dtype=torch.uint8, device=dev))
    _check(lib().qadc_ivf_search(ctypes.byref(index.c), _ptr(queries, torch.float32), nq, nprobe, R, init,
                                 nbins, qmin_mode, _ptr(probes_in, torch.int32), _ptr(out_ids),
                                 _ptr(out_dist), _ptr(dbg_p), _ptr(dbg_q), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream()))
    if debug:
        return out_ids, out_dist, dbg_p, dbg_q
    return out_ids, out_dist


def qadc_pq_train(train, m, ksub, init_rows, iters):
    """train f32 [n][d], init_rows i64 [ksub] -> codebooks f32 [m][ksub][d/m] (Lloyd k-means per sub-space)."""
    n, d = train.shape
    cb = torch.empty((m, ksub, d // m), dtype=torch.float32, device=train.device)
    ws = torch.empty((n * m,), dtype=torch.uint8, device=train.device)
    _check(lib().qadc_pq_train(_ptr(train, torch.float32), n, d, m, ksub, _ptr(init_rows, torch.int64),
                               iters, _ptr(cb), _ptr(ws), ws.numel(), _stream()))
    return cb


def qadc_search(codebooks, queries, codes, R, init, nbins=255, qmin_mode=QADC_QMIN_PER_TABLE,
                workspace=None, out_idx=None, out_dist=None, qluts_out=None, n=None):
    """Whole exhaustive Quick ADC query path in one call -> (idx u32-bits [nq][R], dist u8 [nq][R])."""
    m, ksub, dsub = codebooks.shape
    nq, d = queries.shape
    if n is None:
        n = codes.shape[0]
    dev = queries.device
    if out_idx is None:
        out_idx = torch.empty((nq, R), dtype=torch.int32, device=dev)
    if out_dist is None:
        out_dist = torch.empty((nq, R), dtype=torch.uint8, device=dev)
    if workspace is None:
        need = qadc_workspace_bytes(QADC_WS_SEARCH, n, m, nq, R)
        workspace = qadc_workspace_init(torch.empty((max(need, 256),), dtype=torch.uint8, device=dev))
    _check(lib().qadc_search(_ptr(codebooks, torch.float32), d, m, _ptr(queries, torch.float32), nq,
                             _ptr(codes, torch.uint8), n, R, init, nbins, qmin_mode, _ptr(out_idx),
                             _ptr(out_dist), _ptr(qluts_out, torch.uint8), _ptr(workspace),
                             workspace.numel() * workspace.element_size(), _stream()))
    return out_idx, out_dist


def qadc_static_scratch_bytes() -> int:
    return int(lib().qadc_static_scratch_bytes())


def qadc_search_static(codebooks, queries, codes, R, init, out_idx, out_dist, nbins=255,
                       qmin_mode=QADC_QMIN_PER_TABLE, qluts_out=None, n=None):
    """qadc_search without a workspace and without any allocation: the caller passes the outputs
    (idx i32 [nq][R], dist u8 [nq][R]); the scratch is the library's static device array."""
    m, ksub, dsub = codebooks.shape
    nq, d = queries.shape
    if n is None:
        n = codes.shape[0]
    _check(lib().qadc_search_static(_ptr(codebooks, torch.float32), d, m, _ptr(queries, torch.float32), nq,
                                    _ptr(codes, torch.uint8), n, R, init, nbins, qmin_mode, _ptr(out_idx),
                                    _ptr(out_dist), _ptr(qluts_out, torch.uint8), _stream()))
    return out_idx, out_dist


# ---------------------------------------------------------------------------------------------
# operators of a language model next to the search

_TYPES = {torch.float32: QADC_TYPE_F32, torch.float16: QADC_TYPE_F16, torch.bfloat16: QADC_TYPE_BF16}


def _type(t) -> int:
    if t.dtype not in _TYPES:
        raise ValueError(f"expected float32, float16 or bfloat16, got {t.dtype}")
    return _TYPES[t.dtype]


def _matrix(t, dtype=None, device=None):
    """Pointer and row distance of a matrix whose rows are dense but may lie apart."""
    if t.dim() != 2:
        raise ValueError("expected a matrix")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    rows, cols = t.shape
    ld = t.stride(0) if rows > 1 else cols
    if not (t.is_cuda if device is None else t.get_device() == device) or (cols > 1 and rows > 0 and t.stride(1) != 1) or ld < cols:
        raise _refusal(t, device, "tensor must be a GPU matrix with dense rows that do not overlap")
    return t.data_ptr(), ld


def _vector(t, n, dtype=None, device=None):
    """Pointer of a dense vector of n elements, or None."""
    if t is None:
        return None
    if t.numel() != n:
        raise ValueError(f"expected {n} elements, got {t.numel()}")
    if not (t.is_cuda if device is None else t.get_device() == device) or not t.is_contiguous():
        raise _refusal(t, device, "tensor must be a contiguous GPU tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _weight_type(weight, bias, x) -> int:
    if weight is None:
        weight, bias = bias, None
    if weight is None:
        return QADC_TYPE_F32
    if (bias is not None and bias.dtype != weight.dtype) or weight.dtype not in (torch.float32, x.dtype):
        raise ValueError("weight and bias must both be float32, or both of x's type")
    return _TYPES[weight.dtype]


def _like(t, x, device=None):
    """The caller's dense output tensor, checked to be one like the matrix x, or a new one."""
    if t is None:
        return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if (t.shape != x.shape or t.dtype != x.dtype or not (t.is_cuda if device is None else t.get_device() == device) or
            not t.is_contiguous()):
        raise _refusal(t, device, f"output must be a contiguous {x.dtype} GPU tensor of {tuple(x.shape)}")
    return t


def _pair(device, *shape):
    """Two new float32 tensors (sizes one by one and empty_like: 2.4 us against 2.9 for the halves of one tensor)."""
    one = torch.empty(*shape, dtype=torch.float32, device=device)
    return one, torch.empty_like(one)


def _scratch(workspace, need, sizes, device):
    """The caller's workspace, or a new one of need(*sizes) bytes (not cleared); its size in bytes."""
    if workspace is None:
        workspace = torch.empty((max(need(*sizes), 256),), dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def qadc_layer_norm(x, weight=None, bias=None, eps=1e-5, out=None):
    """x [rows][d] (f32, f16 or bf16; rows may lie apart), weight, bias [d] (f32 or x's type) | None
    -> (y [rows][d] of x's type, mean f32 [rows], rstd f32 [rows])."""
    rows, d = x.shape
    xp, ldx = _matrix(x)
    y = _like(out, x)
    mean, rstd = _pair(x.device, rows)
    _check(lib().qadc_layer_norm(xp, ldx, _type(x), _vector(weight, d), _vector(bias, d), _weight_type(weight, bias, x),
                                 rows, d, eps, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _stream()))
    return y, mean, rstd


def qadc_layer_norm_workspace_bytes(rows: int, d: int) -> int:
    return int(lib().qadc_layer_norm_workspace_bytes(rows, d))


def qadc_layer_norm_backward(dy, x, weight, mean, rstd, workspace=None, out=None, need_dx=True, need_weights=True):
    """dy, x [rows][d], weight [d] | None, mean, rstd f32 [rows] of qadc_layer_norm
    -> (dx [rows][d] of x's type | None, dweight f32 [d] | None, dbias f32 [d] | None)."""
    rows, d = x.shape
    if tuple(dy.shape) != (rows, d):
        raise ValueError("dy must have x's shape")
    dyp, lddy = _matrix(dy, x.dtype)
    xp, ldx = _matrix(x)
    dx = _like(out, x) if need_dx else None
    dw = db = None
    size = 0
    if need_weights:
        dw, db = _pair(x.device, d)
        workspace, size = _scratch(workspace, qadc_layer_norm_workspace_bytes, (rows, d), x.device)
    else:
        workspace = None
    _check(lib().qadc_layer_norm_backward(dyp, lddy, xp, ldx, _type(x), _vector(weight, d), _weight_type(weight, None, x),
                                          _vector(mean, rows, torch.float32), _vector(rstd, rows, torch.float32), rows, d,
                                          _ptr(dx), _ptr(dw), _ptr(db), _ptr(workspace), size, _stream()))
    return dx, dw, db


def qadc_rms_norm(x, weight=None, residual=None, eps=1e-5, out_type=None, sum_out=None, out=None):
    """x [rows][d] (f32, f16 or bf16; rows may lie apart), weight [d] (f32 or x's type) | None, residual like x | None,
    out_type None (x's) or torch.float8_e4m3fn
    -> (y [rows][d], x + residual [rows][d] of x's type | None, scale f32 [rows] | None, rstd f32 [rows])."""
    rows, d = x.shape
    xp, ldx = _matrix(x)
    device = x.get_device()
    xtype = ytype = _type(x)
    rp = sp = scale = None
    ldr = ld_sum = d
    if residual is not None:
        if residual.shape != x.shape:
            raise ValueError("residual must have x's shape")
        rp, ldr = _matrix(residual, x.dtype, device)
        if sum_out is None:
            sum_out = _like(None, x)
        elif sum_out.shape != x.shape:
            raise ValueError(f"sum_out must be {tuple(x.shape)}")
        sp, ld_sum = _matrix(sum_out, x.dtype, device)
    elif sum_out is not None:
        raise ValueError("sum_out needs a residual")
    if out_type is None or out_type == x.dtype:
        y = _like(out, x, device)
    elif out_type == torch.float8_e4m3fn:
        ytype = QADC_TYPE_E4M3
        y = out if out is not None else torch.empty(rows, d, dtype=out_type, device=x.device)
        if y.shape != x.shape or y.dtype != out_type or y.get_device() != device or not y.is_contiguous():
            raise _refusal(y, device, f"output must be a contiguous {out_type} GPU tensor of {tuple(x.shape)}")
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
    else:
        raise ValueError(f"out_type must be {x.dtype} or torch.float8_e4m3fn")
    rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    _check(lib().qadc_rms_norm(xp, ldx, rp, ldr, xtype, _vector(weight, d, None, device), _weight_type(weight, None, x), rows, d, eps, sp,
                               ld_sum, y.data_ptr(), ytype, None if scale is None else scale.data_ptr(), rstd.data_ptr(),
                               _stream_on(device)))
    return y, sum_out, scale, rstd


def qadc_rms_norm_workspace_bytes(rows: int, d: int) -> int:
    return int(lib().qadc_rms_norm_workspace_bytes(rows, d))


def qadc_rms_norm_backward(dy, h, weight, rstd, dsum=None, workspace=None, out=None, need_dx=True, need_weight=True):
    """dy, h [rows][d] (h: x + residual of qadc_rms_norm, or its x), weight [d] | None, rstd f32 [rows], dsum like dy | None
    -> (dx [rows][d] of h's type | None, dweight f32 [d] | None)."""
    rows, d = h.shape
    if tuple(dy.shape) != (rows, d) or (dsum is not None and tuple(dsum.shape) != (rows, d)):
        raise ValueError("dy and dsum must have h's shape")
    hp, ldh = _matrix(h)
    device = h.get_device()
    dyp, lddy = _matrix(dy, h.dtype, device)
    sp, lds = (None, d) if dsum is None else _matrix(dsum, h.dtype, device)
    dx = _like(out, h, device) if need_dx else None
    dw = None
    size = 0
    if need_weight:
        dw = torch.empty(d, dtype=torch.float32, device=h.device)
        workspace, size = _scratch(workspace, qadc_rms_norm_workspace_bytes, (rows, d), h.device)
    else:
        workspace = None
    _check(lib().qadc_rms_norm_backward(dyp, lddy, sp, lds, hp, ldh, _type(h), _vector(weight, d, None, device),
                                        _weight_type(weight, None, h), _vector(rstd, rows, torch.float32, device), rows, d, _ptr(dx), _ptr(dw),
                                        _ptr(workspace, None, device), size, _stream_on(device)))
    return dx, dw


def qadc_weights4_bytes(N: int, K: int, group: int, has_zeros) -> int:
    return int(lib().qadc_weights4_bytes(N, K, group, int(bool(has_zeros))))


def qadc_pack_weights4(codes, scales, zeros, K, group):
    """codes u8 [N][ceil(K/2)], scales f16 or bf16 [N][ceil(K/group)], zeros u8 like scales | None -> qadc_weights4."""
    N = codes.shape[0]
    groups = -(-K // group) if group > 0 else 0
    if tuple(codes.shape) != (N, -(-K // 2)) or tuple(scales.shape) != (N, groups):
        raise ValueError(f"expected codes [N][{-(-K // 2)}] and scales [N][{groups}]")
    if zeros is not None and tuple(zeros.shape) != (N, groups):
        raise ValueError(f"expected zeros [N][{groups}]")
    stype = _type(scales)
    packed = torch.empty((max(16, qadc_weights4_bytes(N, K, group, zeros is not None)),), dtype=torch.uint8, device=codes.device)
    _check(lib().qadc_pack_weights4(_ptr(codes, torch.uint8), _ptr(scales), stype, _ptr(zeros, torch.uint8), N, K, group,
                                    _ptr(packed), _stream()))
    w = qadc_weights4(packed.data_ptr(), N, K, group, stype, int(zeros is not None))
    w.tensor = packed
    return w


def qadc_linear4(weights, x, bias=None, out=None):
    """weights of qadc_pack_weights4, x [M][K] (f32, f16 or bf16; rows may lie apart), bias f32 [N] | None -> y [M][N] of x's type."""
    M, K = x.shape
    if K != weights.K:
        raise ValueError(f"weights of {weights.K} inputs, x of {K}")
    xp, ldx = _matrix(x)
    if out is None:
        out = torch.empty(M, weights.N, dtype=x.dtype, device=x.device)
    elif tuple(out.shape) != (M, weights.N):
        raise ValueError(f"output must be {(M, weights.N)}")
    yp, ldy = _matrix(out, x.dtype)
    _check(lib().qadc_linear4(ctypes.byref(weights), xp, ldx, _type(x), M, _vector(bias, weights.N, torch.float32), yp, ldy,
                              _stream()))
    return out


def qadc_token_logprobs_workspace_bytes(rows: int, V: int, k: int) -> int:
    return int(lib().qadc_token_logprobs_workspace_bytes(rows, V, k))


def _tokens(tokens, rows, device=None):
    """Pointer and number per row of the given tokens, i32 [rows][T] or None."""
    if tokens is None:
        return None, 0
    if tokens.dim() != 2 or tokens.shape[0] != rows:
        raise ValueError(f"expected tokens [{rows}][T]")
    return _ptr(tokens, torch.int32, device), tokens.shape[1]


def qadc_token_logprobs(logits, tokens=None, k=0, scale=1.0, workspace=None):
    """logits [rows][V] (f32, f16 or bf16; rows may lie apart), tokens i32 [rows][T] | None
    -> (logp f32 [rows][T], lse f32 [rows], entropy f32 [rows], top_idx i32-bits-of-u32 [rows][k], top_logp f32 [rows][k])."""
    rows, V = logits.shape
    xp, ld = _matrix(logits)
    tp, T = _tokens(tokens, rows)
    dev = logits.device
    lse, entropy = _pair(dev, rows)
    logp = torch.empty(rows, T, dtype=torch.float32, device=dev)
    top_logp = torch.empty(rows, k, dtype=torch.float32, device=dev)
    top_idx = torch.empty(rows, k, dtype=torch.int32, device=dev)
    workspace, size = _scratch(workspace, qadc_token_logprobs_workspace_bytes, (rows, V, k), dev)
    _check(lib().qadc_token_logprobs(xp, ld, _type(logits), rows, V, scale, tp, T, k, logp.data_ptr(), lse.data_ptr(),
                                     entropy.data_ptr(), top_idx.data_ptr(), top_logp.data_ptr(), _ptr(workspace), size,
                                     _stream()))
    return logp, lse, entropy, top_idx, top_logp


def qadc_token_logprobs_backward(logits, tokens, lse, entropy, dlogp, dentropy=None, scale=1.0, out=None):
    """The gradient with respect to the logits, [rows][V] of their type; entropy may be None without dentropy."""
    rows, V = logits.shape
    xp, ld = _matrix(logits)
    tp, T = _tokens(tokens, rows)
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy needs the entropy")
    if out is None:
        out = torch.empty((rows, V), dtype=logits.dtype, device=logits.device)
    elif tuple(out.shape) != (rows, V):
        raise ValueError(f"output must be {(rows, V)}")
    op, ldd = _matrix(out, logits.dtype)
    _check(lib().qadc_token_logprobs_backward(xp, ld, _type(logits), rows, V, scale, tp, T, _vector(lse, rows, torch.float32),
                                              _vector(entropy, rows, torch.float32),
                                              _vector(dlogp, rows * T, torch.float32) if T else None,
                                              _vector(dentropy, rows, torch.float32), op, ldd, _stream()))
    return out


def qadc_adapters_workspace_bytes(adapters, M: int) -> int:
    return int(lib().qadc_adapters_workspace_bytes(ctypes.byref(adapters), M))


def qadc_add_adapters(adapters, ids, x, base=None, out=None, workspace=None):
    """adapters: a qadc_adapters, ids i32 [M], x [M][K] and base [M][N] | None of the pool's type (rows may lie apart)
    -> y [M][N]: base + each row's own adapter's product with x (out may be base)."""
    M, K = x.shape
    if K != adapters.K:
        raise ValueError(f"adapters of {adapters.K} inputs, x of {K}")
    device = adapters.device
    xp, ldx = _matrix(x, adapters.dtype, device)
    bp, ldb = None, adapters.N
    if base is not None:
        if tuple(base.shape) != (M, adapters.N):
            raise ValueError(f"base must be {(M, adapters.N)}")
        bp, ldb = _matrix(base, adapters.dtype, device)
    if out is None:
        out = torch.empty(M, adapters.N, dtype=adapters.dtype, device=x.device)
    elif tuple(out.shape) != (M, adapters.N):
        raise ValueError(f"output must be {(M, adapters.N)}")
    yp, ldy = _matrix(out, adapters.dtype, device)
    if workspace is None:
        workspace = torch.empty((max(256, qadc_adapters_workspace_bytes(adapters, M)),), dtype=torch.uint8, device=x.device)
    _check(lib().qadc_add_adapters(ctypes.byref(adapters), _vector(ids, M, torch.int32, device), xp, ldx, M, bp, ldb, yp, ldy,
                                   _ptr(workspace, None, device), workspace.numel() * workspace.element_size(), _stream_on(device)))
    return out


def _teacher(top_idx, top_logp, rows, device):
    """Pointers and number per row of a teacher's stored tokens and log probabilities."""
    if top_idx.dim() != 2 or top_idx.shape[0] != rows or top_logp.shape != top_idx.shape:
        raise ValueError(f"expected top_idx and top_logp [{rows}][k]")
    if top_idx.dtype not in (torch.int32, torch.uint32):
        raise ValueError(f"expected 32-bit indexes, got {top_idx.dtype}")
    return _ptr(top_idx, None, device), _ptr(top_logp, torch.float32, device), top_idx.shape[1]


def qadc_distill_workspace_bytes(rows: int, V: int) -> int:
    return int(lib().qadc_distill_workspace_bytes(rows, V))


def qadc_distill(logits, top_idx, top_logp, scale=1.0, tail=True, workspace=None):
    """logits [rows][V] (f32, f16 or bf16; rows may lie apart), top_idx i32-bits-of-u32 and top_logp f32 [rows][k] of a teacher
    (qadc_token_logprobs) -> (loss f32 [rows], lse f32 [rows], log_tail f32 [rows])."""
    rows, V = logits.shape
    xp, ld = _matrix(logits)
    device = logits.get_device()
    ip, lp, k = _teacher(top_idx, top_logp, rows, device)
    loss, lse = _pair(logits.device, rows)
    log_tail = torch.empty_like(loss)
    workspace, size = _scratch(workspace, qadc_distill_workspace_bytes, (rows, V), logits.device)
    _check(lib().qadc_distill(xp, ld, _type(logits), rows, V, scale, ip, lp, k, int(bool(tail)), loss.data_ptr(), lse.data_ptr(),
                              log_tail.data_ptr(), _ptr(workspace, None, device), size, _stream_on(device)))
    return loss, lse, log_tail


def _gradient_like(out, logits):
    """The caller's matrix for a gradient with respect to the logits, or a new one; its pointer and row distance."""
    if out is None:
        out = _like(None, logits)
    elif out.shape != logits.shape:
        raise ValueError(f"output must be {tuple(logits.shape)}")
    return (out, *_matrix(out, logits.dtype, logits.get_device()))


def qadc_distill_backward(logits, top_idx, top_logp, lse, log_tail, dloss, scale=1.0, tail=True, out=None):
    """lse, log_tail f32 [rows] of qadc_distill, dloss f32 [rows] -> the gradient with respect to the logits, [rows][V] of their
    type."""
    rows, V = logits.shape
    xp, ld = _matrix(logits)
    device = logits.get_device()
    ip, lp, k = _teacher(top_idx, top_logp, rows, device)
    out, op, ldd = _gradient_like(out, logits)
    f32 = torch.float32
    _check(lib().qadc_distill_backward(xp, ld, _type(logits), rows, V, scale, ip, lp, k, int(bool(tail)), _vector(lse, rows, f32, device),
                                       _vector(log_tail, rows, f32, device), _vector(dloss, rows, f32, device), op, ldd, _stream_on(device)))
    return out


def qadc_distill_step(logits, top_idx, top_logp, weight, scale=1.0, tail=True, out=None, workspace=None):
    """qadc_distill and, with dloss = weight f32 [rows], qadc_distill_backward in one call
    -> (loss f32 [rows], gradient [rows][V] of the logits' type)."""
    rows, V = logits.shape
    xp, ld = _matrix(logits)
    device = logits.get_device()
    ip, lp, k = _teacher(top_idx, top_logp, rows, device)
    out, op, ldd = _gradient_like(out, logits)
    loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    workspace, size = _scratch(workspace, qadc_distill_workspace_bytes, (rows, V), logits.device)
    _check(lib().qadc_distill_step(xp, ld, _type(logits), rows, V, scale, ip, lp, k, int(bool(tail)),
                                   _vector(weight, rows, torch.float32, device), loss.data_ptr(), op, ldd, _ptr(workspace, None, device), size,
                                   _stream_on(device)))
    return loss, out


def qadc_adjust_logits(logits, history=None, lengths=None, prompt=None, repetition=None, presence=None, frequency=None,
                       bias_tokens=None, bias=None, masks=None, mask_of=None, out=None):
    """logits [rows][V] (f32, f16 or bf16; rows may lie apart), history i32 [rows][H], lengths, prompt i32 [rows], repetition,
    presence, frequency f32 [rows], bias_tokens i32 and bias f32 [rows][B], masks i32 or u32 [states][>= ceil(V/32)], mask_of
    i32 [rows], each | None -> adjusted logits [rows][V] of their type."""
    rows, V = logits.shape
    xp, ld = _matrix(logits)
    device = logits.get_device()
    hp, H = _tokens(history, rows, device)
    bp, B = _tokens(bias_tokens, rows, device)
    if (bias is None) != (bias_tokens is None):
        raise ValueError("bias and bias_tokens belong together")
    if history is None and not (lengths is prompt is repetition is presence is frequency is None):
        raise ValueError("lengths, prompt and penalties need a history")
    mp, ldm, states = None, 0, 0
    if masks is not None:
        if masks.dtype not in (torch.int32, torch.uint32):
            raise ValueError(f"expected masks of 32-bit words, got {masks.dtype}")
        mp, ldm = _matrix(masks, None, device)
        states = masks.shape[0]
        if masks.shape[1] < -(-V // 32):
            raise ValueError(f"expected masks of {-(-V // 32)} words")
    elif mask_of is not None:
        raise ValueError("mask_of needs masks")
    if out is None:
        out = _like(None, logits)
    elif tuple(out.shape) != (rows, V):
        raise ValueError(f"output must be {(rows, V)}")
    op, ldo = _matrix(out, logits.dtype, device)
    f32, i32 = torch.float32, torch.int32
    _check(lib().qadc_adjust_logits(xp, ld, _type(logits), rows, V, hp, H, _vector(lengths, rows, i32, device),
                                    _vector(prompt, rows, i32, device), _vector(repetition, rows, f32, device),
                                    _vector(presence, rows, f32, device), _vector(frequency, rows, f32, device), bp,
                                    _vector(bias, rows * B, f32, device), B, mp, ldm, states, _vector(mask_of, rows, i32, device), op,
                                    ldo, _stream_on(device)))
    return out


def qadc_neighbour_mix(ids, dist, values, tokens, lm_logp, lam, beta, step=None):
    """ids i32-bits-of-u32 [rows][R], dist f32 or u8 [rows][R], values i32 [n], tokens i32 [rows][T], lm_logp f32 [rows][T],
    step f32 [rows] | None -> (mix f32 [rows][T], knn f32 [rows][T])."""
    rows, R = ids.shape
    if tuple(dist.shape) != (rows, R) or dist.dtype not in (torch.float32, torch.uint8):
        raise ValueError("dist must be float32 or uint8 and have the shape of ids")
    if ids.dtype not in (torch.int32, torch.uint32):
        raise ValueError(f"expected 32-bit ids, got {ids.dtype}")
    if tokens is None or tuple(lm_logp.shape) != tuple(tokens.shape):
        raise ValueError("lm_logp must have the shape of tokens")
    tp, T = _tokens(tokens, rows)
    mix, knn = _pair(ids.device, rows, T)
    _check(lib().qadc_neighbour_mix(_ptr(ids), _ptr(dist), dist.element_size(), _vector(step, rows, torch.float32), rows, R,
                                    _ptr(values, torch.int32), values.numel(), beta, tp, T, _ptr(lm_logp, torch.float32), lam,
                                    mix.data_ptr(), knn.data_ptr(), _stream()))
    return mix, knn
