"""ctypes binding of the C ABI in ``include/attn.h`` -- argument marshalling only.

Every step of the attention forward pass runs in the CUDA library; torch is used for
device memory and streams.  The library is never substituted: if ``libattn_b200.so``
is missing or fails to load, importing a symbol here raises.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# ATTN_B200_LIB names another build of the same library (e.g. one compiled with a different
# register split for an A/B run); it is loaded instead of the in-tree one, never in addition.
LIB_PATH = os.environ.get("ATTN_B200_LIB") or os.path.join(_PKG, "libattn_b200.so")

ATTN_OK = 0
STATUS_NAMES = {
    0: "ATTN_OK", 1: "ATTN_ERR_NULL", 2: "ATTN_ERR_SHAPE", 3: "ATTN_ERR_UNSUPPORTED", 4: "ATTN_ERR_ALIGN",
    5: "ATTN_ERR_CUDA", 6: "ATTN_ERR_ARCH", 7: "ATTN_ERR_TIMEOUT", 8: "ATTN_ERR_TOO_LARGE",
}
EXPORTED_SYMBOLS = ("attn_fwd", "attn_fwd_strided", "attn_fwd_host", "attn_fwd_noalloc", "attn_merge", "attn_merge_n",
                    "attn_fwd_splitkv", "attn_splitkv_workspace_bytes", "attn_bwd", "attn_bwd_strided", "attn_bwd_workspace_bytes", "attn_bwd_plan", "attn_bwd_plan_item",
                    "attn_qk_norm_rope", "attn_qk_norm_rope_bwd", "attn_qk_norm_rope_bwd_workspace_bytes",
                    "attn_release_host_staging", "attn_set_option",
                    "attn_get_option",
                    "attn_plan", "attn_plan_item", "attn_plan_item_pair", "attn_last_launch_clock", "attn_launch_clocks", "attn_selftest_wait_timeout", "attn_status_str", "attn_version",
                    "attn_last_device_status")

_lib = None
_BF16 = torch.bfloat16
_LL3 = ctypes.c_longlong * 3


class AttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


def load_library() -> ctypes.CDLL:
    """Loads ``libattn_b200.so`` (built by ``paper_2603_24517_b200.build``); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} not found: run `python -m paper_2603_24517_b200.build` "
                          "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    fwd_args = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, cf, vp]
    lib.attn_fwd.argtypes = fwd_args
    lib.attn_fwd.restype = ci
    lib.attn_fwd_host.argtypes = fwd_args
    lib.attn_fwd_host.restype = ci
    lib.attn_fwd_noalloc.argtypes = fwd_args
    ll3 = ctypes.POINTER(ctypes.c_longlong)
    lib.attn_fwd_strided.argtypes = fwd_args[:11] + [ll3, ll3, ll3, ll3] + fwd_args[11:]
    lib.attn_fwd_strided.restype = ci
    lib.attn_fwd_noalloc.restype = ci
    lib.attn_release_host_staging.argtypes = []
    lib.attn_release_host_staging.restype = ci
    lib.attn_set_option.argtypes = [ctypes.c_char_p, ci]
    lib.attn_set_option.restype = ci
    lib.attn_get_option.argtypes = [ctypes.c_char_p, ctypes.POINTER(ci)]
    lib.attn_get_option.restype = ci
    lib.attn_plan.argtypes = [ci] * 8 + [ctypes.POINTER(ci)]
    lib.attn_plan.restype = ci
    lib.attn_plan_item.argtypes = [ci] * 8 + [ctypes.POINTER(ci)]
    lib.attn_plan_item.restype = ci
    lib.attn_plan_item_pair.argtypes = [ci] * 9 + [ctypes.POINTER(ci)]
    lib.attn_plan_item_pair.restype = ci
    lib.attn_merge.argtypes = [vp, vp, vp, vp, vp, vp, ci, ci, ci, ci, vp]
    lib.attn_merge.restype = ci
    lib.attn_merge_n.argtypes = [vp, vp, ci, vp, vp, ci, ci, ci, ci, vp]
    lib.attn_merge_n.restype = ci
    lib.attn_splitkv_workspace_bytes.argtypes = [ci] * 5
    lib.attn_splitkv_workspace_bytes.restype = ctypes.c_size_t
    lib.attn_fwd_splitkv.argtypes = fwd_args[:13] + [ci, vp, ctypes.c_size_t, vp]
    lib.attn_fwd_splitkv.restype = ci
    bwd_args = [vp] * 10 + [ci] * 6
    lib.attn_bwd.argtypes = bwd_args + [ci, cf, vp, ctypes.c_size_t, vp]
    lib.attn_bwd.restype = ci
    lib.attn_bwd_strided.argtypes = bwd_args + [ll3] * 8 + [ci, cf, vp, ctypes.c_size_t, vp]
    lib.attn_bwd_strided.restype = ci
    lib.attn_bwd_workspace_bytes.argtypes = [ci] * 7
    lib.attn_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.attn_bwd_plan.argtypes = [ci] * 7 + [ctypes.POINTER(ci)]
    lib.attn_bwd_plan.restype = ci
    lib.attn_bwd_plan_item.argtypes = [ci] * 8 + [ctypes.POINTER(ci)]
    lib.attn_bwd_plan_item.restype = ci
    rope_in = [vp, vp, vp, vp, ci, vp, vp, vp, ci, ctypes.POINTER(ctypes.c_longlong)]
    lib.attn_qk_norm_rope.argtypes = rope_in + [vp, vp] + [ci] * 8 + [cf] + [ll3] * 4 + [vp]
    lib.attn_qk_norm_rope.restype = ci
    lib.attn_qk_norm_rope_bwd.argtypes = [vp, vp] + rope_in + [vp] * 4 + [ci] * 8 + [cf] + [ll3] * 6 + [vp, ctypes.c_size_t, vp]
    lib.attn_qk_norm_rope_bwd.restype = ci
    lib.attn_qk_norm_rope_bwd_workspace_bytes.argtypes = []
    lib.attn_qk_norm_rope_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.attn_selftest_wait_timeout.argtypes = [ci, vp]
    lib.attn_selftest_wait_timeout.restype = ci
    lib.attn_status_str.argtypes = [ci]
    lib.attn_status_str.restype = ctypes.c_char_p
    lib.attn_version.argtypes = []
    lib.attn_version.restype = ci
    lib.attn_last_launch_clock.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.attn_last_launch_clock.restype = ci
    lib.attn_launch_clocks.argtypes = [ctypes.POINTER(ctypes.c_double), ci, ctypes.POINTER(ci)]
    lib.attn_launch_clocks.restype = ci
    lib.attn_last_device_status.argtypes = [ctypes.POINTER(ci), ctypes.POINTER(ci)]
    lib.attn_last_device_status.restype = ci
    _lib = lib
    return lib


def _check_layout(q, k, v, o, lse, device_type):
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        if t.dtype != torch.bfloat16 or t.dim() != 4 or not t.is_contiguous() or t.device.type != device_type:
            raise ValueError(f"{name} must be a contiguous 4-D bfloat16 {device_type} tensor [B, S, H, D]")
    B, Sq, Hq, D = q.shape
    Bk, Sk, Hkv, Dk = k.shape
    if v.shape != k.shape or o.shape != q.shape or Bk != B or Dk != D:
        raise ValueError("inconsistent q/k/v/o shapes")
    if lse is not None:
        if lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (B, Hq, Sq) \
                or lse.device.type != device_type:
            raise ValueError("lse must be a contiguous float32 tensor [B, Hq, Sq]")
    return B, Hq, Hkv, Sq, Sk, D


def attn_fwd_status(q, k, v, o, lse, causal: bool, scale: float, stream=None) -> int:
    """Calls ``attn_fwd`` on CUDA tensors and returns its raw status code (no exception)."""
    B, Hq, Hkv, Sq, Sk, D = _check_layout(q, k, v, o, lse, "cuda")
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    with torch.cuda.device(q.device):
        return load_library().attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                       None if lse is None else lse.data_ptr(),
                                       B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), float(scale), stream)


def attn_fwd(q, k, v, o, lse, causal: bool, scale: float, stream=None) -> None:
    """``attn_fwd`` of the C ABI on CUDA tensors: q [B,Sq,Hq,D], k/v [B,Sk,Hkv,D] -> o, lse
    (lse may be None).  Asynchronous on ``stream`` (default: torch's current stream)."""
    st = attn_fwd_status(q, k, v, o, lse, causal, scale, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_fwd")


def _strides3(t):
    """Element strides of the (batch, sequence, head) axes of a [B, S, H, D] tensor as a C array.
    An axis of extent 1 is never stepped along, so it gets the stride a contiguous tensor would
    have (torch may report anything there)."""
    B, S, H, D = t.shape
    b, s, h, _ = t.stride()
    return _LL3(S * H * D if B == 1 else b, H * D if S == 1 else s, D if H == 1 else h)


def attn_fwd_strided_status(q, k, v, o, lse, causal: bool, scale: float, stream=None) -> int:
    """Calls ``attn_fwd_strided`` on CUDA tensors of shape [B, S, H, D] with arbitrary batch,
    sequence and head strides (the head dimension must be contiguous); returns the raw status."""
    for name, t in (("q", q), ("k", k), ("v", v), ("o", o)):
        if t.dtype != torch.bfloat16 or t.dim() != 4 or t.stride(3) != 1 or t.device.type != "cuda":
            raise ValueError(f"{name} must be a 4-D bfloat16 cuda tensor [B, S, H, D] with a contiguous last axis")
    B, Sq, Hq, D = q.shape
    Bk, Sk, Hkv, Dk = k.shape
    if v.shape != k.shape or o.shape != q.shape or Bk != B or Dk != D:
        raise ValueError("inconsistent q/k/v/o shapes")
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous()
                            or tuple(lse.shape) != (B, Hq, Sq) or lse.device.type != "cuda"):
        raise ValueError("lse must be a contiguous float32 tensor [B, Hq, Sq]")
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    with torch.cuda.device(q.device):
        return load_library().attn_fwd_strided(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                               None if lse is None else lse.data_ptr(),
                                               B, Hq, Hkv, Sq, Sk, D, _strides3(q), _strides3(k), _strides3(v),
                                               _strides3(o), int(bool(causal)), float(scale), stream)


def attn_fwd_strided(q, k, v, o, lse, causal: bool, scale: float, stream=None) -> None:
    """``attn_fwd_strided`` of the C ABI: ``attn_fwd`` on views -- a [B, H, S, D] buffer seen as
    [B, S, H, D], slices of a packed QKV projection, a key range of a longer sequence."""
    st = attn_fwd_strided_status(q, k, v, o, lse, causal, scale, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_fwd_strided")


def attn_fwd_noalloc_status(q, k, v, o, lse, causal: bool, scale: float, stream=None) -> int:
    """Calls ``attn_fwd_noalloc`` on CUDA tensors and returns its raw status code."""
    B, Hq, Hkv, Sq, Sk, D = _check_layout(q, k, v, o, lse, "cuda")
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    with torch.cuda.device(q.device):
        return load_library().attn_fwd_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                               None if lse is None else lse.data_ptr(),
                                               B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), float(scale), stream)


def attn_fwd_noalloc(q, k, v, o, lse, causal: bool, scale: float, stream=None) -> None:
    """``attn_fwd_noalloc`` of the C ABI: ``attn_fwd`` for callers that may not allocate device
    memory.  The library keeps the kernel's scratch in a fixed 256-byte device array instead
    of allocating it, so calls that could overlap on the GPU must not use this entry point,
    and problems beyond ``ATTN_NOALLOC_MAX_Q_TILES`` query tiles are refused
    (``ATTN_ERR_TOO_LARGE``).  Make the first call on a device outside stream capture."""
    st = attn_fwd_noalloc_status(q, k, v, o, lse, causal, scale, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_fwd_noalloc")


def attn_fwd_host(q, k, v, o, lse, causal: bool, scale: float, device=0, stream=None) -> None:
    """``attn_fwd_host`` of the C ABI on CPU tensors (pinned or pageable); synchronous."""
    B, Hq, Hkv, Sq, Sk, D = _check_layout(q, k, v, o, lse, "cpu")
    dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream
    with torch.cuda.device(dev):
        st = load_library().attn_fwd_host(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                          None if lse is None else lse.data_ptr(),
                                          B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), float(scale), stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_fwd_host")


def attn_release_host_staging() -> None:
    st = load_library().attn_release_host_staging()
    if st != ATTN_OK:
        raise AttnError(st, "attn_release_host_staging")


def attn_set_option(name: str, value: int) -> None:
    st = load_library().attn_set_option(name.encode(), int(value))
    if st != ATTN_OK:
        raise AttnError(st, f"attn_set_option({name}={value})")


OPTION_DEFAULTS = {"scheduler": 2, "max_ctas": 0, "rescale_threshold": 8, "split_p": 1, "overlap_epilogue": 1,
                   "gqa_pack": 1, "host_pipeline": 1, "kernel": 0}


def attn_get_option(name: str) -> int:
    value = ctypes.c_int(0)
    st = load_library().attn_get_option(name.encode(), ctypes.byref(value))
    if st != ATTN_OK:
        raise AttnError(st, f"attn_get_option({name})")
    return value.value


def attn_plan(B, Hq, Hkv, Sq, Sk, D, causal, sm_count) -> dict:
    """Host-only: the tile scheduler's decomposition of a problem (see include/attn.h)."""
    out = (ctypes.c_int * 6)()
    st = load_library().attn_plan(B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), sm_count, out)
    if st != ATTN_OK:
        raise AttnError(st, "attn_plan")
    keys = ("n_work", "pair_heads", "items_per_group", "n_q_tiles", "n_kv_blocks", "ctas")
    return dict(zip(keys, list(out)))


def attn_plan_item(B, Hq, Hkv, Sq, Sk, D, causal, w) -> dict:
    """Host-only: work item ``w`` in launch order (see include/attn.h)."""
    out = (ctypes.c_int * 8)()
    st = load_library().attn_plan_item(B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), w, out)
    if st != ATTN_OK:
        raise AttnError(st, "attn_plan_item")
    keys = ("b", "hkv", "hq0", "hq1", "row0_0", "row0_1", "n_blocks_0", "n_blocks_1")
    return dict(zip(keys, list(out)))


def attn_plan_item_pair(B, Hq, Hkv, Sq, Sk, D, causal, w, rank) -> dict:
    """Host-only: work item ``w`` of the CTA-pair kernel as CTA ``rank`` of the pair sees it."""
    out = (ctypes.c_int * 8)()
    st = load_library().attn_plan_item_pair(B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), w, rank, out)
    if st != ATTN_OK:
        raise AttnError(st, "attn_plan_item_pair")
    keys = ("b", "hkv", "hq0", "hq1", "row0_0", "row0_1", "n_blocks_0", "n_blocks_1")
    return dict(zip(keys, list(out)))


def attn_merge_status(o1, lse1, o2, lse2, o, lse, stream=None) -> int:
    """Calls ``attn_merge`` on CUDA tensors and returns its raw status code."""
    for name, t in (("o1", o1), ("o2", o2), ("o", o)):
        if t.dtype != torch.bfloat16 or t.dim() != 4 or not t.is_contiguous() or t.device.type != "cuda":
            raise ValueError(f"{name} must be a contiguous 4-D bfloat16 cuda tensor [B, Sq, Hq, D]")
    B, Sq, Hq, D = o1.shape
    if o2.shape != o1.shape or o.shape != o1.shape:
        raise ValueError("inconsistent o shapes")
    for name, t in (("lse1", lse1), ("lse2", lse2), ("lse", lse)):
        if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != (B, Hq, Sq) or t.device.type != "cuda":
            raise ValueError(f"{name} must be a contiguous float32 cuda tensor [B, Hq, Sq]")
    if stream is None:
        stream = torch.cuda.current_stream(o1.device).cuda_stream
    with torch.cuda.device(o1.device):
        return load_library().attn_merge(o1.data_ptr(), lse1.data_ptr(), o2.data_ptr(), lse2.data_ptr(),
                                         o.data_ptr(), lse.data_ptr(), B, Hq, Sq, D, stream)


def attn_merge(o1, lse1, o2, lse2, o, lse, stream=None) -> None:
    """``attn_merge`` of the C ABI: attention over the union of two disjoint key sets from the
    two partial results (o_i BF16 [B,Sq,Hq,D], lse_i FP32 [B,Hq,Sq]).  ``o`` may be ``o1`` or
    ``o2``; ``lse`` must be a separate tensor."""
    st = attn_merge_status(o1, lse1, o2, lse2, o, lse, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_merge")


def attn_merge_n(o_parts, lse_parts, o, lse, stream=None) -> None:
    """``attn_merge_n`` of the C ABI: o_parts BF16 [n,B,Sq,Hq,D] and lse_parts FP32 [n,B,Hq,Sq]
    (contiguous) -> o [B,Sq,Hq,D], lse [B,Hq,Sq] (lse may be None)."""
    if o_parts.dtype != torch.bfloat16 or o_parts.dim() != 5 or not o_parts.is_contiguous() or not o_parts.is_cuda:
        raise ValueError("o_parts must be a contiguous bfloat16 cuda tensor [n, B, Sq, Hq, D]")
    n, B, Sq, Hq, D = o_parts.shape
    if lse_parts.dtype != torch.float32 or not lse_parts.is_contiguous() or tuple(lse_parts.shape) != (n, B, Hq, Sq):
        raise ValueError("lse_parts must be a contiguous float32 tensor [n, B, Hq, Sq]")
    if o.dtype != torch.bfloat16 or not o.is_contiguous() or tuple(o.shape) != (B, Sq, Hq, D):
        raise ValueError("o must be a contiguous bfloat16 tensor [B, Sq, Hq, D]")
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous() or tuple(lse.shape) != (B, Hq, Sq)):
        raise ValueError("lse must be a contiguous float32 tensor [B, Hq, Sq]")
    if stream is None:
        stream = torch.cuda.current_stream(o.device).cuda_stream
    with torch.cuda.device(o.device):
        st = load_library().attn_merge_n(o_parts.data_ptr(), lse_parts.data_ptr(), n, o.data_ptr(),
                                         None if lse is None else lse.data_ptr(), B, Hq, Sq, D, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_merge_n")


def attn_splitkv_workspace_bytes(B: int, Hq: int, Sq: int, D: int, n_splits: int) -> int:
    return int(load_library().attn_splitkv_workspace_bytes(B, Hq, Sq, D, n_splits))


def attn_fwd_splitkv_status(q, k, v, o, lse, causal: bool, scale: float, n_splits: int, workspace=None,
                            stream=None) -> int:
    """Calls ``attn_fwd_splitkv``; ``workspace`` is a uint8 cuda tensor (allocated here when None)."""
    B, Hq, Hkv, Sq, Sk, D = _check_layout(q, k, v, o, lse, "cuda")
    need = attn_splitkv_workspace_bytes(B, Hq, Sq, D, n_splits) if 1 <= n_splits <= 64 else 0
    if workspace is None and need > 0:
        workspace = _new_workspace(q, need, stream)
    if stream is None:
        stream = torch.cuda.current_stream(q.device).cuda_stream
    with torch.cuda.device(q.device):
        return load_library().attn_fwd_splitkv(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                               None if lse is None else lse.data_ptr(), B, Hq, Hkv, Sq, Sk, D,
                                               int(bool(causal)), float(scale), int(n_splits),
                                               None if workspace is None else workspace.data_ptr(),
                                               0 if workspace is None else workspace.numel(), stream)


def attn_fwd_splitkv(q, k, v, o, lse, causal: bool, scale: float, n_splits: int, workspace=None, stream=None) -> None:
    """``attn_fwd_splitkv`` of the C ABI: the forward with the key sequence cut into up to
    ``n_splits`` ranges that run concurrently and are merged (for few query rows, many keys)."""
    st = attn_fwd_splitkv_status(q, k, v, o, lse, causal, scale, n_splits, workspace, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_fwd_splitkv")


def attn_bwd_workspace_bytes(B: int, Hq: int, Hkv: int, Sq: int, Sk: int, D: int, causal: bool) -> int:
    return int(load_library().attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Sk, D, int(bool(causal))))


def attn_bwd_plan(B, Hq, Hkv, Sq, Sk, D, causal) -> dict:
    """Host-only: how ``attn_bwd`` cuts a problem into work items (see include/attn.h)."""
    out = (ctypes.c_int * 9)()
    st = load_library().attn_bwd_plan(B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), out)
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd_plan")
    keys = ("n_items", "q_heads", "pack_log2", "n_q_tiles", "n_k_tiles", "key_splits", "query_splits", "run", "run_extra")
    return dict(zip(keys, list(out)))


def attn_bwd_plan_item(B, Hq, Hkv, Sq, Sk, D, causal, w) -> dict:
    """Host-only: work item ``w`` of ``attn_bwd`` in launch order (see include/attn.h)."""
    out = (ctypes.c_int * 9)()
    st = load_library().attn_bwd_plan_item(B, Hq, Hkv, Sq, Sk, D, int(bool(causal)), w, out)
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd_plan_item")
    return dict(zip(("keys", "b", "head", "row0", "first", "per_head", "t0", "n", "split"), list(out)))


def _raw_stream(dev, stream):
    """cudaStream_t of ``stream``, or of torch's current stream on ``dev`` when None."""
    return torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream


def _torch_stream(dev, stream):
    """torch's stream for what the C ABI takes as one: a cudaStream_t as a number or a ``c_void_p``, or a ``torch.cuda.Stream``."""
    handle = getattr(stream, "cuda_stream", stream)
    if isinstance(handle, ctypes.c_void_p):
        handle = handle.value or 0
    # 0 and 1 (cudaStreamLegacy) both name the default stream; an ExternalStream of them would not
    return torch.cuda.default_stream(dev) if handle in (0, 1) else torch.cuda.ExternalStream(handle, device=dev)


def _new_workspace(like, n_bytes: int, stream):
    """A workspace that is dropped when the call returns, out of memory of the stream that the call goes to: memory of
    torch's current stream may still be in use by what is queued there, and may be handed out again before ``stream`` is
    done with it."""
    if stream is None:
        return like.new_empty(n_bytes, dtype=torch.uint8)
    target = _torch_stream(like.device, stream)
    with torch.cuda.stream(target):
        workspace = like.new_empty(n_bytes, dtype=torch.uint8)
    # torch's own allocator keeps memory by stream and has nothing to record here; one plugged into torch need not
    workspace.record_stream(target)
    return workspace


def _on_device(dev, fn, *args):
    """fn(*args) with ``dev`` current; switching devices costs more than a call that need not."""
    if torch.cuda.current_device() == dev.index:
        return fn(*args)
    with torch.cuda.device(dev):
        return fn(*args)


def _refuse_bwd(tensors, shape, kv_shape, strided):
    """Names the tensor that is not what ``_bwd_status`` needs."""
    dev = tensors[1].device
    for name, t in zip(("dout", "q", "k", "v", "o", "dq", "dk", "dv"), tensors):
        want = kv_shape if name in ("k", "v", "dk", "dv") else shape
        if t.dtype is not _BF16 or t.device != dev or t.shape != want or not (t.stride(3) == 1 if strided else t.is_contiguous()):
            layout = "with a contiguous last axis" if strided else "that is contiguous"
            raise ValueError(f"{name} must be a bfloat16 tensor {layout}, of the shape [B, S, H, D] of "
                             f"{'k' if want is kv_shape else 'q'}, on q's device")


def _bwd_status(dout, q, k, v, o, lse, dq, dk, dv, causal, scale, dlse, workspace, stream, strided, made_here=False):
    """``made_here``: dq, dk, dv are new contiguous tensors of the right kind."""
    dev, shape, kv_shape = q.device, q.shape, k.shape
    if len(shape) != 4 or len(kv_shape) != 4 or dev.type != "cuda" or kv_shape[0] != shape[0] or kv_shape[3] != shape[3]:
        raise ValueError("q and k must be 4-D cuda tensors [B, S, H, D] of one batch size and head dimension")
    # one expression for the usual call: these checks are a good part of its time
    if not (q.dtype is _BF16 and k.dtype is _BF16 and v.dtype is _BF16 and o.dtype is _BF16 and dout.dtype is _BF16
            and v.shape == kv_shape and o.shape == shape and dout.shape == shape
            and k.device == dev and v.device == dev and o.device == dev and dout.device == dev):
        _refuse_bwd((dout, q, k, v, o), shape, kv_shape, strided)
    if not made_here:
        _refuse_bwd((dout, q, k, v, o, dq, dk, dv), shape, kv_shape, strided)
    elif strided and not (q.stride(3) == k.stride(3) == v.stride(3) == o.stride(3) == dout.stride(3) == 1):
        _refuse_bwd((dout, q, k, v, o), shape, kv_shape, strided)
    B, Sq, Hq, D = shape
    _, Sk, Hkv, _ = kv_shape
    for name, t in (("lse", lse),) if dlse is None else (("lse", lse), ("dlse", dlse)):
        if t is None or t.dtype is not torch.float32 or not t.is_contiguous() or t.shape != (B, Hq, Sq) or t.device != dev:
            raise ValueError(f"{name} must be a contiguous float32 tensor [B, Hq, Sq] on q's device")
    lib = load_library()
    causal = 1 if causal else 0
    if workspace is None:
        workspace = _new_workspace(q, max(lib.attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Sk, D, causal), 16), stream)
    elif not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError("workspace must be a contiguous tensor on q's device")
    args = (dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
            None if dlse is None else dlse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, Hq, Hkv, Sq, Sk, D)
    tail = (causal, float(scale), workspace.data_ptr(), workspace.nbytes, _raw_stream(dev, stream))
    if strided:
        dense, kv_dense = _LL3(Sq * Hq * D, Hq * D, D), _LL3(Sk * Hkv * D, Hkv * D, D)
        return _on_device(dev, lib.attn_bwd_strided, *args,
                          *[(kv_dense if i in (2, 3, 6, 7) else dense) if t.is_contiguous() else _strides3(t)
                            for i, t in enumerate((dout, q, k, v, o, dq, dk, dv))], *tail)
    return _on_device(dev, lib.attn_bwd, *args, *tail)


def attn_bwd_status(dout, q, k, v, o, lse, dq, dk, dv, causal: bool, scale: float, dlse=None, workspace=None,
                    stream=None) -> int:
    """Calls ``attn_bwd`` on CUDA tensors and returns its raw status code.  ``workspace`` is a contiguous
    cuda tensor (allocated here when None)."""
    return _bwd_status(dout, q, k, v, o, lse, dq, dk, dv, causal, scale, dlse, workspace, stream, False)


def attn_bwd(dout, q, k, v, o, lse, dq, dk, dv, causal: bool, scale: float, dlse=None, workspace=None, stream=None) -> None:
    """``attn_bwd`` of the C ABI: the gradients dq, dk, dv (written) of ``attn_fwd`` from its inputs q, k, v, its
    results o, lse and the gradients dout (and dlse, may be None) with respect to them."""
    st = attn_bwd_status(dout, q, k, v, o, lse, dq, dk, dv, causal, scale, dlse, workspace, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd")


def attn_bwd_strided_status(dout, q, k, v, o, lse, dq, dk, dv, causal: bool, scale: float, dlse=None, workspace=None,
                            stream=None) -> int:
    """Calls ``attn_bwd_strided`` on CUDA tensors of shape [B, S, H, D] with arbitrary batch, sequence and
    head strides (the head dimension must be contiguous); returns the raw status."""
    return _bwd_status(dout, q, k, v, o, lse, dq, dk, dv, causal, scale, dlse, workspace, stream, True)


def attn_bwd_strided(dout, q, k, v, o, lse, dq, dk, dv, causal: bool, scale: float, dlse=None, workspace=None,
                     stream=None) -> None:
    """``attn_bwd_strided`` of the C ABI: ``attn_bwd`` on views (see ``attn_fwd_strided``)."""
    st = attn_bwd_strided_status(dout, q, k, v, o, lse, dq, dk, dv, causal, scale, dlse, workspace, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd_strided")


def _rope_args(q, k, q_weight, k_weight, cos, sin, positions, others):
    """Checks the tensors and marshals what both directions share: (leading arguments, sizes).  ``others``: pairs of
    tensors shaped like (q, k)."""
    dev, shape, kv_shape = q.device, q.shape, k.shape
    if dev.type != "cuda" or len(shape) != 4 or len(kv_shape) != 4 or kv_shape[:2] != shape[:2] or kv_shape[3] != shape[3]:
        raise ValueError("q and k must be cuda tensors [B, S, Hq, D] and [B, S, Hkv, D]")
    for x, y in ((q, k), *others):
        if not (x.dtype is _BF16 and y.dtype is _BF16 and (x is q or x.shape == shape and y.shape == kv_shape)
                and x.stride(3) == 1 and y.stride(3) == 1 and x.device == dev and y.device == dev):
            raise ValueError("queries, keys, their outputs and gradients must be bfloat16 tensors [B, S, H, D] of q's and "
                             "k's shapes with a contiguous last axis, all on q's device")
    B, S, Hq, D = shape
    weight_type = 0
    for w in (q_weight, k_weight):
        if w is None:
            continue
        weight_type = 1 if w.dtype is _BF16 else 0
        if not (weight_type or w.dtype is torch.float32) or w.shape != (D,) or not w.is_contiguous() or w.device != dev:
            raise ValueError("q_weight and k_weight must be contiguous float32 or bfloat16 tensors [D] on q's device")
    if q_weight is not None and k_weight is not None and q_weight.dtype is not k_weight.dtype:
        raise ValueError("q_weight and k_weight must have one type")
    table = cos.shape
    if not (len(table) == 2 and cos.dtype is torch.float32 and sin.dtype is torch.float32 and sin.shape == table
            and cos.is_contiguous() and sin.is_contiguous() and cos.device == dev and sin.device == dev):
        raise ValueError("cos and sin must be contiguous float32 tensors [positions, rot_dim / 2] on q's device")
    pos_ptr, pos_type, pos_strides = None, 0, None
    if positions is not None:
        pos_type = 1 if positions.dtype is torch.int64 else 0
        if not (pos_type or positions.dtype is torch.int32) or positions.device != dev or positions.shape not in ((B, S), (S,)):
            raise ValueError("positions must be an int32 or int64 tensor [B, S] or [S] on q's device")
        pos_ptr = positions.data_ptr()
        if positions.dim() == 1:
            pos_strides = (ctypes.c_longlong * 2)(0, positions.stride(0))
        elif not positions.is_contiguous():
            pos_strides = (ctypes.c_longlong * 2)(*positions.stride())
    return (q.data_ptr(), k.data_ptr(), None if q_weight is None else q_weight.data_ptr(),
            None if k_weight is None else k_weight.data_ptr(), weight_type, cos.data_ptr(), sin.data_ptr(), pos_ptr, pos_type,
            pos_strides), (B, S, Hq, kv_shape[2], D, 2 * table[1], table[0])


def _strides3_or_none(t):
    return None if t.is_contiguous() else _strides3(t)


def attn_qk_norm_rope_status(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions=None, eps: float = 1e-6,
                             interleaved: bool = False, stream=None) -> int:
    """Calls ``attn_qk_norm_rope`` on CUDA tensors and returns its raw status code."""
    return _rope_status(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions, eps, interleaved, stream,
                        ((q_out, k_out),))


def _rope_status(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions, eps, interleaved, stream, check):
    lead, sizes = _rope_args(q, k, q_weight, k_weight, cos, sin, positions, check)
    return _on_device(q.device, load_library().attn_qk_norm_rope, *lead, q_out.data_ptr(), k_out.data_ptr(), *sizes,
                      1 if interleaved else 0, float(eps), _strides3_or_none(q), _strides3_or_none(k),
                      _strides3_or_none(q_out), _strides3_or_none(k_out),
                      _raw_stream(q.device, stream))


def attn_qk_norm_rope(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions=None, eps: float = 1e-6,
                      interleaved: bool = False, stream=None) -> None:
    """``attn_qk_norm_rope`` of the C ABI: per-head root-mean-square norm and rotation of q [B,S,Hq,D] and k [B,S,Hkv,D]
    into q_out and k_out (which may be q and k, or views of a cache).  Tables ``cos``, ``sin`` [positions, rot_dim / 2],
    ``positions`` [B,S] or [S] (None: 0 .. S-1), weights [D] or None."""
    st = attn_qk_norm_rope_status(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions, eps, interleaved, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_qk_norm_rope")


def attn_qk_norm_rope_bwd_workspace_bytes() -> int:
    return int(load_library().attn_qk_norm_rope_bwd_workspace_bytes())


def attn_qk_norm_rope_bwd_status(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight,
                                 positions=None, eps: float = 1e-6, interleaved: bool = False, workspace=None,
                                 stream=None) -> int:
    """Calls ``attn_qk_norm_rope_bwd``; ``workspace`` is a contiguous cuda tensor (allocated here when None)."""
    return _rope_bwd_status(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight, positions, eps,
                            interleaved, workspace, stream, False)


def _rope_bwd_status(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight, positions, eps,
                     interleaved, workspace, stream, made_here):
    """``made_here``: the outputs are new contiguous tensors of the right kind."""
    lead, sizes = _rope_args(q, k, q_weight, k_weight, cos, sin, positions,
                             ((dq_out, dk_out),) if made_here else ((dq_out, dk_out), (dq, dk)))
    dev = q.device
    for name, t in () if made_here else (("dq_weight", dq_weight), ("dk_weight", dk_weight)):
        if t is not None and (t.dtype is not torch.float32 or t.shape != q.shape[3:] or not t.is_contiguous()
                              or t.device != dev):
            raise ValueError(f"{name} must be a contiguous float32 tensor [D] on q's device")
    lib = load_library()
    if workspace is None:
        if dq_weight is not None or dk_weight is not None:
            workspace = _new_workspace(q, lib.attn_qk_norm_rope_bwd_workspace_bytes(), stream)
    elif not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError("workspace must be a contiguous tensor on q's device")
    return _on_device(dev, lib.attn_qk_norm_rope_bwd, dq_out.data_ptr(), dk_out.data_ptr(), *lead, dq.data_ptr(),
                      dk.data_ptr(), None if dq_weight is None else dq_weight.data_ptr(),
                      None if dk_weight is None else dk_weight.data_ptr(), *sizes, int(bool(interleaved)), float(eps),
                      *[_strides3_or_none(t) for t in (dq_out, dk_out, q, k, dq, dk)],
                      None if workspace is None else workspace.data_ptr(),
                      0 if workspace is None else workspace.nbytes, _raw_stream(dev, stream))


def attn_qk_norm_rope_bwd(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight, positions=None,
                          eps: float = 1e-6, interleaved: bool = False, workspace=None, stream=None) -> None:
    """``attn_qk_norm_rope_bwd`` of the C ABI: gradients of ``attn_qk_norm_rope`` with respect to q, k (BF16) and both weights
    (FP32 [D], each may be None)."""
    st = attn_qk_norm_rope_bwd_status(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight,
                                      positions, eps, interleaved, workspace, stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_qk_norm_rope_bwd")


def attn_selftest_wait_timeout(limit_ms: int, device=0, stream=None) -> None:
    """Launches the bounded-wait self-test (see include/attn.h); read the outcome with
    ``attn_last_device_status``."""
    dev = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream
    with torch.cuda.device(dev):
        st = load_library().attn_selftest_wait_timeout(int(limit_ms), stream)
    if st != ATTN_OK:
        raise AttnError(st, "attn_selftest_wait_timeout")


def attn_status_str(status: int) -> str:
    return load_library().attn_status_str(int(status)).decode()


def attn_version() -> int:
    return load_library().attn_version()


def attn_last_launch_clock():
    """(SM MHz, milliseconds) of the most recent launch of the default kernel on the current
    device, or None when there has been none (see include/attn.h)."""
    mhz, ms = ctypes.c_double(0.0), ctypes.c_double(0.0)
    st = load_library().attn_last_launch_clock(ctypes.byref(mhz), ctypes.byref(ms))
    if st == 3:
        return None
    if st != ATTN_OK:
        raise AttnError(st, "attn_last_launch_clock")
    return mhz.value, ms.value


def attn_launch_clocks(max_n: int = 64):
    """SM MHz of the most recent launches on the current device, newest first (at most 64;
    see include/attn.h).  Synchronises the device."""
    buf = (ctypes.c_double * max_n)()
    n = ctypes.c_int(0)
    st = load_library().attn_launch_clocks(buf, int(max_n), ctypes.byref(n))
    if st != ATTN_OK:
        raise AttnError(st, "attn_launch_clocks")
    return [buf[i] for i in range(n.value)]


def attn_last_device_status():
    """(status, code, detail) -- synchronises the device."""
    code, detail = ctypes.c_int(0), ctypes.c_int(0)
    st = load_library().attn_last_device_status(ctypes.byref(code), ctypes.byref(detail))
    return st, code.value, detail.value


def attention_forward(q, k, v, causal: bool = False, scale: float | None = None, return_lse: bool = True):
    """Convenience wrapper: allocates o (and lse) with torch and calls ``attn_fwd``.  Not part of autograd's graph: its
    gradients are ``attention_backward``'s."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    o = torch.empty_like(q)
    lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device) \
        if return_lse else None
    attn_fwd(q, k, v, o, lse, causal, scale)
    return (o, lse) if return_lse else o


def _ordered(grad):
    """A gradient as it comes: one that is expanded (of a sum or a mean) or turned is copied into an order of its own."""
    if grad.dim() == 4 and not grad.is_contiguous() and (grad.stride(3) != 1 or 0 in grad.stride()):
        return grad.contiguous()
    return grad


def _new_like(t):
    return torch.empty_like(t) if t.is_contiguous() else torch.empty_like(t, memory_format=torch.contiguous_format)


def attention_backward(dout, q, k, v, o, lse, causal: bool = False, scale: float | None = None, dlse=None):
    """Gradients (dq, dk, dv) of ``attention_forward(q, k, v, causal, scale)`` from its results ``o``, ``lse`` and the
    gradient ``dout`` with respect to ``o`` (and ``dlse`` with respect to ``lse``).  Inputs may be views as in
    ``attn_fwd_strided``; a ``dout`` without an order of its own (the expanded gradient of a sum), and a ``dlse`` that is
    not contiguous, is copied first; ``lse`` is contiguous, as the forward pass leaves it.
    The gradients are new contiguous tensors."""
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    dout = _ordered(dout)
    if dlse is not None and not dlse.is_contiguous():
        dlse = dlse.contiguous()
    dq, dk, dv = _new_like(q), _new_like(k), _new_like(v)
    strided = not (dout.is_contiguous() and q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and o.is_contiguous())
    st = _bwd_status(dout, q, k, v, o, lse, dq, dk, dv, causal, scale, dlse, None, None, strided, True)
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd_strided" if strided else "attn_bwd")
    return dq, dk, dv


def qk_norm_rope(q, k, q_weight, k_weight, cos, sin, positions=None, eps: float = 1e-6, interleaved: bool = False):
    """Convenience wrapper: the normed and rotated queries and keys as new contiguous tensors (see ``attn_qk_norm_rope``),
    ready for ``attention_forward``.  Not part of autograd's graph (``qk_norm_rope_backward``)."""
    q_out, k_out = _new_like(q), _new_like(k)
    st = _rope_status(q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions, eps, interleaved, None, ())
    if st != ATTN_OK:
        raise AttnError(st, "attn_qk_norm_rope")
    return q_out, k_out


def qk_norm_rope_backward(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, positions=None, eps: float = 1e-6,
                          interleaved: bool = False):
    """Gradients (dq, dk, dq_weight, dk_weight) of ``qk_norm_rope``; a weight that is None has the gradient None."""
    dq_out, dk_out = _ordered(dq_out), _ordered(dk_out)
    dq, dk = _new_like(q), _new_like(k)
    dq_weight = None if q_weight is None else torch.empty_like(q_weight, dtype=torch.float32)
    dk_weight = None if k_weight is None else torch.empty_like(k_weight, dtype=torch.float32)
    st = _rope_bwd_status(dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight, positions, eps,
                          interleaved, None, None, True)
    if st != ATTN_OK:
        raise AttnError(st, "attn_qk_norm_rope_bwd")
    return dq, dk, dq_weight, dk_weight
