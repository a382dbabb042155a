"""ctypes binding of libcorm.so: same names and argument order as include/corm.h.

Argument marshalling only -- every step of the path runs in the HIP kernels.
torch is used for device memory and streams: tensors are passed as their
``data_ptr()``.  There is no CPU fallback: if the library has not been built
(``python -c "import __graft_entry__ as g; g.build()"``) loading raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import operator
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcorm.so")

CORM_F32, CORM_BF16, CORM_BIT, CORM_I8, CORM_E4M3 = 0, 1, 2, 3, 4
CORM_OK, CORM_EINVAL, CORM_EUNSUPPORTED, CORM_ECAPACITY, CORM_EHIP = 0, -1, -2, -3, -4
CORM_DEV_UNIT_FULL, CORM_DEV_BAD_STEP, CORM_DEV_BAD_LENS, CORM_DEV_BAD_BLOCK, CORM_DEV_BAD_PAGE = 1, 2, 4, 8, 16
CORM_HALVES, CORM_NEIGHBOURS = 0, 1
BLOCK = 64   # slots per block of the 8-bit cache and of the calls that choose blocks
CORM_STATIC_SCRATCH_BYTES = 40 << 20

EXPORTS = ("corm_version", "corm_strerror", "corm_workspace_bytes", "corm_workspace_init", "corm_append",
           "corm_decode_attend", "corm_decode_attend_static", "corm_evict_mask", "corm_evict_mask_summary", "corm_row_density", "corm_compact",
           "corm_decode_step", "corm_step_attend", "corm_step_evict", "corm_decode_step_lazy", "corm_prefill_seed",
           "corm_selected_path", "corm_threshold", "corm_blocks_workspace_bytes", "corm_q8_append", "corm_q8_attend",
           "corm_block_bounds", "corm_block_select", "corm_block_attend", "corm_decode_attend_weigh", "corm_evict_mask_weight",
           "corm_rotate", "corm_paged_append", "corm_paged_read", "corm_paged_workspace_bytes", "corm_paged_attend")


class corm_desc(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("Lcap", ctypes.c_int32), ("Tcap", ctypes.c_int32), ("w", ctypes.c_int32), ("r", ctypes.c_int32),
                ("kv_dtype", ctypes.c_int32), ("score_dtype", ctypes.c_int32),
                ("thr_scale", ctypes.c_float), ("sm_scale", ctypes.c_float)]


class corm_launch_opts(ctypes.Structure):
    _fields_ = [("path", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("attend_start_event", ctypes.c_void_p), ("attend_stop_event", ctypes.c_void_p)]


class corm_rows(ctypes.Structure):
    # (the header's arrays of three strides one by one: arrays take longer to fill than a launch does to be queued)
    _fields_ = [(x, ctypes.c_void_p) for x in "qkv"] + [(f"{x}_{of}", ctypes.c_int64) for x in "qkv" for of in ("seq", "token", "head")]


class corm_rotation(ctypes.Structure):
    _fields_ = [("rot", ctypes.c_int32), ("pairing", ctypes.c_int32), ("axes", ctypes.c_int32), ("in_turn", ctypes.c_int32),
                ("section", ctypes.c_int32 * 4), ("eps", ctypes.c_float), ("gain", ctypes.c_float), ("inv_freq", ctypes.c_void_p),
                ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p)]


class corm_pages(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("page", ctypes.c_int32), ("npages", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("table_heads", ctypes.c_int32), ("reserved", ctypes.c_int32), ("K", ctypes.c_void_p), ("V", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("table", ctypes.c_void_p)]


class CormError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Load libcorm.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (__graft_entry__.build()); "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t
        dp = ctypes.POINTER(corm_desc)
        op = ctypes.POINTER(corm_launch_opts)
        L.corm_version.restype = ctypes.c_int
        L.corm_version.argtypes = []
        L.corm_strerror.restype = ctypes.c_char_p
        L.corm_strerror.argtypes = [ctypes.c_int]
        L.corm_workspace_bytes.argtypes = [dp, ctypes.POINTER(ctypes.c_size_t)]
        L.corm_workspace_init.argtypes = [dp, vp, sz, vp]
        L.corm_append.argtypes = [dp, vp, vp, i32p, i32p, i32p, vp, vp, i32p, i32p, vp]
        L.corm_decode_attend.argtypes = [dp, vp, vp, vp, i32p, i32p, i32p, vp, i32p, vp, vp, sz, i32p, op, vp]
        L.corm_decode_attend_static.argtypes = [dp, vp, vp, vp, i32p, i32p, i32p, vp, i32p, vp, i32p, op, vp]
        L.corm_evict_mask.argtypes = [dp, vp, i32p, i32p, i32p, i32p, vp, vp]
        L.corm_evict_mask_summary.argtypes = [dp, i32p, i32p, i32p, i32p, vp, vp]
        L.corm_row_density.argtypes = [dp, vp, i32p, i32p, i32p, vp, vp]
        L.corm_compact.argtypes = [dp, vp, vp, i32p, i32p, i32p, vp, i32p, vp, sz, vp]
        L.corm_step_attend.argtypes = [dp, vp, vp, vp, vp, vp, i32p, i32p, i32p, i32p, i32p, vp, vp, vp, vp, sz,
                                       i32p, op, vp]
        L.corm_step_evict.argtypes = [dp, vp, vp, i32p, i32p, i32p, i32p, vp, sz, vp]
        L.corm_selected_path.argtypes = [dp, op]
        L.corm_decode_step.argtypes = [dp, vp, vp, vp, vp, vp, i32p, i32p, i32p, i32p, i32p, vp, vp, vp, i32p,
                                       vp, sz, i32p, op, vp]
        L.corm_decode_step_lazy.argtypes = [dp, vp, vp, vp, vp, vp, i32p, vp, i32p, i32p, i32p, i32p, vp, vp, vp,
                                            i32p, ctypes.c_int32, ctypes.c_int32, vp, sz, i32p, op, vp]
        L.corm_prefill_seed.argtypes = [dp, vp, ctypes.c_int32, vp, vp, i32p, i32p, i32p, i32p, i32p, vp, vp, i32p,
                                        vp, sz, i32p, vp]
        i32 = ctypes.c_int32
        L.corm_blocks_workspace_bytes.argtypes = [dp, ctypes.POINTER(ctypes.c_size_t)]
        L.corm_q8_append.argtypes = [dp, i32, vp, vp, i32, i32p, vp, vp, vp, vp, vp, vp, i32p, i32p, vp, i32p, vp]
        L.corm_q8_attend.argtypes = [dp, i32, vp, vp, vp, vp, vp, vp, vp, i32p, i32p, i32, vp, vp, sz, i32p, vp]
        L.corm_block_bounds.argtypes = [dp, vp, i32p, i32, vp, vp]
        L.corm_block_select.argtypes = [dp, vp, vp, i32p, i32, i32, i32p, vp, sz, vp]
        L.corm_block_attend.argtypes = [dp, vp, vp, vp, i32p, i32p, i32, vp, vp, sz, i32p, vp]
        L.corm_decode_attend_weigh.argtypes = [dp, vp, vp, vp, i32p, vp, vp, vp, vp, sz, i32p, op, vp]
        L.corm_evict_mask_weight.argtypes = [dp, vp, i32p, i32, vp, vp, sz, vp]
        rp, tp, pp = (ctypes.POINTER(c) for c in (corm_rows, corm_rotation, corm_pages))
        L.corm_rotate.argtypes = [dp, rp, tp, i32p, i32, i32p, vp, vp, vp, vp]
        L.corm_paged_append.argtypes = [dp, pp, rp, tp, i32p, i32, i32p, vp, i32p, i32p, i32p, vp]
        L.corm_paged_read.argtypes = [dp, pp, i32p, i32, vp, vp, i32p, vp]
        L.corm_paged_workspace_bytes.argtypes = [dp, ctypes.POINTER(ctypes.c_size_t)]
        L.corm_paged_attend.argtypes = [dp, pp, vp, i32p, vp, vp, sz, i32p, vp]
        L.corm_threshold.argtypes = [ctypes.c_float, i32p, ctypes.c_int32, vp, vp]
        for name in EXPORTS:
            if name not in ("corm_version", "corm_strerror"):
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().corm_strerror(code).decode()


def _ptr(x) -> Optional[int]:
    """Device (or raw integer) pointer of an argument; None stays NULL."""
    if x is None:
        return None
    if isinstance(x, torch.Tensor):
        return x.data_ptr()
    return int(x)


# The current stream's handle alone: building a Stream object takes longer than a launch.  Not a documented entry of
# torch, so a build without it takes the documented one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else None
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _as_current(stream):
    """For torch's own operations beside a call that is given `stream`."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))


def _capturing(stream) -> bool:
    if not torch.cuda.is_initialized():
        return False
    with _as_current(stream):
        return torch.cuda.is_current_stream_capturing()


# Launch options of the attend / step wrappers below when a call passes none: a setting of this BINDING (the
# library itself keeps no such state), so that a test fixture or the benchmark can route every call of a
# run through one launch path.
_default_path = 0


def set_default_path(path: int) -> None:
    """0 = by shape, 1 = split kernels, 2 = one workgroup per unit, 3 = split kernels without MFMA."""
    global _default_path
    if path not in (0, 1, 2, 3):
        raise ValueError("path must be 0..3")
    _default_path = path


def make_opts(path: Optional[int] = None, attend_events=None) -> corm_launch_opts:
    """attend_events: (start, stop) raw hipEvent_t handles (ints), recorded around the launch that streams K and V."""
    ev = attend_events or (None, None)
    return corm_launch_opts(_default_path if path is None else path, 0, ev[0], ev[1])


def _opts(opts):
    """The pointer argument for a call: the caller's options, or the binding's defaults (NULL when there are none)."""
    if opts is None:
        if _default_path == 0:
            return None
        opts = make_opts()
    return ctypes.byref(opts)


def _check(code: int, what: str) -> int:
    if code != CORM_OK:
        raise CormError(code, what)
    return code


def make_desc(B, Hq, Hkv, d, Lcap, Tcap, w, r, kv_dtype, score_dtype=None, thr_scale=1.0, sm_scale=0.0) -> corm_desc:
    def code(x):
        if x in (CORM_F32, CORM_BF16, CORM_BIT):
            return x
        return {"f32": CORM_F32, "bf16": CORM_BF16, "bit": CORM_BIT, torch.float32: CORM_F32,
                torch.bfloat16: CORM_BF16}[x]
    kv = code(kv_dtype)
    sc = kv if score_dtype is None else code(score_dtype)
    return corm_desc(B, Hq, Hkv, d, Lcap, Tcap, w, r, kv, sc, thr_scale, sm_scale)


# ---- the C entry points, one wrapper each (raise=False returns the status code instead)

def corm_version() -> int:
    return lib().corm_version()


def corm_workspace_bytes(desc: corm_desc, check=True) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().corm_workspace_bytes(ctypes.byref(desc), ctypes.byref(n))
    if check:
        _check(rc, "corm_workspace_bytes")
        return n.value
    return rc


def corm_workspace_init(desc, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    nbytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    rc = lib().corm_workspace_init(ctypes.byref(desc), _ptr(workspace), nbytes, _stream(stream))
    return _check(rc, "corm_workspace_init") if check else rc


def corm_append(desc, K, V, lens, pos, last_hit, k_new, v_new, t, status=None, stream=None, check=True) -> int:
    rc = lib().corm_append(ctypes.byref(desc), _ptr(K), _ptr(V), _ptr(lens), _ptr(pos), _ptr(last_hit),
                           _ptr(k_new), _ptr(v_new), _ptr(t), _ptr(status), _stream(stream))
    return _check(rc, "corm_append") if check else rc


def corm_decode_attend(desc, q, K, V, lens, pos, t, score_ring, last_hit, out, workspace, workspace_bytes=None,
                       status=None, stream=None, check=True, opts=None) -> int:
    nbytes = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    rc = lib().corm_decode_attend(ctypes.byref(desc), _ptr(q), _ptr(K), _ptr(V), _ptr(lens), _ptr(pos), _ptr(t),
                                  _ptr(score_ring), _ptr(last_hit), _ptr(out), _ptr(workspace), nbytes,
                                  _ptr(status), _opts(opts), _stream(stream))
    return _check(rc, "corm_decode_attend") if check else rc


def corm_decode_attend_static(desc, q, K, V, lens, pos, t, score_ring, last_hit, out, status=None, stream=None,
                              check=True, opts=None) -> int:
    rc = lib().corm_decode_attend_static(ctypes.byref(desc), _ptr(q), _ptr(K), _ptr(V), _ptr(lens), _ptr(pos),
                                         _ptr(t), _ptr(score_ring), _ptr(last_hit), _ptr(out), _ptr(status),
                                         _opts(opts), _stream(stream))
    return _check(rc, "corm_decode_attend_static") if check else rc


def corm_evict_mask(desc, score_ring, lens, pos, t, t_first, keep, stream=None, check=True) -> int:
    rc = lib().corm_evict_mask(ctypes.byref(desc), _ptr(score_ring), _ptr(lens), _ptr(pos), _ptr(t), _ptr(t_first),
                               _ptr(keep), _stream(stream))
    return _check(rc, "corm_evict_mask") if check else rc


def corm_evict_mask_summary(desc, last_hit, lens, t, t_first, keep, stream=None, check=True) -> int:
    rc = lib().corm_evict_mask_summary(ctypes.byref(desc), _ptr(last_hit), _ptr(lens), _ptr(t), _ptr(t_first),
                                       _ptr(keep), _stream(stream))
    return _check(rc, "corm_evict_mask_summary") if check else rc


def _nbytes(workspace, workspace_bytes):
    if workspace_bytes is not None:
        return workspace_bytes
    return 0 if workspace is None or not isinstance(workspace, torch.Tensor) else workspace.numel() * workspace.element_size()


def corm_compact(desc, K, V, pos, last_hit, lens, keep, kept_idx=None, workspace=None, workspace_bytes=None,
                 stream=None, check=True) -> int:
    rc = lib().corm_compact(ctypes.byref(desc), _ptr(K), _ptr(V), _ptr(pos), _ptr(last_hit), _ptr(lens), _ptr(keep),
                            _ptr(kept_idx), _ptr(workspace), _nbytes(workspace, workspace_bytes), _stream(stream))
    return _check(rc, "corm_compact") if check else rc


def corm_step_attend(desc, q, k_new, v_new, K, V, lens, pos, last_hit, t, t_first, score_ring, out, keep=None,
                     workspace=None, workspace_bytes=None, status=None, stream=None, check=True, opts=None) -> int:
    rc = lib().corm_step_attend(ctypes.byref(desc), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V), _ptr(lens),
                                _ptr(pos), _ptr(last_hit), _ptr(t), _ptr(t_first), _ptr(score_ring), _ptr(out),
                                _ptr(keep), _ptr(workspace), _nbytes(workspace, workspace_bytes), _ptr(status),
                                _opts(opts), _stream(stream))
    return _check(rc, "corm_step_attend") if check else rc


def corm_step_evict(desc, K, V, lens, pos, last_hit, kept_idx=None, workspace=None, workspace_bytes=None,
                    stream=None, check=True) -> int:
    rc = lib().corm_step_evict(ctypes.byref(desc), _ptr(K), _ptr(V), _ptr(lens), _ptr(pos), _ptr(last_hit),
                               _ptr(kept_idx), _ptr(workspace), _nbytes(workspace, workspace_bytes), _stream(stream))
    return _check(rc, "corm_step_evict") if check else rc


def corm_row_density(desc, score_ring, lens, pos, t, density, stream=None, check=True) -> int:
    rc = lib().corm_row_density(ctypes.byref(desc), _ptr(score_ring), _ptr(lens), _ptr(pos), _ptr(t), _ptr(density),
                                _stream(stream))
    return _check(rc, "corm_row_density") if check else rc


def corm_selected_path(desc, opts=None, check=True) -> int:
    rc = lib().corm_selected_path(ctypes.byref(desc), _opts(opts))
    if rc < 0 and check:
        raise CormError(rc, "corm_selected_path")
    return rc


def corm_decode_step(desc, q, k_new, v_new, K, V, lens, pos, last_hit, t, t_first, score_ring, out, keep=None,
                     kept_idx=None, workspace=None, workspace_bytes=None, status=None, stream=None, check=True,
                     opts=None) -> int:
    nbytes = workspace_bytes
    if nbytes is None:
        nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().corm_decode_step(ctypes.byref(desc), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V), _ptr(lens),
                                _ptr(pos), _ptr(last_hit), _ptr(t), _ptr(t_first), _ptr(score_ring), _ptr(out),
                                _ptr(keep), _ptr(kept_idx), _ptr(workspace), nbytes, _ptr(status), _opts(opts),
                                _stream(stream))
    return _check(rc, "corm_decode_step") if check else rc


def corm_decode_step_lazy(desc, q, k_new, v_new, K, V, lens, live, pos, last_hit, t, t_first, score_ring, out,
                          keep=None, nlive=None, dead_num=1, dead_den=4, workspace=None, workspace_bytes=None,
                          status=None, stream=None, check=True, opts=None) -> int:
    nbytes = workspace_bytes
    if nbytes is None:
        nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().corm_decode_step_lazy(ctypes.byref(desc), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V),
                                     _ptr(lens), _ptr(live), _ptr(pos), _ptr(last_hit), _ptr(t), _ptr(t_first),
                                     _ptr(score_ring), _ptr(out), _ptr(keep), _ptr(nlive), dead_num, dead_den,
                                     _ptr(workspace), nbytes, _ptr(status), _opts(opts), _stream(stream))
    return _check(rc, "corm_decode_step_lazy") if check else rc


def corm_prefill_seed(desc, q_tail, m, K, V, lens, pos, last_hit, t, t_first, score_ring, keep=None, kept_idx=None,
                      workspace=None, workspace_bytes=None, status=None, stream=None, check=True) -> int:
    nbytes = workspace_bytes
    if nbytes is None:
        nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().corm_prefill_seed(ctypes.byref(desc), _ptr(q_tail), m, _ptr(K), _ptr(V), _ptr(lens), _ptr(pos),
                                 _ptr(last_hit), _ptr(t), _ptr(t_first), _ptr(score_ring), _ptr(keep), _ptr(kept_idx),
                                 _ptr(workspace), nbytes, _ptr(status), _stream(stream))
    return _check(rc, "corm_prefill_seed") if check else rc


def corm_threshold(c: float, t, n: int, thr, stream=None, check=True) -> int:
    rc = lib().corm_threshold(c, _ptr(t), n, _ptr(thr), _stream(stream))
    return _check(rc, "corm_threshold") if check else rc


# ---- fewer bits, fewer blocks, another eviction rule

_FLOATS = {CORM_F32: torch.float32, CORM_BF16: torch.bfloat16}
_CODES = {CORM_I8: (torch.int8,), CORM_E4M3: (torch.float8_e4m3fn, torch.uint8, torch.int8)}
_code_ids = {"i8": CORM_I8, "e4m3": CORM_E4M3, torch.int8: CORM_I8, torch.float8_e4m3fn: CORM_E4M3}


def _code(x) -> int:
    return x if isinstance(x, int) else _code_ids[x]


_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device() -> int:
    """The current device, asked once per call; no tensor is on -2, the answer before anything is on one."""
    return _get_device() if torch.cuda.is_initialized() else -2


def _on(stream, device: int) -> Optional[int]:
    """_stream, for a call that knows the current device."""
    if stream is None and _raw_stream is not None and device >= 0:
        return _raw_stream(device)
    return _stream(stream)


def _dev(x, n: Optional[int], dtypes, name: str, device: int) -> Optional[int]:
    """Pointer of an argument whose layout the call takes for granted.  A tensor has to be whole, of the right type, of n elements (None: any
    number) and on the current device (the call goes to one of its streams); a raw pointer is taken as it is."""
    if x is None:
        return None
    try:
        if x.dtype in dtypes and (x.numel() == n or n is None) and x.is_contiguous() and x.get_device() == device:
            return x.data_ptr()
    except AttributeError:   # not a tensor
        return int(x)
    raise ValueError(f"{name}: expected {n} contiguous elements of {dtypes} on the current device, got {x.dtype} {tuple(x.shape)} with "
                     f"strides {x.stride()} on {x.device}")


def _scratch(x, device: int):
    """Pointer of a workspace: any whole tensor on the current device, or a raw pointer."""
    if isinstance(x, torch.Tensor) and not (x.is_contiguous() and x.get_device() == device):
        raise ValueError(f"workspace: expected contiguous memory on the current device, got strides {x.stride()} on {x.device}")
    return _ptr(x)


_I32, _F4, _U8 = (torch.int32,), (torch.float32,), (torch.uint8, torch.bool)


def _sizes(desc):
    """units, heads, blocks per unit, dtypes of q, K and V"""
    return desc.B * desc.Hkv, desc.B * desc.Hq, (desc.Lcap + BLOCK - 1) // BLOCK, (_FLOATS.get(desc.kv_dtype),)


def corm_blocks_workspace_bytes(desc: corm_desc, check=True) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().corm_blocks_workspace_bytes(ctypes.byref(desc), ctypes.byref(n))
    if check:
        _check(rc, "corm_blocks_workspace_bytes")
        return n.value
    return rc


def corm_q8_append(desc, code, k_new, v_new, n, n_new, K_codes, V_codes, k_scale, v_scale, K_tail, V_tail, lens, lens_out,
                   bounds=None, status=None, stream=None, check=True) -> int:
    """code: "i8" or "e4m3"; n_new: rows per sequence, None = n for all."""
    code = _code(code)
    units, _, nblk, kv = _sizes(desc)
    at = _device()
    ct, d = _CODES.get(code, ()), desc.d
    rc = lib().corm_q8_append(ctypes.byref(desc), code, _dev(k_new, units * n * d, kv, "k_new", at), _dev(v_new, units * n * d, kv, "v_new", at),
                              n, _dev(n_new, desc.B, _I32, "n_new", at), _dev(K_codes, units * nblk * BLOCK * d, ct, "K_codes", at),
                              _dev(V_codes, units * nblk * BLOCK * d, ct, "V_codes", at), _dev(k_scale, units * nblk, _F4, "k_scale", at),
                              _dev(v_scale, units * nblk, _F4, "v_scale", at), _dev(K_tail, units * BLOCK * d, kv, "K_tail", at),
                              _dev(V_tail, units * BLOCK * d, kv, "V_tail", at), _dev(lens, units, _I32, "lens", at),
                              _dev(lens_out, units, _I32, "lens_out", at), _dev(bounds, units * nblk * 2 * d, kv, "bounds", at),
                              _dev(status, None, _I32, "status", at), _on(stream, at))
    return _check(rc, "corm_q8_append") if check else rc


def corm_q8_attend(desc, code, q, K_codes, V_codes, k_scale, v_scale, K_tail, V_tail, lens, out, workspace, workspace_bytes=None,
                   blocks=None, nsel=0, status=None, stream=None, check=True) -> int:
    code = _code(code)
    units, heads, nblk, kv = _sizes(desc)
    at = _device()
    ct, d = _CODES.get(code, ()), desc.d
    rc = lib().corm_q8_attend(ctypes.byref(desc), code, _dev(q, heads * d, kv, "q", at), _dev(K_codes, units * nblk * BLOCK * d, ct, "K_codes", at),
                              _dev(V_codes, units * nblk * BLOCK * d, ct, "V_codes", at), _dev(k_scale, units * nblk, _F4, "k_scale", at),
                              _dev(v_scale, units * nblk, _F4, "v_scale", at), _dev(K_tail, units * BLOCK * d, kv, "K_tail", at),
                              _dev(V_tail, units * BLOCK * d, kv, "V_tail", at), _dev(lens, units, _I32, "lens", at),
                              _dev(blocks, units * nsel, _I32, "blocks", at), nsel, _dev(out, heads * d, _F4, "out", at), _scratch(workspace, at),
                              _nbytes(workspace, workspace_bytes), _dev(status, None, _I32, "status", at), _on(stream, at))
    return _check(rc, "corm_q8_attend") if check else rc


def corm_block_bounds(desc, K, lens, bounds, newest=0, stream=None, check=True) -> int:
    """newest: renew the blocks that hold one of the newest `newest` slots; 0 = every block."""
    units, _, nblk, kv = _sizes(desc)
    at = _device()
    rc = lib().corm_block_bounds(ctypes.byref(desc), _dev(K, units * desc.Lcap * desc.d, kv, "K", at), _dev(lens, units, _I32, "lens", at), newest,
                                 _dev(bounds, units * nblk * 2 * desc.d, kv, "bounds", at), _on(stream, at))
    return _check(rc, "corm_block_bounds") if check else rc


def corm_block_select(desc, q, bounds, lens, nsel, nlast, blocks, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    units, heads, nblk, kv = _sizes(desc)
    at = _device()
    rc = lib().corm_block_select(ctypes.byref(desc), _dev(q, heads * desc.d, kv, "q", at), _dev(bounds, units * nblk * 2 * desc.d, kv, "bounds", at),
                                 _dev(lens, units, _I32, "lens", at), nsel, nlast, _dev(blocks, units * nsel, _I32, "blocks", at), _scratch(workspace, at),
                                 _nbytes(workspace, workspace_bytes), _on(stream, at))
    return _check(rc, "corm_block_select") if check else rc


def corm_block_attend(desc, q, K, V, lens, blocks, nsel, out, workspace, workspace_bytes=None, status=None, stream=None,
                      check=True) -> int:
    units, heads, _, kv = _sizes(desc)
    at = _device()
    rows = units * desc.Lcap * desc.d
    rc = lib().corm_block_attend(ctypes.byref(desc), _dev(q, heads * desc.d, kv, "q", at), _dev(K, rows, kv, "K", at), _dev(V, rows, kv, "V", at),
                                 _dev(lens, units, _I32, "lens", at), _dev(blocks, units * nsel, _I32, "blocks", at), nsel,
                                 _dev(out, heads * desc.d, _F4, "out", at), _scratch(workspace, at), _nbytes(workspace, workspace_bytes),
                                 _dev(status, None, _I32, "status", at), _on(stream, at))
    return _check(rc, "corm_block_attend") if check else rc


def corm_decode_attend_weigh(desc, q, K, V, lens, weight_in, weight, out, workspace, workspace_bytes=None, status=None, stream=None,
                             check=True, opts=None) -> int:
    units, heads, _, kv = _sizes(desc)
    at = _device()
    rows = units * desc.Lcap * desc.d
    rc = lib().corm_decode_attend_weigh(ctypes.byref(desc), _dev(q, heads * desc.d, kv, "q", at), _dev(K, rows, kv, "K", at), _dev(V, rows, kv, "V", at),
                                        _dev(lens, units, _I32, "lens", at), _dev(weight_in, units * desc.Lcap, _F4, "weight_in", at),
                                        _dev(weight, units * desc.Lcap, _F4, "weight", at), _dev(out, heads * desc.d, _F4, "out", at),
                                        _scratch(workspace, at), _nbytes(workspace, workspace_bytes), _dev(status, None, _I32, "status", at),
                                        _opts(opts), _on(stream, at))
    return _check(rc, "corm_decode_attend_weigh") if check else rc


def corm_evict_mask_weight(desc, weight, lens, budget, keep, workspace, workspace_bytes=None, stream=None, check=True) -> int:
    units, at = desc.B * desc.Hkv, _device()
    rc = lib().corm_evict_mask_weight(ctypes.byref(desc), _dev(weight, units * desc.Lcap, _F4, "weight", at), _dev(lens, units, _I32, "lens", at),
                                      budget, _dev(keep, units * desc.Lcap, _U8, "keep", at), _scratch(workspace, at),
                                      _nbytes(workspace, workspace_bytes), _on(stream, at))
    return _check(rc, "corm_evict_mask_weight") if check else rc


# ---- a cache of pages, and the rows on their way into it

def _watched(name):
    """An attribute that holds a tensor: set anew, it is looked at by the next call."""
    def put(self, x):
        setattr(self, "_" + name, x)
        self._seen = None
    return property(operator.attrgetter("_" + name), put)


def _memory(x):
    """A tensor's memory, which stays its own as long as this is held: no other tensor gets its address meanwhile."""
    return None if x is None else x.detach()


class Rotation:
    """What a model does to its queries and keys before attention (corm_rotation): norms per head and the position rotation.  Made once.

    inv_freq [rot / 2] float32 (None: norms alone); q_norm, k_norm [d] in the KV type; pairing "halves" or "neighbours"; sections: the pairs of
    each axis (None: one axis), dealt in blocks or in_turn.  A tensor may be set anew, or get other memory or another type (a module that is moved): it is
    looked at again.  One whose shape or strides are changed in place has to be set anew."""

    inv_freq, q_norm, k_norm = (_watched(x) for x in ("inv_freq", "q_norm", "k_norm"))

    def __init__(self, inv_freq, q_norm=None, k_norm=None, eps=1e-6, pairing="halves", sections=None, in_turn=False, gain=1.0):
        half = 0 if inv_freq is None else inv_freq.numel()
        sections = [half] if sections is None else [operator.index(x) for x in sections]
        if not 1 <= len(sections) <= 4:
            raise ValueError(f"sections: one to four axes, got {len(sections)}")
        if min(sections) < 0 or max(sections) > half:   # (the structure's integers would keep the lower 32 bits)
            raise ValueError(f"sections: {sections} of {half} pairs")
        self.inv_freq, self.q_norm, self.k_norm, self.axes, self.rot = inv_freq, q_norm, k_norm, len(sections), 2 * half
        self.c = corm_rotation(2 * half, {"halves": CORM_HALVES, "neighbours": CORM_NEIGHBOURS}[pairing], len(sections), int(bool(in_turn)),
                               tuple(sections), eps, gain)
        self._seen = None

    def _bind(self, desc, device):
        f, q, k = self._inv_freq, self._q_norm, self._k_norm
        seen = (device, desc.kv_dtype, desc.d, None if f is None else (f.data_ptr(), f.dtype), None if q is None else (q.data_ptr(), q.dtype),
                None if k is None else (k.data_ptr(), k.dtype))
        if seen != self._seen:
            _, _, _, kv = _sizes(desc)
            self._seen = None
            self.c.inv_freq = _dev(f, self.rot // 2, _F4, "inv_freq", device)
            self.c.q_norm = _dev(q, desc.d, kv, "q_norm", device)
            self.c.k_norm = _dev(k, desc.d, kv, "k_norm", device)
            self._held, self._seen = (_memory(f), _memory(q), _memory(k)), seen
        return ctypes.byref(self.c)


class Pages:
    """A pool of pages and the tables of the units (corm_pages).  Made once; the tensors' contents may change, the tables' among them.

    K, V [npages, page, d] with table [B, Hkv, max_pages] int32, or [npages, Hkv, page, d] with table [B, 1, max_pages]: in the KV type, or int8 or
    float8_e4m3fn with k_scale and v_scale, float32, of the same shape without d.  (As in Rotation: set anew or moved, a tensor is looked at again.)"""

    K, V, table, k_scale, v_scale = (_watched(x) for x in ("K", "V", "table", "k_scale", "v_scale"))

    def __init__(self, desc, K, V, table, k_scale=None, v_scale=None):
        self._of = (desc.B, desc.Hkv, desc.d, desc.kv_dtype)
        self.sizes = (desc.B, desc.Hkv, desc.d, (_FLOATS.get(desc.kv_dtype),))   # of the descriptor that every call's is like, and the KV type
        self._K, self._V, self._table, self._k_scale, self._v_scale = K, V, table, k_scale, v_scale
        self.c = corm_pages()
        self._seen = None
        self._look()

    def _look(self) -> None:
        """What the tensors' shapes and types say."""
        K, V, table = self._K, self._V, self._table
        B, Hkv, d, kv = self.sizes
        if table.dim() != 3 or K.dim() not in (3, 4) or K.shape != V.shape or K.dtype != V.dtype:
            raise ValueError(f"pages: K {tuple(K.shape)} {K.dtype}, V {tuple(V.shape)} {V.dtype}, table {tuple(table.shape)}")
        shared = K.dim() == 4
        if tuple(K.shape[1:]) != ((Hkv,) if shared else ()) + (K.shape[-2], d) or tuple(table.shape[:2]) != (B, 1 if shared else Hkv):
            raise ValueError(f"pages: K {tuple(K.shape)} and table {tuple(table.shape)} are not those of B {B}, Hkv {Hkv}, d {d}")
        code, c = _code_ids.get(K.dtype), self.c
        self.types = kv if code is None else (K.dtype,)
        self.tables = B * table.shape[1]
        c.dtype, c.page, c.npages, c.max_pages, c.table_heads = self._of[3] if code is None else code, K.shape[-2], K.shape[0], table.shape[2], table.shape[1]

    def _bind(self, desc, device):
        if (desc.B, desc.Hkv, desc.d, desc.kv_dtype) != self._of:
            raise ValueError("pages: made for another descriptor")
        K, V, t, ks, vs = self._K, self._V, self._table, self._k_scale, self._v_scale
        seen = (device, K.data_ptr(), K.dtype, V.data_ptr(), V.dtype, t.data_ptr(), t.dtype, None if ks is None else (ks.data_ptr(), ks.dtype),
                None if vs is None else (vs.data_ptr(), vs.dtype))
        if seen != self._seen:
            self._seen = None
            self._look()
            n, c = K.numel(), self.c
            c.K, c.V = _dev(K, n, self.types, "K", device), _dev(V, n, self.types, "V", device)
            c.k_scale = _dev(ks, n // desc.d, _F4, "k_scale", device)
            c.v_scale = _dev(vs, n // desc.d, _F4, "v_scale", device)
            c.table = _dev(t, self.tables * c.max_pages, _I32, "table", device)
            self._held, self._seen = tuple(_memory(x) for x in (K, V, t, ks, vs)), seen
        return ctypes.byref(self.c)


def _strided(x, shape, kv, name, device):
    """Pointer and strides (sequence, token, head) of rows [B, heads, n, d] or, of one token, [B, heads, d]: any view whose rows lie whole."""
    at = x.stride()
    if x.dtype is not kv or x.shape != (shape if len(at) == 4 else shape[:2] + shape[3:]) or at[-1] != 1 or x.get_device() != device:
        raise ValueError(f"{name}: expected {shape} of {kv} on the current device with its rows whole, got {x.dtype} {tuple(x.shape)} with strides "
                         f"{at} on {x.device}")
    B, heads, n, _ = shape
    return x.data_ptr(), at[0] if B > 1 else 0, at[2] if n > 1 else 0, at[1] if heads > 1 else 0


def _rows_of(desc, q, k, v, n, device):
    B, Hkv, d, kv = desc.B, desc.Hkv, desc.d, _FLOATS.get(desc.kv_dtype)
    q, *qs = (None, 0, 0, 0) if q is None else _strided(q, (B, desc.Hq, n, d), kv, "q", device)
    k, *ks = _strided(k, (B, Hkv, n, d), kv, "k", device)
    v, *vs = _strided(v, (B, Hkv, n, d), kv, "v", device)
    return corm_rows(q, k, v, *qs, *ks, *vs)


def _tokens(k) -> int:
    return 1 if k.dim() == 3 else k.shape[2]


def corm_rotate(desc, q, k, v, rotation, positions, q_out, k_out, v_out, n_new=None, stream=None, check=True) -> int:
    """q [B,Hq,n,d] (with q_out None: not read), k, v [B,Hkv,n,d], any strides (a projection's output token by token: its view, transposed);
    positions [axes,B,n] int32."""
    at, n = _device(), _tokens(k)
    rows = _rows_of(desc, None if q_out is None else q, k, v, n, at)
    kv, each = (_FLOATS.get(desc.kv_dtype),), desc.B * n * desc.d
    rc = lib().corm_rotate(ctypes.byref(desc), ctypes.byref(rows), rotation._bind(desc, at),
                           _dev(positions, rotation.axes * desc.B * n, _I32, "positions", at), n, _dev(n_new, desc.B, _I32, "n_new", at),
                           _dev(q_out, desc.Hq * each, kv, "q_out", at), _dev(k_out, desc.Hkv * each, kv, "k_out", at),
                           _dev(v_out, desc.Hkv * each, kv, "v_out", at), _on(stream, at))
    return _check(rc, "corm_rotate") if check else rc


def corm_paged_append(desc, pages, k, v, lens, lens_out, n_new=None, q=None, q_out=None, rotation=None, positions=None, status=None,
                      stream=None, check=True) -> int:
    """k, v (and q, where q_out is given) as in corm_rotate; lens, lens_out [B, tables per sequence]."""
    at, n = _device(), _tokens(k)
    rows = _rows_of(desc, None if q_out is None else q, k, v, n, at)
    turn = pos = None
    if rotation is not None:
        turn, pos = rotation._bind(desc, at), _dev(positions, rotation.axes * desc.B * n, _I32, "positions", at)
    of = pages._bind(desc, at)
    B, _, d, kv = pages.sizes
    rc = lib().corm_paged_append(ctypes.byref(desc), of, ctypes.byref(rows), turn, pos, n, _dev(n_new, B, _I32, "n_new", at),
                                 _dev(q_out, B * desc.Hq * n * d, kv, "q_out", at), _dev(lens, pages.tables, _I32, "lens", at),
                                 _dev(lens_out, pages.tables, _I32, "lens_out", at), _dev(status, None, _I32, "status", at), _on(stream, at))
    return _check(rc, "corm_paged_append") if check else rc


def corm_paged_read(desc, pages, lens, K_out, V_out, status=None, stream=None, check=True) -> int:
    """K_out, V_out [B,Hkv,n,d]"""
    at = _device()
    if K_out.dim() != 4 or K_out.shape != V_out.shape:
        raise ValueError(f"K_out {tuple(K_out.shape)}, V_out {tuple(V_out.shape)}: expected [B, Hkv, n, d]")
    of, n = pages._bind(desc, at), K_out.shape[2]
    B, Hkv, d, kv = pages.sizes
    rc = lib().corm_paged_read(ctypes.byref(desc), of, _dev(lens, pages.tables, _I32, "lens", at), n, _dev(K_out, B * Hkv * n * d, kv, "K_out", at),
                               _dev(V_out, B * Hkv * n * d, kv, "V_out", at), _dev(status, None, _I32, "status", at), _on(stream, at))
    return _check(rc, "corm_paged_read") if check else rc


def corm_paged_workspace_bytes(desc: corm_desc, check=True) -> int:
    n = ctypes.c_size_t(0)
    rc = lib().corm_paged_workspace_bytes(ctypes.byref(desc), ctypes.byref(n))
    if check:
        _check(rc, "corm_paged_workspace_bytes")
        return n.value
    return rc


def corm_paged_attend(desc, pages, q, lens, out, workspace, workspace_bytes=None, status=None, stream=None, check=True) -> int:
    """q [B,Hq,d] -> out [B,Hq,d] float32"""
    at = _device()
    of = pages._bind(desc, at)
    B, _, d, kv = pages.sizes
    heads = B * desc.Hq
    rc = lib().corm_paged_attend(ctypes.byref(desc), of, _dev(q, heads * d, kv, "q", at), _dev(lens, pages.tables, _I32, "lens", at),
                                 _dev(out, heads * d, _F4, "out", at), _scratch(workspace, at), _nbytes(workspace, workspace_bytes),
                                 _dev(status, None, _I32, "status", at), _on(stream, at))
    return _check(rc, "corm_paged_attend") if check else rc


# ---- device-memory plumbing for one layer (allocation only; no arithmetic of the method)

class LayerState:
    """The device arrays of one layer, allocated with torch, in the layouts corm.h documents."""

    def __init__(self, B, Hq, Hkv, d, Lcap, Tcap, w, r, dtype, thr_scale=1.0, device="cuda",
                 workspace: Optional[torch.Tensor] = None, want_masks=False, want_ring=True, score_dtype=None, want_bounds=False,
                 want_weight=False, blocks_workspace: Optional[torch.Tensor] = None):
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.desc = make_desc(B, Hq, Hkv, d, Lcap, Tcap, w, r, dtype, score_dtype=score_dtype, thr_scale=thr_scale)
        self.ring_bits = self.desc.score_dtype == CORM_BIT
        self.B, self.Hq, self.Hkv, self.d, self.Lcap, self.Tcap, self.w, self.r = B, Hq, Hkv, d, Lcap, Tcap, w, r
        self.dtype = tdt
        self.K = torch.zeros(B, Hkv, Lcap, d, dtype=tdt, device=device)
        self.V = torch.zeros(B, Hkv, Lcap, d, dtype=tdt, device=device)
        self.lens = torch.zeros(B, Hkv, dtype=torch.int32, device=device)
        self.pos = torch.zeros(B, Hkv, Lcap, dtype=torch.int32, device=device)
        self.last_hit = torch.zeros(B, Hkv, Lcap, dtype=torch.int32, device=device)
        # want_ring=False: summary-only state (score_ring == NULL in every call)
        if not want_ring:
            self.ring = None
        elif self.ring_bits:   # the boolean message: bit pos % 32 of word pos // 32
            self.ring = torch.zeros(B, Hq, w, (Tcap + 31) // 32, dtype=torch.int32, device=device)
        else:
            sdt = tdt if score_dtype is None else {"f32": torch.float32, "bf16": torch.bfloat16}[score_dtype]
            self.ring = torch.zeros(B, Hq, w, Tcap, dtype=sdt, device=device)
        self.out = torch.zeros(B, Hq, d, dtype=torch.float32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.keep = torch.zeros(B, Hkv, Lcap, dtype=torch.uint8, device=device) if want_masks else None
        self.kept_idx = torch.zeros(B, Hkv, Lcap, dtype=torch.int32, device=device) if want_masks else None
        # deferred compaction (step_lazy): live masks, all ones = every slot below lens holds a live key
        self.live = torch.full((B, Hkv, (Lcap + 63) // 64), -1, dtype=torch.int64, device=device)
        self.nlive = torch.zeros(B, Hkv, dtype=torch.int32, device=device)
        if workspace is None:
            workspace = torch.empty(corm_workspace_bytes(self.desc), dtype=torch.uint8, device=device)
            corm_workspace_init(self.desc, workspace)
        elif want_weight:
            _check_room(workspace, corm_workspace_bytes(self.desc), "workspace")
        self.workspace = workspace
        # want_bounds: bounds of the blocks' keys, for step_blocks; want_weight: the keys' accounts, for step_weigh
        nblk = (Lcap + BLOCK - 1) // BLOCK
        self.bounds = torch.zeros(B, Hkv, nblk, 2, d, dtype=tdt, device=device) if want_bounds else None
        self._lists = _block_lists(self.desc, device) if want_bounds else None
        self.weight = torch.zeros(B, Hkv, Lcap, dtype=torch.float32, device=device) if want_weight else None
        self.weight_keep = torch.zeros(B, Hkv, Lcap, dtype=torch.uint8, device=device) if want_weight else None
        self._dead = False  # there may be dead slots (step_lazy)
        self._rule = None   # what a state with accounts has evicted by since its prompt: "hits" or "weight"
        # (tens of megabytes for hundreds of heads: layers whose steps follow one another may share it, as they may `workspace`)
        self.blocks_workspace = blocks_workspace
        if blocks_workspace is None and (want_bounds or want_weight):
            self.blocks_workspace = torch.empty(corm_blocks_workspace_bytes(self.desc), dtype=torch.uint8, device=device)
        elif blocks_workspace is not None:
            _check_room(blocks_workspace, corm_blocks_workspace_bytes(self.desc), "blocks_workspace")

    def preload(self, K0: torch.Tensor, V0: torch.Tensor) -> None:
        """Copy n prompt keys/values [B,Hkv,n,d] into slots 0..n-1 (positions 0..n-1, never important yet, none dead, accounts empty)."""
        n = K0.shape[2]
        self.K[:, :, :n].copy_(K0)
        self.V[:, :, :n].copy_(V0)
        self.pos[:, :, :n] = torch.arange(n, dtype=torch.int32, device=self.pos.device)
        self.last_hit[:, :, :n] = 0
        self.lens.fill_(n)
        self.live.fill_(-1)
        if self.weight is not None:
            self.weight.zero_()
        self._rule, self._dead = None, False
        if self.bounds is not None:
            with torch.cuda.device_of(self.K):
                self._rows_moved()

    def _rows_moved(self, stream=None) -> None:
        """Behind a call that moves rows, or may (which only the device knows): the bounds of what lies there now."""
        if self.bounds is not None:
            corm_block_bounds(self.desc, self.K, self.lens, self.bounds, 0, stream=stream)

    def _check_rule(self, rule: str) -> None:
        """CORM's steps move rows without their accounts, step_weigh without last_hit, so a state with accounts evicts by one of them from a prompt
        to the next preload.  (A graph counts where it is captured: one of the other kind is not to be replayed behind a preload.)"""
        if self.weight is not None and self._rule not in (None, rule):
            raise RuntimeError("a state with accounts evicts by hits (step, step_lazy, step_attend, step_evict) or by weight (step_weigh), "
                               "not by both: preload it, or make another one")

    def step_attend(self, q, k_new, v_new, t, t_first, stream=None, workspace=None, opts=None) -> None:
        self._check_rule("hits")
        corm_step_attend(self.desc, q, k_new, v_new, self.K, self.V, self.lens, self.pos, self.last_hit, t, t_first,
                         self.ring, self.out, self.keep, self.workspace if workspace is None else workspace,
                         status=self.status, stream=stream, opts=opts)
        self._rule = "hits"

    def step_evict(self, stream=None, workspace=None) -> None:
        self._check_rule("hits")
        corm_step_evict(self.desc, self.K, self.V, self.lens, self.pos, self.last_hit, self.kept_idx,
                        self.workspace if workspace is None else workspace, stream=stream)
        self._rule = "hits"
        self._rows_moved(stream)

    def step(self, q, k_new, v_new, t, t_first, stream=None, opts=None) -> None:
        self._check_rule("hits")
        corm_decode_step(self.desc, q, k_new, v_new, self.K, self.V, self.lens, self.pos, self.last_hit, t, t_first,
                         self.ring, self.out, self.keep, self.kept_idx, self.workspace, status=self.status,
                         stream=stream, opts=opts)
        self._rule = "hits"
        self._rows_moved(stream)

    def step_lazy(self, q, k_new, v_new, t, t_first, dead_num=1, dead_den=4, stream=None, workspace=None,
                  opts=None) -> None:
        self._check_rule("hits")
        corm_decode_step_lazy(self.desc, q, k_new, v_new, self.K, self.V, self.lens, self.live, self.pos,
                              self.last_hit, t, t_first, self.ring, self.out, self.keep, self.nlive, dead_num,
                              dead_den, self.workspace if workspace is None else workspace, status=self.status,
                              stream=stream, opts=opts)
        self._rule, self._dead = "hits", True

    def prefill_seed(self, q_tail, t, t_first, stream=None, workspace=None) -> None:
        """q_tail [B,Hq,m,d]; the cache must already hold the whole prompt (preload).  Accounts are empty behind it."""
        corm_prefill_seed(self.desc, q_tail, q_tail.shape[2], self.K, self.V, self.lens, self.pos, self.last_hit, t,
                          t_first, self.ring, self.keep, self.kept_idx,
                          self.workspace if workspace is None else workspace, status=self.status, stream=stream)
        if self.weight is not None:
            with _as_current(stream):
                self.weight.zero_()
        self._rows_moved(stream)

    def renew_bounds(self, newest=0, stream=None) -> None:
        """Bounds of the blocks' keys (all of them, or those of the newest slots): after rows were written by other means than the state's own
        preload and steps, which keep them up."""
        if self.bounds is None:
            raise RuntimeError("made without want_bounds")
        corm_block_bounds(self.desc, self.K, self.lens, self.bounds, newest, stream=stream)

    def step_blocks(self, q, k_new, v_new, t, nsel, nlast=1, stream=None) -> None:
        """One decode step that attends to nsel blocks of 64 slots (the nlast newest and those with the highest score bounds): append,
        the newest block's bounds, choice (self.blocks, until the next step), attention.  Nothing is evicted, and nothing recorded: a
        ring's row of this step keeps what an older step left in it, so the literal corm_evict_mask is not for windows with such a step."""
        if self.bounds is None:
            raise RuntimeError("made without want_bounds")
        if self._dead:
            raise RuntimeError("behind step_lazy a state may hold dead slots, which step_blocks would attend to: preload it, or go on with step_lazy")
        _check_choice(self.desc, nsel, nlast)
        _check_query(self.desc, q)
        self.blocks = _lists_of(self._lists, self.desc, nsel)
        ws = self.blocks_workspace
        # The new row's entry of what the state evicts by.  While it has evicted by neither, all accounts behind the rows are empty, so last_hit
        # is the one to set; a graph may be replayed behind a cut by weight, so one that is captured sets the account and goes by that rule.
        rule = "weight" if self.weight is not None and self._rule is None and _capturing(stream) else self._rule
        entry = self.weight if rule == "weight" else self.last_hit
        corm_append(self.desc, self.K, self.V, self.lens, self.pos, entry, k_new, v_new, t, self.status, stream=stream)
        self._rule = rule
        self.renew_bounds(1, stream=stream)
        corm_block_select(self.desc, q, self.bounds, self.lens, nsel, nlast, self.blocks, ws, stream=stream)
        corm_block_attend(self.desc, q, self.K, self.V, self.lens, self.blocks, nsel, self.out, ws, status=self.status, stream=stream)

    def step_weigh(self, q, k_new, v_new, t, budget=None, stream=None) -> None:
        """One decode step of eviction by accumulated attention weight: append, attend and account (self.weight), and with a budget cut every
        longer unit to it (the r newest slots and the heaviest others; self.weight_keep: the slots that stayed).  last_hit is left behind."""
        if self.weight is None:
            raise RuntimeError("made without want_weight")
        self._check_rule("weight")
        _check_query(self.desc, q)
        if budget is not None and not self.r <= operator.index(budget) < 1 << 31:
            raise CormError(CORM_EINVAL, f"budget {budget} with r {self.r}")
        account = self.weight   # 4-byte entries: append and the gather carry them in the place of last_hit
        corm_append(self.desc, self.K, self.V, self.lens, self.pos, account, k_new, v_new, t, self.status, stream=stream)
        self._rule = "weight"
        corm_decode_attend_weigh(self.desc, q, self.K, self.V, self.lens, account, account, self.out, self.workspace,
                                 status=self.status, stream=stream)
        if budget is None:
            if self.bounds is not None:
                self.renew_bounds(1, stream=stream)
        else:
            corm_evict_mask_weight(self.desc, account, self.lens, budget, self.weight_keep, self.blocks_workspace, stream=stream)
            corm_compact(self.desc, self.K, self.V, self.pos, account, self.lens, self.weight_keep, self.kept_idx, self.workspace,
                         stream=stream)
            self._rows_moved(stream)


# A step of several calls looks at what the later ones would refuse before the first one has put a row in.

def _most_listed(desc) -> int:
    return max((desc.Lcap + BLOCK - 1) // BLOCK, 512)


def _check_choice(desc, nsel, nlast) -> None:
    if not 1 <= operator.index(nlast) <= operator.index(nsel) <= _most_listed(desc):
        raise CormError(CORM_EINVAL, f"nsel {nsel}, nlast {nlast}")


def _check_query(desc, q) -> None:
    _, heads, _, kv = _sizes(desc)
    p = _dev(q, heads * desc.d, kv, "q", _device())
    if not p or p % 16:
        raise CormError(CORM_EINVAL, "q")


def _check_room(x, nbytes, name) -> None:
    if not x.is_contiguous():
        raise ValueError(f"{name}: expected contiguous memory")
    if x.numel() * x.element_size() < nbytes or x.data_ptr() % 256:
        raise CormError(CORM_ECAPACITY, f"{name}: {nbytes} bytes, 256-byte aligned")


def _block_lists(desc, device) -> torch.Tensor:
    """Room for the longest lists of chosen blocks."""
    return torch.empty(desc.B * desc.Hkv * _most_listed(desc), dtype=torch.int32, device=device)


def _lists_of(room, desc, nsel) -> torch.Tensor:
    """Lists of nsel blocks in it: a step allocates nothing, since it may be given another stream than the current one."""
    return room[:desc.B * desc.Hkv * nsel].view(desc.B, desc.Hkv, nsel)


class Q8State:
    """The device arrays of one layer's 8-bit cache, in the layouts corm.h documents.  want_bounds: keep up the blocks' bounds, for
    steps that attend to chosen blocks."""

    def __init__(self, B, Hq, Hkv, d, Lcap, dtype, code="i8", device="cuda", want_bounds=False, workspace: Optional[torch.Tensor] = None):
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.desc = make_desc(B, Hq, Hkv, d, Lcap, Lcap, 1, 1, dtype)
        self.B, self.Hq, self.Hkv, self.d, self.Lcap, self.dtype, self.code = B, Hq, Hkv, d, Lcap, tdt, code
        n = (Lcap + BLOCK - 1) // BLOCK
        cdt = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}[code]
        self.K_codes = torch.zeros(B, Hkv, n, d // BLOCK, BLOCK, BLOCK, dtype=torch.int8, device=device).view(cdt)
        self.V_codes = torch.zeros(B, Hkv, n, d, BLOCK, dtype=torch.int8, device=device).view(cdt)
        self.k_scale = torch.zeros(B, Hkv, n, dtype=torch.float32, device=device)
        self.v_scale = torch.zeros(B, Hkv, n, dtype=torch.float32, device=device)
        self.K_tail = torch.zeros(B, Hkv, BLOCK, d, dtype=tdt, device=device)
        self.V_tail = torch.zeros(B, Hkv, BLOCK, d, dtype=tdt, device=device)
        self.lens = torch.zeros(B, Hkv, dtype=torch.int32, device=device)
        self.out = torch.zeros(B, Hq, d, dtype=torch.float32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.bounds = torch.zeros(B, Hkv, n, 2, d, dtype=tdt, device=device) if want_bounds else None
        self._lists = _block_lists(self.desc, device) if want_bounds else None
        if workspace is None:
            workspace = torch.empty(corm_blocks_workspace_bytes(self.desc), dtype=torch.uint8, device=device)
        else:
            _check_room(workspace, corm_blocks_workspace_bytes(self.desc), "workspace")
        self.workspace = workspace

    def append(self, k, v, n_new=None, stream=None) -> None:
        """k, v [B,Hkv,n,d] (or [B,Hkv,d]: one row); n_new [B]: the rows of a sequence that count."""
        n = 1 if k.dim() == 3 else k.shape[2]
        corm_q8_append(self.desc, self.code, k, v, n, n_new, self.K_codes, self.V_codes, self.k_scale, self.v_scale, self.K_tail,
                       self.V_tail, self.lens, self.lens, self.bounds, self.status, stream=stream)

    def _check_choice(self, nsel, nlast) -> None:
        if self.bounds is None:
            raise RuntimeError("made without want_bounds")
        _check_choice(self.desc, nsel, nlast)

    def attend(self, q, nsel=0, nlast=1, stream=None) -> None:
        """q [B,Hq,d] -> out.  nsel > 0: over the nlast newest blocks and those with the highest score bounds, nsel in all."""
        if nsel:
            self._check_choice(nsel, nlast)
            self.blocks = _lists_of(self._lists, self.desc, nsel)
            corm_block_select(self.desc, q, self.bounds, self.lens, nsel, nlast, self.blocks, self.workspace, stream=stream)
        corm_q8_attend(self.desc, self.code, q, self.K_codes, self.V_codes, self.k_scale, self.v_scale, self.K_tail, self.V_tail,
                       self.lens, self.out, self.workspace, blocks=self.blocks if nsel else None, nsel=nsel, status=self.status,
                       stream=stream)

    def step(self, q, k_new, v_new, nsel=0, nlast=1, stream=None) -> None:
        """One decode step: the new row goes in, the query attends to all keys (or the chosen blocks), itself among them."""
        if nsel:
            self._check_choice(nsel, nlast)
        _check_query(self.desc, q)
        self.append(k_new, v_new, stream=stream)
        self.attend(q, nsel, nlast, stream=stream)


def _of_pages(name):
    return property(lambda self: getattr(self.pages, name), lambda self, x: setattr(self.pages, name, x))


class PagedState:
    """The device arrays of one layer's cache of pages, in the layouts corm.h documents.  The caller deals the pages: table [B, 1, max_pages], or
    [B, Hkv, max_pages] with per_head, holds -1 (no page) until it is written (deal() gives every unit max_pages of its own).  The pools, their scales and
    the table are those of `pages`; set anew on either, they are the ones that the next call takes."""

    K, V, table, k_scale, v_scale = (_of_pages(x) for x in ("K", "V", "table", "k_scale", "v_scale"))

    def __init__(self, B, Hq, Hkv, d, npages, max_pages, dtype, page=16, code=None, per_head=False, device="cuda",
                 workspace: Optional[torch.Tensor] = None):
        tdt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        cdt = {None: tdt, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}[code]
        cap = max_pages * page
        self.desc = make_desc(B, Hq, Hkv, d, cap, cap, 1, 1, dtype)
        self.B, self.Hq, self.Hkv, self.d, self.page, self.dtype, self.code = B, Hq, Hkv, d, page, tdt, code
        shape = (npages,) + (() if per_head else (Hkv,)) + (page, d)
        tables = Hkv if per_head else 1
        K, V = (torch.zeros(shape, dtype=torch.int8 if code else tdt, device=device).view(cdt) for _ in range(2))
        ks, vs = (torch.zeros(shape[:-1], dtype=torch.float32, device=device) if code else None for _ in range(2))
        self.pages = Pages(self.desc, K, V, torch.full((B, tables, max_pages), -1, dtype=torch.int32, device=device), ks, vs)
        self.lens = torch.zeros(B, tables, dtype=torch.int32, device=device)
        self.q = torch.zeros(B, Hq, d, dtype=tdt, device=device)   # a step's queries, rotated
        self.out = torch.zeros(B, Hq, d, dtype=torch.float32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        if workspace is None:
            workspace = torch.empty(corm_paged_workspace_bytes(self.desc), dtype=torch.uint8, device=device)
        else:
            _check_room(workspace, corm_paged_workspace_bytes(self.desc), "workspace")
        self.workspace = workspace

    def deal(self) -> None:
        """Every unit's pages, one unit behind the other."""
        if self.K.shape[0] < self.table.numel():
            raise CormError(CORM_ECAPACITY, f"{self.K.shape[0]} pages for tables of {self.table.numel()}")
        self.table.copy_(torch.arange(self.table.numel(), dtype=torch.int32, device=self.table.device).view_as(self.table))

    def append(self, k, v, n_new=None, q=None, q_out=None, rotation=None, positions=None, stream=None) -> None:
        """k, v [B,Hkv,n,d] (or [B,Hkv,d]: one row), any strides; n_new [B]: the rows of a sequence that count.  With a rotation keys are normed and
        rotated on the way, and queries q [B,Hq,n,d] into q_out."""
        corm_paged_append(self.desc, self.pages, k, v, self.lens, self.lens, n_new=n_new, q=q, q_out=q_out, rotation=rotation, positions=positions,
                          status=self.status, stream=stream)

    def read(self, K_out, V_out, stream=None) -> None:
        """The rows of every unit's slots into K_out, V_out [B,Hkv,n,d]."""
        corm_paged_read(self.desc, self.pages, self.lens, K_out, V_out, status=self.status, stream=stream)

    def attend(self, q, stream=None) -> None:
        """q [B,Hq,d] -> out"""
        corm_paged_attend(self.desc, self.pages, q, self.lens, self.out, self.workspace, status=self.status, stream=stream)

    def step(self, q, k_new, v_new, rotation=None, positions=None, stream=None) -> None:
        """One decode step: the new row goes in, the query attends to all keys, itself among them.  With a rotation queries and keys come as the
        projection leaves them (positions [axes,B,1])."""
        if _tokens(k_new) != 1:
            raise ValueError(f"k_new {tuple(k_new.shape)}: a step has one token")
        if rotation is None:
            _check_query(self.desc, q)
            self.append(k_new, v_new, stream=stream)
            self.attend(q, stream=stream)
        else:
            self.append(k_new, v_new, q=q, q_out=self.q, rotation=rotation, positions=positions, stream=stream)
            self.attend(self.q, stream=stream)
