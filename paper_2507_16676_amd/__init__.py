"""Flash-ABFT attention forward on AMD MI355X (gfx950).

Thin Python binding over the C ABI of ``libfabft.so`` (declared in
``include/fabft.h``): argument marshalling only. Every step of the attention
and of the checksum runs in the library's HIP kernels; torch supplies device
memory and the current stream. There is no fallback: if the library is not
built, every call raises.

    o, resid, flags = attn_fwd(q, k, v, causal=True)       # checksum on
    o = attn_fwd(q, k, v, causal=True, check=False)         # checksum off

q: [B, H, Lq, d], k and v: [B, H, Lk, d], torch.bfloat16 on the GPU,
contiguous; d in {64, 96, 128, 256}. scale defaults to 1/sqrt(d). Every
caller-supplied tensor (out=, workspaces) is checked for shape, dtype,
contiguity and device before the library sees its pointer.

A key/value cache held in 4 bits, for decoding over long contexts:

    cache = cache_new(B, H, capacity, d)                    # H key/value heads
    cache_append(cache, k, v, start)                        # the new tokens' K and V
    o, resid, flags = attn_fwd_cache(q, cache, lengths, causal=True, weight=w)
    index, lengths = cache_evict(cache, w, lengths, keep)   # the keys least looked at
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree build, or another build of the same library named by FABFT_LIB
# (the host-sanitized one of `python -m paper_2507_16676_amd.build
# --host-sanitize OUT`)
LIB_PATH = os.environ.get("FABFT_LIB") or os.path.join(_HERE, "libfabft.so")

_vp, _i, _f = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
_fp = ctypes.POINTER(ctypes.c_float)

FABFT_OK = 0
E_NULL, E_SHAPE, E_HEADDIM, E_ALIGN, E_LAUNCH, E_SCALE, E_FAULT, E_THRESHOLD, E_WORKSPACE, \
    E_MODE = -1, -2, -3, -4, -5, -6, -7, -8, -9, -10
PERSIST_OFF, PERSIST_AUTO, PERSIST_ALWAYS = 0, 1, 2
FLAG_RESID, FLAG_NONFINITE, FLAG_WEIGHTED, FLAG_SCORES = 1, 2, 4, 8
SITE_NONE, SITE_S, SITE_P, SITE_O, SITE_V, SITE_C, SITE_L, SITE_M, SITE_Q, SITE_VS = range(10)
SITES = {"none": SITE_NONE, "S": SITE_S, "P": SITE_P, "O": SITE_O, "V": SITE_V,
         "C": SITE_C, "L": SITE_L, "M": SITE_M, "Q": SITE_Q, "VS": SITE_VS}
MAX_FAULTS = 8


class FabftFault(ctypes.Structure):
    _fields_ = [("site", _i), ("b", _i), ("h", _i), ("row", _i), ("col", _i),
                ("tile", _i), ("bit", _i)]


class FabftDebugOut(ctypes.Structure):
    _fields_ = [("pred", _vp), ("actual", _vp), ("pred_w", _vp), ("actual_w", _vp),
                ("score_lhs", _vp), ("score_rhs", _vp), ("score_bound", _vp)]


_LIB = None
# set by _load: torch, and the raw handle of a device's current stream
_torch = None
_raw_stream = None


def _load() -> ctypes.CDLL:
    """Load libfabft.so once; raise if it is not built (no CPU fallback)."""
    global _LIB, _torch, _raw_stream
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -m paper_2507_16676_amd.build` "
            "(hipcc, gfx950). There is no CPU fallback.")
    # torch first: it brings its own HIP runtime, and the library must bind to
    # that same runtime (the one that owns torch's memory and streams); loaded
    # before torch, it would pull in the system runtime instead and launches
    # on torch's streams fail
    import torch
    _torch = torch
    # the handle without a Stream object around it (0.2 against 1.5 us)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda index: torch.cuda.current_stream(index).cuda_stream)
    L = ctypes.CDLL(LIB_PATH)
    L.fabft_attn_fwd.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _f]
    L.fabft_attn_fwd.restype = _i
    L.fabft_attn_fwd_nocheck.argtypes = [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _f]
    L.fabft_attn_fwd_nocheck.restype = _i
    L.fabft_attn_fwd_twopass.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _f]
    L.fabft_attn_fwd_twopass.restype = _i
    L.fabft_set_algorithm.argtypes = [_i]
    L.fabft_set_algorithm.restype = _i
    L.fabft_get_algorithm.argtypes = []
    L.fabft_get_algorithm.restype = _i
    L.fabft_attn_fwd_inject.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i,
                                        _f, ctypes.POINTER(FabftFault), _vp, _vp, _vp, _vp]
    L.fabft_attn_fwd_inject.restype = _i
    L.fabft_attn_fwd_inject_n.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i,
                                          _f, ctypes.POINTER(FabftFault), _i, _vp, _vp, _vp,
                                          _vp]
    L.fabft_attn_fwd_inject_n.restype = _i
    L.fabft_attn_fwd_debug.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i,
                                       _f, ctypes.POINTER(FabftFault), _i,
                                       ctypes.POINTER(FabftDebugOut)]
    L.fabft_attn_fwd_debug.restype = _i
    L.fabft_score_check_workspace_bytes.argtypes = [_i, _i, _i, _i]
    L.fabft_score_check_workspace_bytes.restype = ctypes.c_longlong
    L.fabft_set_score_check.argtypes = [_vp, ctypes.c_longlong, _f]
    L.fabft_set_score_check.restype = _i
    L.fabft_get_score_threshold.argtypes = []
    L.fabft_get_score_threshold.restype = _f
    L.fabft_set_stream.argtypes = [_vp]
    L.fabft_set_stream.restype = None
    L.fabft_set_threshold.argtypes = [_f, _f]
    L.fabft_set_threshold.restype = _i
    L.fabft_get_threshold.argtypes = [_fp, _fp]
    L.fabft_get_threshold.restype = None
    L.fabft_splitkv_workspace_bytes.argtypes = [_i, _i, _i, _i, _i]
    L.fabft_splitkv_workspace_bytes.restype = ctypes.c_longlong
    L.fabft_attn_fwd_splitkv.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i,
                                         _f, _i, _vp, ctypes.c_longlong]
    L.fabft_attn_fwd_splitkv.restype = _i
    L.fabft_attn_fwd_splitkv_noalloc.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i,
                                                 _i, _i, _f, _i]
    L.fabft_attn_fwd_splitkv_noalloc.restype = _i
    _ll = ctypes.c_longlong
    L.fabft_cache_bytes.argtypes = [_i, _i, _i, _i]
    L.fabft_cache_bytes.restype = _ll
    L.fabft_cache_append.argtypes = [_vp, _i, _i, _i, _i, _vp, _vp, _i, _vp, _vp, _vp]
    L.fabft_cache_append.restype = _i
    L.fabft_cache_read.argtypes = [_vp, _i, _i, _i, _i, _vp, _vp, _i, _vp, _vp]
    L.fabft_cache_read.restype = _i
    L.fabft_cache_splits.argtypes = [_i, _i, _i, _i, _i]
    L.fabft_cache_splits.restype = _i
    L.fabft_cache_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _i, _i]
    L.fabft_cache_workspace_bytes.restype = _ll
    L.fabft_attn_fwd_cache.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _vp,
                                       _i, _f, _vp, _f, _i, _vp, _ll]
    L.fabft_attn_fwd_cache.restype = _i
    L.fabft_cache_evict.argtypes = [_vp, _i, _i, _i, _i, _vp, _vp, _i, _i, _vp, _i, _vp, _vp, _vp]
    L.fabft_cache_evict.restype = _i
    L.fabft_recompute_flagged.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i,
                                          _f, _vp, _vp, _i, ctypes.POINTER(_i),
                                          ctypes.POINTER(_i)]
    L.fabft_recompute_flagged.restype = _i
    L.fabft_global_check.argtypes = [_vp, _vp, _i, _i, _i, _i, _vp, _vp]
    L.fabft_global_check.restype = _i
    L.fabft_set_weighted_check.argtypes = [_i]
    L.fabft_set_weighted_check.restype = None
    L.fabft_get_weighted_check.argtypes = []
    L.fabft_get_weighted_check.restype = _i
    L.fabft_set_persistent.argtypes = [_i]
    L.fabft_set_persistent.restype = _i
    L.fabft_get_persistent.argtypes = []
    L.fabft_get_persistent.restype = _i
    L.fabft_key_tile.argtypes = [_i]
    L.fabft_key_tile.restype = _i
    L.fabft_query_tile.argtypes = [_i]
    L.fabft_query_tile.restype = _i
    L.fabft_status_str.argtypes = [_i]
    L.fabft_status_str.restype = ctypes.c_char_p
    _LIB = L
    return L


EXPORTS = ("fabft_attn_fwd", "fabft_attn_fwd_nocheck", "fabft_attn_fwd_twopass",
           "fabft_attn_fwd_inject",
           "fabft_attn_fwd_inject_n", "fabft_attn_fwd_debug", "fabft_score_check_workspace_bytes",
           "fabft_set_score_check", "fabft_get_score_threshold",
           "fabft_attn_fwd_splitkv", "fabft_splitkv_workspace_bytes",
           "fabft_attn_fwd_splitkv_noalloc",
           "fabft_set_stream", "fabft_set_threshold", "fabft_get_threshold",
           "fabft_global_check", "fabft_recompute_flagged",
           "fabft_set_weighted_check", "fabft_get_weighted_check",
           "fabft_set_persistent", "fabft_get_persistent",
           "fabft_set_algorithm", "fabft_get_algorithm",
           "fabft_cache_bytes", "fabft_cache_append", "fabft_cache_read",
           "fabft_attn_fwd_cache", "fabft_cache_splits", "fabft_cache_workspace_bytes",
           "fabft_cache_evict",
           "fabft_key_tile", "fabft_query_tile", "fabft_status_str")


class FabftError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} (status {status})")


def status_str(status: int) -> str:
    return _load().fabft_status_str(int(status)).decode()


def lib() -> ctypes.CDLL:
    """The loaded C library (for tests of the raw ABI)."""
    return _load()


def _check(rc: int, where: str):
    if rc != FABFT_OK:
        raise FabftError(rc, where)


def set_threshold(tau_rel: float, tau_abs: float = 0.0):
    _check(_load().fabft_set_threshold(float(tau_rel), float(tau_abs)), "fabft_set_threshold")


def get_threshold() -> tuple[float, float]:
    a, b = ctypes.c_float(), ctypes.c_float()
    _load().fabft_get_threshold(ctypes.byref(a), ctypes.byref(b))
    return a.value, b.value


def score_check_workspace_bytes(B: int, H: int, Lk: int, d: int) -> int:
    r = _load().fabft_score_check_workspace_bytes(B, H, Lk, d)
    _check(int(r) if r < 0 else 0, "fabft_score_check_workspace_bytes")
    return int(r)


_SCORE_WS = None   # keeps the workspace tensor alive while the check is on


def set_score_check(workspace=None, tau_s: float = 0.0):
    """Switch the score check on with a device workspace (a tensor of at
    least score_check_workspace_bytes bytes), or off with None."""
    global _SCORE_WS
    if workspace is None:
        _check(_load().fabft_set_score_check(None, 0, 0.0), "fabft_set_score_check")
        _SCORE_WS = None
        return
    import torch
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or \
            not workspace.is_contiguous():
        raise ValueError("the score-check workspace must be a contiguous GPU tensor")
    nbytes = workspace.numel() * workspace.element_size()
    _check(_load().fabft_set_score_check(workspace.data_ptr(), nbytes, float(tau_s)),
           "fabft_set_score_check")
    _SCORE_WS = workspace


def get_score_threshold() -> float:
    return float(_load().fabft_get_score_threshold())


def set_weighted_check(on: bool):
    """Switch the second, weighted checksum on or off (process-global)."""
    _load().fabft_set_weighted_check(int(bool(on)))


def get_weighted_check() -> bool:
    return bool(_load().fabft_get_weighted_check())


def set_persistent(mode: int):
    """Persistent workgroups for attn_fwd (process-global): PERSIST_OFF,
    PERSIST_AUTO (default) or PERSIST_ALWAYS. A launch shape only: the
    results are bitwise the same."""
    _check(_load().fabft_set_persistent(int(mode)), "fabft_set_persistent")


def get_persistent() -> int:
    return int(_load().fabft_get_persistent())


def set_algorithm(alg: int):
    """The algorithm hosting the checksum in attn_fwd, the injection and
    debug paths and recompute_flagged (process-global): 3 (one pass, the
    default) or 1 (two passes, as attn_fwd_twopass)."""
    _check(_load().fabft_set_algorithm(int(alg)), "fabft_set_algorithm")


def get_algorithm() -> int:
    return int(_load().fabft_get_algorithm())


def key_tile(d: int) -> int:
    r = _load().fabft_key_tile(int(d))
    _check(min(r, 0), "fabft_key_tile")
    return r


def query_tile(d: int = 128) -> int:
    """Query rows per workgroup for head dimension d (the V/VS fault tile unit)."""
    r = _load().fabft_query_tile(int(d))
    _check(r if r < 0 else 0, "fabft_query_tile")
    return r


def _shape(q, k, v):
    if _torch is None:
        _load()
    bf16 = _torch.bfloat16
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dtype is not bf16:
            raise TypeError(f"{name} must be torch.bfloat16, got {t.dtype}")
        if not t.is_cuda:
            raise ValueError(f"{name} must be on the GPU")
        if t.dim() != 4 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous [B, H, L, d] tensor")
    B, H, Lq, d = q.shape
    ks = k.shape
    if ks[0] != B or ks[1] != H or ks[3] != d or v.shape != ks:
        raise ValueError(f"shape mismatch: q {tuple(q.shape)} k {tuple(k.shape)} v {tuple(v.shape)}")
    return B, H, Lq, ks[2], d


def _check_out(t, name: str, shape, dtype, device):
    """A caller-supplied tensor must have exactly this shape and dtype, be
    contiguous and sit on `device`: the library only sees its pointer and
    would write past the end of a short or mistyped buffer."""
    if not isinstance(t, _torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}, got {t.dtype} "
                         f"{tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    return t


def _check_workspace(t, name: str, need: int, device):
    """A workspace: a contiguous tensor on `device` of at least `need` bytes."""
    if not isinstance(t, _torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} must be a contiguous tensor on {device}")
    if t.numel() * t.element_size() < need:
        raise ValueError(f"{name} holds {t.numel() * t.element_size()} bytes, {need} needed")
    return t


def _stream(dev):
    _LIB.fabft_set_stream(_raw_stream(dev.index))


def _outputs(q, B: int, H: int, Lq: int):
    """New o, resid and flags for the queries q."""
    dev = q.device
    return (_torch.empty_like(q), _torch.empty((B, H, Lq), dtype=_torch.float32, device=dev),
            _torch.empty((B, H, Lq), dtype=_torch.uint8, device=dev))


def attn_fwd(q, k, v, causal: bool = False, scale: float | None = None, check: bool = True,
             out=None):
    """Flash-ABFT forward. Returns (o, resid, flags) with check=True, else o.

    out: optional preallocated (o[, resid, flags]) tensors to write into.
    """
    B, H, Lq, Lk, d = _shape(q, k, v)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dev = q.device
    if out is not None:
        if len(out) not in (1, 3) or (check and len(out) != 3):
            raise ValueError("out must be (o,) with check=False, or (o, resid, flags)")
        o = _check_out(out[0], "out[0] (o)", q.shape, _torch.bfloat16, dev)
        if check:
            resid = _check_out(out[1], "out[1] (resid)", (B, H, Lq), _torch.float32, dev)
            flags = _check_out(out[2], "out[2] (flags)", (B, H, Lq), _torch.uint8, dev)
    elif check:
        o, resid, flags = _outputs(q, B, H, Lq)
    else:
        o = _torch.empty_like(q)
    _stream(dev)
    if not check:
        _check(_LIB.fabft_attn_fwd_nocheck(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                           B, H, Lq, Lk, d, int(bool(causal)), scale),
               "fabft_attn_fwd_nocheck")
        return o
    _check(_LIB.fabft_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                               resid.data_ptr(), flags.data_ptr(), B, H, Lq, Lk, d,
                               int(bool(causal)), scale), "fabft_attn_fwd")
    return o, resid, flags


def attn_fwd_twopass(q, k, v, causal: bool = False, scale: float | None = None, out=None):
    """Flash-ABFT checksum on Algorithm 1 (the row max in a first pass over
    the keys, then o, l and c with that fixed max). Returns (o, resid, flags)
    with the meaning of attn_fwd's. out: optional preallocated (o, resid,
    flags)."""
    B, H, Lq, Lk, d = _shape(q, k, v)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dev = q.device
    if out is not None:
        if len(out) != 3:
            raise ValueError("out must be (o, resid, flags)")
        o = _check_out(out[0], "out[0] (o)", q.shape, _torch.bfloat16, dev)
        resid = _check_out(out[1], "out[1] (resid)", (B, H, Lq), _torch.float32, dev)
        flags = _check_out(out[2], "out[2] (flags)", (B, H, Lq), _torch.uint8, dev)
    else:
        o, resid, flags = _outputs(q, B, H, Lq)
    _stream(dev)
    _check(_LIB.fabft_attn_fwd_twopass(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                       resid.data_ptr(), flags.data_ptr(), B, H, Lq, Lk, d,
                                       int(bool(causal)), scale), "fabft_attn_fwd_twopass")
    return o, resid, flags


@functools.lru_cache(maxsize=256)
def _splitkv_bytes(B: int, H: int, Lq: int, d: int, nsplit: int) -> int:
    """splitkv_workspace_bytes, remembered per shape (a pure function)."""
    return splitkv_workspace_bytes(B, H, Lq, d, nsplit)


def splitkv_workspace_bytes(B: int, H: int, Lq: int, d: int, nsplit: int) -> int:
    r = _load().fabft_splitkv_workspace_bytes(int(B), int(H), int(Lq), int(d), int(nsplit))
    _check(min(int(r), 0), "fabft_splitkv_workspace_bytes")
    return int(r)


def splitkv_default_splits(B: int, H: int, Lq: int, Lk: int, d: int) -> int:
    """A split count that gives the launch about 512 workgroups (two per CU),
    with at least 32 key tiles per split (shorter splits pay their start-up
    and merge too often) and at most 64 splits. Measured on decode shapes that
    fill the device, one to 64 queries over 8K-128K keys: it picks the fastest
    count or one within 1% of it. Over short caches of few heads attn_fwd_splitkv
    takes more."""
    n_qt = -(-Lq // query_tile(d))
    tiles = -(-Lk // key_tile(d))
    return max(1, min(64, -(-512 // (B * H * n_qt)), tiles // 32))


@functools.lru_cache(maxsize=256)
def _launch_splits(B: int, H: int, Lq: int, Lk: int, d: int) -> int:
    """Splits of a call that names none: splitkv_default_splits, and for short
    caches, where that leaves most CUs idle, as many more as give 128
    workgroups (one query row), or as fit on the 256 CUs at once (several rows,
    whose work per key is larger), of at least 4 key tiles each. Measured (both
    kernels, us, default -> this): one row, B=1 H=32 Lk=4097 d=128 26.4 -> 18.9,
    H=8 24.0 -> 15, H=16 d=256 42.2 -> 19.3; 16 rows, H=32 Lk=4097 45.8 -> 22.3; 64
    rows, H=8 Lk=8192 45.7 -> 20.6. A few workgroups more than CUs cost a second
    round: B=3 H=5, 4 rows, Lk=29014 d=128, 14 splits 57.5, 18 (270 workgroups) 88.5."""
    ns = splitkv_default_splits(B, H, Lq, Lk, d)
    wgs = B * H * -(-Lq // query_tile(d))
    tiles = -(-Lk // key_tile(d))
    return max(ns, min(64, -(-128 // wgs) if Lq == 1 else 256 // wgs, tiles // 4))


def attn_fwd_splitkv(q, k, v, causal: bool = False, scale: float | None = None,
                     nsplit: int | None = None, workspace=None, out=None):
    """Flash-ABFT forward with the keys split into nsplit ranges and a merge
    (for few queries over many keys). Returns (o, resid, flags). nsplit
    defaults to splitkv_default_splits(...), or more of them over a short
    cache. workspace: optional uint8 GPU tensor of at least
    splitkv_workspace_bytes(...) bytes (of splitkv_default_splits(...) without
    nsplit; a call takes more splits only if the workspace holds them, which
    splitkv_workspace_bytes(B, H, Lq, d, 64) always does)."""
    B, H, Lq, Lk, d = _shape(q, k, v)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dev = q.device
    if nsplit is None:
        nsplit = _launch_splits(B, H, Lq, Lk, d)
        # a workspace sized for the default count stays good for it
        if isinstance(workspace, _torch.Tensor) and \
                workspace.numel() * workspace.element_size() < \
                _splitkv_bytes(B, H, Lq, d, nsplit):
            nsplit = splitkv_default_splits(B, H, Lq, Lk, d)
    nsplit = int(nsplit)   # the sizes below are remembered by value
    need = _splitkv_bytes(B, H, Lq, d, nsplit)
    if workspace is None:
        workspace = _torch.empty(need, dtype=_torch.uint8, device=dev)
    _check_workspace(workspace, "workspace", need, dev)
    if out is not None:
        o, resid, flags = out
        _check_out(o, "out[0] (o)", q.shape, _torch.bfloat16, dev)
        _check_out(resid, "out[1] (resid)", (B, H, Lq), _torch.float32, dev)
        _check_out(flags, "out[2] (flags)", (B, H, Lq), _torch.uint8, dev)
    else:
        o, resid, flags = _outputs(q, B, H, Lq)
    _stream(dev)
    _check(_LIB.fabft_attn_fwd_splitkv(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                          resid.data_ptr(), flags.data_ptr(), B, H, Lq, Lk, d,
                                          int(bool(causal)), scale, nsplit,
                                          workspace.data_ptr(),
                                          workspace.numel() * workspace.element_size()),
           "fabft_attn_fwd_splitkv")
    return o, resid, flags


def recompute_flagged(q, k, v, o, resid, flags, causal: bool = False,
                      scale: float | None = None, max_retries: int = 2):
    """Re-run the checked forward on every head with a flagged row (in place,
    up to max_retries times each). Returns (n_recovered, n_persistent)."""
    import torch
    B, H, Lq, Lk, d = _shape(q, k, v)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    _check_out(o, "o", q.shape, torch.bfloat16, q.device)
    _check_out(resid, "resid", (B, H, Lq), torch.float32, q.device)
    _check_out(flags, "flags", (B, H, Lq), torch.uint8, q.device)
    hf = torch.empty(B * H, dtype=torch.uint8, device=q.device)
    # pinned (torch keeps and reuses it): the copy back needs no staging buffer
    hf_host = torch.empty(B * H, dtype=torch.uint8, pin_memory=True)
    nr, npers = ctypes.c_int(), ctypes.c_int()
    _stream(q.device)
    _check(_load().fabft_recompute_flagged(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                           resid.data_ptr(), flags.data_ptr(), B, H, Lq, Lk, d,
                                           int(bool(causal)), scale, hf.data_ptr(),
                                           hf_host.data_ptr(),
                                           int(max_retries), ctypes.byref(nr),
                                           ctypes.byref(npers)),
           "fabft_recompute_flagged")
    return nr.value, npers.value


def global_check(o, resid):
    """Per-head global check from attn_fwd's o and resid: returns (gsum [B, H]
    fp64 = sum of the row residuals, gflags [B, H] uint8)."""
    import torch
    _load()   # the checks below need it, and this may be a process's first call
    if o.dtype != torch.bfloat16 or not o.is_cuda or not o.is_contiguous() or o.dim() != 4:
        raise ValueError("o must be a contiguous bf16 [B, H, Lq, d] GPU tensor")
    B, H, Lq, d = o.shape
    _check_out(resid, "resid", (B, H, Lq), torch.float32, o.device)
    gsum = torch.empty((B, H), dtype=torch.float64, device=o.device)
    gflags = torch.empty((B, H), dtype=torch.uint8, device=o.device)
    _stream(o.device)
    _check(_load().fabft_global_check(o.data_ptr(), resid.data_ptr(), B, H, Lq, d,
                                      gsum.data_ptr(), gflags.data_ptr()), "fabft_global_check")
    return gsum, gflags


CACHE_TILE = 64


@dataclass(frozen=True, eq=False)
class Cache:
    """A key/value cache held in 4 bits (fabft_cache_bytes in include/fabft.h): `data` is the
    buffer, its layout the library's; `capacity` the slots per head, a multiple of CACHE_TILE.
    It keeps no lengths: each call is told them. cache_new makes one."""
    data: "torch.Tensor"   # noqa: F821  uint8 [B, H, capacity / 64, bytes of a tile]
    B: int
    H: int
    capacity: int
    d: int

    def __post_init__(self):
        n = int(_load().fabft_cache_bytes(self.B, self.H, self.capacity, self.d))
        _check(min(n, 0), "fabft_cache_bytes")
        t = self.data
        if not isinstance(t, _torch.Tensor) or t.dtype is not _torch.uint8 or not t.is_cuda or \
                not t.is_contiguous() or t.numel() != n:
            raise ValueError(f"data must be a contiguous uint8 GPU tensor of {n} bytes")


def cache_new(B: int, H: int, capacity: int, d: int, device="cuda") -> Cache:
    """An empty cache for B sequences of H key/value heads of d channels, with at least
    `capacity` slots (rounded up to a multiple of 64) per head."""
    B, H, d = int(B), int(H), int(d)
    capacity = -(-int(capacity) // CACHE_TILE) * CACHE_TILE
    n = int(_load().fabft_cache_bytes(B, H, capacity, d))
    _check(min(n, 0), "fabft_cache_bytes")
    tiles = capacity // CACHE_TILE
    data = _torch.zeros((B, H, tiles, n // (B * H * tiles)), dtype=_torch.uint8, device=device)
    return Cache(data, B, H, capacity, d)


def _device_of(c, name: str = "cache"):
    if not isinstance(c, Cache):
        raise TypeError(f"{name} must be a Cache (cache_new), got {type(c).__name__}")
    return c.data.device


def _at(t, name: str, shape, dtype, device):
    """The address of a tensor that has to be as _check_out says; None for None."""
    if t is None:
        return None
    if not (isinstance(t, _torch.Tensor) and t.dtype is dtype and t.shape == shape and
            t.device == device and t.is_contiguous()):
        _check_out(t, name, shape, dtype, device)
    return t.data_ptr()


def _needed(t, name: str):
    if t is None:
        raise ValueError(f"{name} must be a torch tensor")
    return t


def _call(dev, name: str, f, *args):
    """An entry point on dev's current stream, with dev current while it runs: a kernel
    goes to the device that is current, also on the null stream."""
    if _torch._C._cuda_getDevice() == dev.index:
        _LIB.fabft_set_stream(_raw_stream(dev.index))
        rc = f(*args)
    else:
        with _torch.cuda.device(dev):
            _LIB.fabft_set_stream(_raw_stream(dev.index))
            rc = f(*args)
    if rc:
        _check(rc, name)


@functools.lru_cache(maxsize=64)
def _strides(*st):
    return (ctypes.c_longlong * 6)(*st)


def _check_rows(c, t, name: str, dev):
    """New rows [B, H, n, d]. Returns n."""
    if not isinstance(t, _torch.Tensor) or t.dtype is not _torch.bfloat16:
        raise TypeError(f"{name} must be a torch.bfloat16 tensor")
    s = t.shape
    if len(s) != 4 or s[0] != c.B or s[1] != c.H or s[3] != c.d:
        raise ValueError(f"{name} must be [B={c.B}, H={c.H}, n, d={c.d}], got {tuple(s)}")
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")
    if t.stride(3) != 1:
        raise ValueError(f"{name}: the channels must be contiguous")
    return s[2]


def cache_append(cache: Cache, k, v, start, counts=None):
    """Quantise the rows of k and v (bfloat16 [B, H, n, d]; any strides over B, H and n that are
    multiples of 8 elements) into slots start[b] + i of the cache; with counts, of rows
    i < counts[b] only. start, counts: int32 [B] on the GPU. Rows whose slot is not in
    [0, capacity) are dropped."""
    c, dev = cache, _device_of(cache)
    n, nv = _check_rows(c, k, "k", dev), _check_rows(c, v, "v", dev)
    if n != nv:
        raise ValueError(f"shape mismatch: k {tuple(k.shape)} v {tuple(v.shape)}")
    st = None
    if not (k.is_contiguous() and v.is_contiguous()):
        # (0 along a size of 1, whose stride is of no account)
        st = _strides(*(0 if t.shape[i] == 1 else t.stride(i) for t in (k, v) for i in range(3)))
    i32, B = _torch.int32, (c.B,)
    at = _at(_needed(start, "start"), "start", B, i32, dev)
    cnt = _at(counts, "counts", B, i32, dev)
    if n:
        _call(dev, "fabft_cache_append", _LIB.fabft_cache_append, c.data.data_ptr(), c.B, c.H,
              c.capacity, c.d, k.data_ptr(), v.data_ptr(), n, st, at, cnt)


def cache_read(cache: Cache, start, n: int, counts=None, out=None):
    """The values of slots start[b] .. start[b] + n - 1 as (k, v), bfloat16 [B, H, n, d] (exact:
    the cache's values are bfloat16 numbers); zeros for rows i >= counts[b] and outside the
    cache. out: optional preallocated (k, v)."""
    c, dev, n = cache, _device_of(cache), int(n)
    if n < 0:
        raise ValueError("n must be >= 0")
    i32, B = _torch.int32, (c.B,)
    at = _at(_needed(start, "start"), "start", B, i32, dev)
    cnt = _at(counts, "counts", B, i32, dev)
    shape = (c.B, c.H, n, c.d)
    if out is not None:
        if len(out) != 2:
            raise ValueError("out must be (k, v)")
        k = _check_out(out[0], "out[0] (k)", shape, _torch.bfloat16, dev)
        v = _check_out(out[1], "out[1] (v)", shape, _torch.bfloat16, dev)
    else:
        k = _torch.empty(shape, dtype=_torch.bfloat16, device=dev)
        v = _torch.empty_like(k)
    if n:
        _call(dev, "fabft_cache_read", _LIB.fabft_cache_read, c.data.data_ptr(), c.B, c.H, c.capacity,
              c.d, k.data_ptr(), v.data_ptr(), n, at, cnt)
    return k, v


def cache_splits(B: int, H: int, G: int, Lq: int, capacity: int) -> int:
    """The split count of attn_fwd_cache calls that name none."""
    r = _load().fabft_cache_splits(int(B), int(H), int(G), int(Lq), int(capacity))
    _check(min(r, 0), "fabft_cache_splits")
    return r


def cache_workspace_bytes(B: int, H: int, G: int, Lq: int, d: int, nsplit: int,
                          with_weight: bool = False) -> int:
    r = int(_load().fabft_cache_workspace_bytes(int(B), int(H), int(G), int(Lq), int(d), int(nsplit),
                                                int(bool(with_weight))))
    _check(min(r, 0), "fabft_cache_workspace_bytes")
    return r


@functools.lru_cache(maxsize=256)
def _cache_plan(B: int, H: int, G: int, Lq: int, capacity: int, d: int, nsplit: int | None,
                with_weight: bool):
    """(splits, workspace bytes) of a call, remembered per shape (a pure function)."""
    if nsplit is None:
        nsplit = cache_splits(B, H, G, Lq, capacity)
    return nsplit, cache_workspace_bytes(B, H, G, Lq, d, nsplit, with_weight)


def attn_fwd_cache(q, cache: Cache, lengths, counts=None, causal: bool = False,
                   scale: float | None = None, weight=None, decay: float = 1.0,
                   nsplit: int | None = None, workspace=None, out=None):
    """Flash-ABFT forward over the 4-bit cache. q: bfloat16 [B, H * G, Lq, d], contiguous, G query
    heads per key/value head. lengths: int32 [B] on the GPU, the keys of each sequence; counts:
    int32 [B], its query rows (the others are padding: O = 0, no flag). causal: the query rows are
    the last counts[b] keys. Returns (o, resid, flags) as attn_fwd; where a row's number of keys times
    the largest sum of |v| over a row of V passes 2^118, its sums can overflow (FLAG_NONFINITE).

    weight: optional fp32 [B, H, capacity], updated in place: decay * weight + the softmax weights
    of each key summed over the rows of its group (decay 0 overwrites; rows with a flag add nothing;
    slots from lengths[b] on stay as they were). nsplit: ranges of the keys, by default
    cache_splits(...). workspace: optional GPU tensor of cache_workspace_bytes(...) bytes. out:
    optional preallocated (o, resid, flags); o must not overlap q."""
    c, dev = cache, _device_of(cache)
    if not isinstance(q, _torch.Tensor) or q.dtype is not _torch.bfloat16:
        raise TypeError("q must be a torch.bfloat16 tensor")
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [B, H * G, Lq, d] tensor")
    if q.device != dev:
        raise ValueError(f"q must be on {dev}, got {q.device}")
    B, HG, Lq, d = q.shape
    H = c.H
    G = HG // H
    if B != c.B or d != c.d or G < 1 or G * H != HG:
        raise ValueError(f"shape mismatch: q {tuple(q.shape)}, cache B={c.B} H={c.H} d={c.d}")
    i32, f32 = _torch.int32, _torch.float32
    lens = _at(_needed(lengths, "lengths"), "lengths", (B,), i32, dev)
    cnt = _at(counts, "counts", (B,), i32, dev)
    wt = _at(weight, "weight", (B, H, c.capacity), f32, dev)
    nsplit, need = _cache_plan(B, H, G, Lq, c.capacity, d, None if nsplit is None else int(nsplit),
                               weight is not None)
    ws, size = None, 0
    if workspace is not None:
        _check_workspace(workspace, "workspace", need, dev)
        ws, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    elif need:
        workspace = _torch.empty(need, dtype=_torch.uint8, device=dev)
        ws, size = workspace.data_ptr(), need
    if out is not None:
        if len(out) != 3:
            raise ValueError("out must be (o, resid, flags)")
        o = _check_out(out[0], "out[0] (o)", q.shape, _torch.bfloat16, dev)
        resid = _check_out(out[1], "out[1] (resid)", (B, HG, Lq), f32, dev)
        flags = _check_out(out[2], "out[2] (flags)", (B, HG, Lq), _torch.uint8, dev)
        if abs(o.data_ptr() - q.data_ptr()) < 2 * q.numel():
            raise ValueError("out[0] (o) must not overlap q")
    else:
        o, resid, flags = _outputs(q, B, HG, Lq)
    _call(dev, "fabft_attn_fwd_cache", _LIB.fabft_attn_fwd_cache, q.data_ptr(), c.data.data_ptr(),
          o.data_ptr(), resid.data_ptr(), flags.data_ptr(), B, H, G, Lq, c.capacity, d, lens, cnt,
          1 if causal else 0, 1.0 / math.sqrt(d) if scale is None else float(scale), wt, float(decay),
          nsplit, ws, size)
    return o, resid, flags


def cache_evict(cache: Cache, weight, lengths, keep: int, recent: int = 0, into: Cache | None = None,
                into_weight=None):
    """Keep min(lengths[b], keep) slots of every head: the last `recent` ones and those of the
    others with the largest weight (fp32 [B, H, capacity]; equal ones: the lowest slot). They move,
    in their order, to the first slots of the cache, their weights with them (0 behind them); with
    into and into_weight, of another cache, and this one stays as it was. Returns (index int32
    [B, H, keep], each place's former slot, -1 behind the last; new lengths int32 [B])."""
    c, dev = cache, _device_of(cache)
    i32, f32 = _torch.int32, _torch.float32
    wt = _at(_needed(weight, "weight"), "weight", (c.B, c.H, c.capacity), f32, dev)
    lens = _at(_needed(lengths, "lengths"), "lengths", (c.B,), i32, dev)
    if (into is None) != (into_weight is None):
        raise ValueError("into and into_weight go together")
    if into is None:
        into, iw = c, wt
    else:
        if _device_of(into, "into") != dev or (into.B, into.H, into.d) != (c.B, c.H, c.d):
            raise ValueError("into must have the cache's B, H, d and device")
        iw = _at(into_weight, "into_weight", (c.B, c.H, into.capacity), f32, dev)
    keep, recent = int(keep), int(recent)
    if not 1 <= keep <= into.capacity or not 0 <= recent <= keep:
        raise ValueError(f"keep must be 1..{into.capacity} and recent 0..keep, got {keep}, {recent}")
    index = _torch.empty((c.B, c.H, keep), dtype=i32, device=dev)
    new = _torch.empty((c.B,), dtype=i32, device=dev)
    _call(dev, "fabft_cache_evict", _LIB.fabft_cache_evict, c.data.data_ptr(), c.B, c.H, c.capacity,
          c.d, wt, lens, keep, recent, into.data.data_ptr(), into.capacity, iw, index.data_ptr(),
          new.data_ptr())
    return index, new


@dataclass
class Fault:
    """One single-bit fault for attn_fwd_inject (fields as in fabft_fault)."""
    site: str          # "S", "P", "O", "V", "C", "L", "M", "Q", "VS" or "none"
    b: int = 0
    h: int = 0
    row: int = 0
    col: int = 0
    tile: int = 0
    bit: int = 0

    def to_c(self) -> FabftFault:
        return FabftFault(SITES[self.site], self.b, self.h, self.row, self.col, self.tile,
                          self.bit)


def _faults_array(fault):
    faults = [] if fault is None else ([fault] if isinstance(fault, Fault) else list(fault))
    if len(faults) > MAX_FAULTS:
        raise ValueError(f"at most {MAX_FAULTS} faults per launch")
    return (FabftFault * max(1, len(faults)))(*[f.to_c() for f in faults]), len(faults)


def attn_fwd_debug(q, k, v, causal: bool = False, scale: float | None = None, fault=None,
                   outputs=("pred", "actual", "pred_w", "actual_w", "score_lhs",
                            "score_rhs", "score_bound")):
    """Debug / fault-injection forward with the debug outputs named in
    `outputs` (see fabft_debug_out). Returns a dict with o, resid, flags and
    one fp32 [B, H, Lq] tensor per requested output."""
    import torch
    B, H, Lq, Lk, d = _shape(q, k, v)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dev = q.device
    res = {"o": torch.empty_like(q),
           "resid": torch.empty((B, H, Lq), dtype=torch.float32, device=dev),
           "flags": torch.empty((B, H, Lq), dtype=torch.uint8, device=dev)}
    dbg = FabftDebugOut()
    for name in outputs:
        if name not in dict(FabftDebugOut._fields_):
            raise ValueError(f"unknown debug output {name!r}")
        res[name] = torch.empty((B, H, Lq), dtype=torch.float32, device=dev)
        setattr(dbg, name, res[name].data_ptr())
    arr, n = _faults_array(fault)
    _stream(dev)
    _check(_load().fabft_attn_fwd_debug(q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                        res["o"].data_ptr(), res["resid"].data_ptr(),
                                        res["flags"].data_ptr(), B, H, Lq, Lk, d,
                                        int(bool(causal)), scale, arr, n, ctypes.byref(dbg)),
           "fabft_attn_fwd_debug")
    return res


def attn_fwd_inject(q, k, v, causal: bool = False, scale: float | None = None,
                    fault=None, out=None, weighted_out: bool = False):
    """Debug / fault-injection forward. fault: None, one Fault, or a list of
    up to MAX_FAULTS Faults applied in the same launch. Returns (o, resid,
    flags, pred, actual), followed by (pred_w, actual_w) with weighted_out=True.
    out: optional preallocated (o, resid, flags, pred, actual)."""
    import torch
    B, H, Lq, Lk, d = _shape(q, k, v)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dev = q.device
    if out is None:
        o = torch.empty_like(q)
        resid = torch.empty((B, H, Lq), dtype=torch.float32, device=dev)
        flags = torch.empty((B, H, Lq), dtype=torch.uint8, device=dev)
        pred = torch.empty((B, H, Lq), dtype=torch.float32, device=dev)
        actual = torch.empty((B, H, Lq), dtype=torch.float32, device=dev)
    else:
        if len(out) != 5:
            raise ValueError("out must be (o, resid, flags, pred, actual)")
        o, resid, flags, pred, actual = out
        _check_out(o, "out[0] (o)", q.shape, torch.bfloat16, dev)
        _check_out(resid, "out[1] (resid)", (B, H, Lq), torch.float32, dev)
        _check_out(flags, "out[2] (flags)", (B, H, Lq), torch.uint8, dev)
        _check_out(pred, "out[3] (pred)", (B, H, Lq), torch.float32, dev)
        _check_out(actual, "out[4] (actual)", (B, H, Lq), torch.float32, dev)
    pw = aw = None
    if weighted_out:
        pw = torch.empty((B, H, Lq), dtype=torch.float32, device=dev)
        aw = torch.empty((B, H, Lq), dtype=torch.float32, device=dev)
    arr, n = _faults_array(fault)
    _stream(dev)
    _check(_load().fabft_attn_fwd_inject_n(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                        resid.data_ptr(), flags.data_ptr(), B, H, Lq, Lk, d,
                                        int(bool(causal)), scale, arr, n,
                                        pred.data_ptr(), actual.data_ptr(),
                                        pw.data_ptr() if pw is not None else None,
                                        aw.data_ptr() if aw is not None else None),
           "fabft_attn_fwd_inject_n")
    if weighted_out:
        return o, resid, flags, pred, actual, pw, aw
    return o, resid, flags, pred, actual


__all__ = ["attn_fwd", "attn_fwd_twopass", "attn_fwd_inject", "attn_fwd_debug", "attn_fwd_splitkv", "splitkv_workspace_bytes",
           "splitkv_default_splits",
           "Cache", "CACHE_TILE", "cache_new", "cache_append", "cache_read", "cache_splits",
           "cache_workspace_bytes", "attn_fwd_cache", "cache_evict",
           "global_check", "recompute_flagged", "Fault", "FabftError", "set_threshold",
           "set_score_check", "score_check_workspace_bytes", "get_score_threshold",
           "get_threshold", "set_weighted_check", "get_weighted_check", "set_persistent",
           "get_persistent", "set_algorithm", "get_algorithm", "key_tile",
           "query_tile", "status_str", "lib", "LIB_PATH", "EXPORTS", "MAX_FAULTS", "FLAG_RESID",
           "FLAG_NONFINITE", "FLAG_WEIGHTED", "FLAG_SCORES", "PERSIST_OFF", "PERSIST_AUTO",
           "PERSIST_ALWAYS"]
