"""GB300 (sm_103a) ValueDiff KV-cache eviction: Python binding of libvd.so.

A thin ctypes layer over the C ABI in ``include/vd.h``, with the same names.
It only marshals arguments -- torch tensors in, device pointers and the
caller's CUDA stream out -- and checks dtypes, devices and shapes so that no
wrong pointer reaches the library.  Every step of the eviction runs in the
CUDA kernels of ``csrc/``; there is no CPU or PyTorch fallback: if
``libvd.so`` has not been built, every call raises.

The method (paper: ValueDiff, Sec. 3.2 Eq. vd; Sec. 2.1 Eq. eviction;
Sec. 2.2 Eq. block_processing): per (sequence, layer, KV head), score each
cached token by ||v_j - mean(V)||_2 (or the Dir / Norm variants), keep the N
highest scores (ties to the lower slot) and compact K and V in place.
"""
from __future__ import annotations

import ctypes
import os
import threading

__all__ = [
    "VD_SCORE_L2", "VD_SCORE_DIR", "VD_SCORE_NORM", "VD_MU_RECOMPUTE", "VD_MU_RUNNING",
    "VdError", "Cache", "vd_score", "vd_score_ex", "vd_evict_block", "vd_evict_block_ex",
    "vd_append_evict_block", "vd_append_evict_block_ex", "vd_append_evict_decode",
    "vd_evict_decode",
    "vd_evict_block_holefill", "vd_evict_decode_holefill", "vd_append",
    "vd_running_sum_init", "vd_running_sum_init_ex", "vd_workspace_size", "vd_status_string",
    "vd_get_device_status",
    "Q4Cache", "vd_q4_append", "vd_q4_pack", "vd_q4_unpack", "vd_q4_attend", "vd_qkv_norm_rope",
    "VD_PAGED_BF16", "VD_PAGED_E4M3", "PagedCache", "vd_paged_append", "vd_paged_attend",
    "vd_paged_attend_workspace", "vd_paged_advance", "vd_paged_pack", "vd_paged_unpack",
    "library_path", "load_library",
]

VD_SCORE_L2, VD_SCORE_DIR, VD_SCORE_NORM = 0, 1, 2
VD_MU_RECOMPUTE, VD_MU_RUNNING = 0, 1
VD_PAGED_BF16, VD_PAGED_E4M3 = 0, 1
VARIANTS = {"l2": VD_SCORE_L2, "dir": VD_SCORE_DIR, "norm": VD_SCORE_NORM}

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libvd.so")
_lib = None
_lock = threading.Lock()


class VdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {vd_status_string(code)} (status {code})")


class _VdCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("n_seq", ctypes.c_int32), ("n_layer", ctypes.c_int32),
                ("n_kv_head", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity", ctypes.c_int32)]


class _VdQ4Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("len", ctypes.c_void_p), ("n_seq", ctypes.c_int32),
                ("n_layer", ctypes.c_int32), ("n_kv_head", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("capacity", ctypes.c_int32)]


class _VdPagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
                ("len", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("slot_stride", ctypes.c_int64), ("type", ctypes.c_int32),
                ("n_seq", ctypes.c_int32), ("n_layer", ctypes.c_int32),
                ("n_kv_head", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_page", ctypes.c_int32),
                ("max_pages", ctypes.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load the in-tree libvd.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_LIB_PATH):
                raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                                   "paper_2609_23314_gb300.build.build() (nvcc, sm_103a)")
            lib = ctypes.CDLL(_LIB_PATH)
            P, I32, S = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int
            cp = ctypes.POINTER(_VdCache)
            lib.vd_score.argtypes = [cp, S, P, P]
            lib.vd_evict_block.argtypes = [cp, I32, P, I32, S, S, P, P, P, P]
            lib.vd_append_evict_block.argtypes = [cp, P, P, I32, I32, P, S, S, P, P, P, P, P, P]
            lib.vd_append_evict_decode.argtypes = [cp, P, P, I32, P, S, S, P, P, P, P, P, P, P]
            lib.vd_evict_decode.argtypes = [cp, I32, P, S, S, P, P, P, P, P]
            lib.vd_evict_block_holefill.argtypes = [cp, I32, P, I32, S, S, P, P, P, P, P, P]
            lib.vd_evict_decode_holefill.argtypes = [cp, I32, P, S, S, P, P, P, P, P, P, P]
            lib.vd_score_ex.argtypes = [cp, S, S, P, I32, P, P, P]
            lib.vd_evict_block_ex.argtypes = [cp, I32, P, I32, S, S, P, I32, P, P, P, P, P]
            lib.vd_append_evict_block_ex.argtypes = [cp, P, P, I32, I32, P, S, S, P, I32, P, P, P,
                                                     P, P]
            lib.vd_append.argtypes = [cp, P, P, I32, P]
            lib.vd_running_sum_init.argtypes = [cp, P, P]
            lib.vd_running_sum_init_ex.argtypes = [cp, I32, P, P]
            qp, F = ctypes.POINTER(_VdQ4Cache), ctypes.c_float
            lib.vd_q4_append.argtypes = [qp, P, P, I32, P]
            lib.vd_q4_pack.argtypes = [qp, I32, cp, P]
            lib.vd_q4_unpack.argtypes = [qp, I32, cp, P]
            lib.vd_q4_attend.argtypes = [qp, I32, P, I32, P, P, I32, F, P, P, P]
            lib.vd_qkv_norm_rope.argtypes = [P, I32, I32, I32, I32, I32, P, P, F, P, I32, I32, P,
                                             P, P, P, I32, I32, P]
            pp, Z = ctypes.POINTER(_VdPagedCache), ctypes.c_size_t
            lib.vd_paged_append.argtypes = [pp, I32, P, I32, I32, P, P, P, F, P, I32, I32, P, P, P]
            lib.vd_paged_attend.argtypes = [pp, I32, P, I32, I32, P, I32, F, P, P, P, Z, P]
            lib.vd_paged_attend_workspace.argtypes = [pp, I32, I32]
            lib.vd_paged_attend_workspace.restype = Z
            lib.vd_paged_advance.argtypes = [pp, P, I32, P]
            lib.vd_paged_pack.argtypes = [pp, I32, cp, P]
            lib.vd_paged_unpack.argtypes = [pp, I32, cp, P]
            lib.vd_workspace_size.argtypes = [cp]
            lib.vd_workspace_size.restype = ctypes.c_size_t
            lib.vd_status_string.argtypes = [S]
            lib.vd_status_string.restype = ctypes.c_char_p
            lib.vd_get_device_status.argtypes = [P]
            for f in ("vd_score", "vd_score_ex", "vd_evict_block_ex", "vd_evict_block",
                      "vd_append_evict_block", "vd_append_evict_block_ex", "vd_append_evict_decode",
                      "vd_evict_decode", "vd_evict_block_holefill",
                      "vd_evict_decode_holefill", "vd_append", "vd_running_sum_init",
                      "vd_running_sum_init_ex", "vd_q4_append", "vd_q4_pack", "vd_q4_unpack",
                      "vd_q4_attend", "vd_qkv_norm_rope", "vd_paged_append", "vd_paged_attend",
                      "vd_paged_advance", "vd_paged_pack", "vd_paged_unpack",
                      "vd_get_device_status"):
                getattr(lib, f).restype = S
            _lib = lib
        return _lib


# ---------------------------------------------------------------------------
# marshalling helpers
# ---------------------------------------------------------------------------
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _stream(stream):
    if stream is None:
        # the current stream of the current device as a raw handle:
        # torch.cuda.current_stream() builds a Stream object for it, 3.2 us of
        # a call that takes 9 on the device (0.3 us this way)
        torch = _torch()
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None or not torch.cuda.is_initialized():
            return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        return raw(torch._C._cuda_getDevice())
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t, dtype, shape, what, device):
    """The tensor's device pointer after checking its type, device, layout
    and shape (so that no wrong pointer reaches the library)."""
    if t is None:
        return None
    try:
        if (t.dtype is dtype and t.get_device() == device.index and t.is_contiguous()
                and t.shape == shape):
            return t.data_ptr()
        where, contiguous, got = t.device, t.is_contiguous(), t.shape
    except AttributeError:
        raise TypeError(f"{what} must be a torch tensor") from None
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if where != device:
        raise ValueError(f"{what} must live on {device}, got {where}")
    if not contiguous:
        raise ValueError(f"{what} must be contiguous")
    if got != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(got)}")
    return t.data_ptr()  # a CPU tensor of a CPU cache, which ref() refuses


def _check(code: int, where: str):
    if code != 0:
        raise VdError(code, where)


def _on_gpu(device):
    """Refuses tensors that are not on a GPU: the library takes every address for a device
    one, and a kernel would follow it into host memory."""
    if device.type != "cuda":
        raise ValueError(f"the tensors of a call must live on a CUDA device, got {device}")


class Cache:
    """A KV cache in the library's layout: K and V bf16
    [n_seq, n_layer, n_kv_head, capacity, head_dim] and len int32 [n_seq],
    all on one CUDA device.  Holds references to the tensors only."""

    def __init__(self, k, v, len):
        torch = _torch()
        if k.dim() != 5 or k.shape != v.shape:
            raise ValueError("k and v must both be [n_seq, n_layer, n_kv_head, capacity, head_dim]")
        self.k, self.v, self.len = k, v, len
        self.n_seq, self.n_layer, self.n_kv_head, self.capacity, self.head_dim = (int(x) for x in k.shape)
        self.device = k.device
        _ptr(k, torch.bfloat16, k.shape, "k", self.device)
        _ptr(v, torch.bfloat16, k.shape, "v", self.device)
        _ptr(len, torch.int32, (self.n_seq,), "len", self.device)
        self._s = _VdCache(k.data_ptr(), v.data_ptr(), len.data_ptr(), self.n_seq, self.n_layer,
                           self.n_kv_head, self.head_dim, self.capacity)
        self._ref = ctypes.byref(self._s)
        self._gpu = self.device.type == "cuda"
        self._unit_shape = (self.n_seq, self.n_layer, self.n_kv_head)

    @classmethod
    def empty(cls, n_seq, n_layer, n_kv_head, capacity, head_dim, device="cuda"):
        torch = _torch()
        shape = (n_seq, n_layer, n_kv_head, capacity, head_dim)
        return cls(torch.zeros(shape, dtype=torch.bfloat16, device=device),
                   torch.zeros(shape, dtype=torch.bfloat16, device=device),
                   torch.zeros(n_seq, dtype=torch.int32, device=device))

    @property
    def units(self) -> int:
        return self.n_seq * self.n_layer * self.n_kv_head

    def unit_shape(self):
        return self._unit_shape

    def ref(self):
        """What a call hands to the library; a cache that is not on a GPU is refused."""
        if not self._gpu:
            _on_gpu(self.device)
        return self._ref


class Q4Cache:
    """A KV cache in 4 bits (format: vd_q4_cache in ``include/vd.h``): codes uint8
    [n_seq, n_layer, n_kv_head, capacity, head_dim / 2], scales uint8 [..., head_dim / 16]
    and len int32 [n_seq], all on one CUDA device.  head_dim is a multiple of 32 (at most
    256), capacity a multiple of 8.  Holds references to the tensors only."""

    def __init__(self, k, v, k_scale, v_scale, len):
        torch = _torch()
        if k.dim() != 5:
            raise ValueError("k must be [n_seq, n_layer, n_kv_head, capacity, head_dim / 2]")
        self.k, self.v, self.k_scale, self.v_scale, self.len = k, v, k_scale, v_scale, len
        self.n_seq, self.n_layer, self.n_kv_head, self.capacity = (int(x) for x in k.shape[:4])
        self.head_dim = 2 * int(k.shape[4])
        self.device = k.device
        scales = tuple(k.shape[:4]) + (self.head_dim // 16,)
        _ptr(k, torch.uint8, k.shape, "k", self.device)
        _ptr(v, torch.uint8, k.shape, "v", self.device)
        _ptr(k_scale, torch.uint8, scales, "k_scale", self.device)
        _ptr(v_scale, torch.uint8, scales, "v_scale", self.device)
        _ptr(len, torch.int32, (self.n_seq,), "len", self.device)
        self._s = _VdQ4Cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                             len.data_ptr(), self.n_seq, self.n_layer, self.n_kv_head,
                             self.head_dim, self.capacity)
        self._ref = ctypes.byref(self._s)
        self._gpu = self.device.type == "cuda"
        self._unit_shape = (self.n_seq, self.n_layer, self.n_kv_head)

    @classmethod
    def empty(cls, n_seq, n_layer, n_kv_head, capacity, head_dim, device="cuda"):
        torch = _torch()
        shape = (n_seq, n_layer, n_kv_head, capacity)
        codes, scales = ([torch.zeros(shape + (head_dim // k,), dtype=torch.uint8, device=device)
                          for _ in range(2)] for k in (2, 16))
        return cls(codes[0], codes[1], scales[0], scales[1],
                   torch.zeros(n_seq, dtype=torch.int32, device=device))

    @property
    def units(self) -> int:
        return self.n_seq * self.n_layer * self.n_kv_head

    def unit_shape(self):
        return self._unit_shape

    def ref(self):
        """What a call hands to the library; a cache that is not on a GPU is refused."""
        if not self._gpu:
            _on_gpu(self.device)
        return self._ref


class PagedCache:
    """A KV cache in pages (layout: vd_paged_cache in ``include/vd.h``): K and V bf16 or
    float8_e4m3fn [n_layer, n_page, n_kv_head, page_size, head_dim], of equal strides and with
    rows that lie together (a transposed [n_layer, n_page, page_size, n_kv_head, head_dim] is
    one), the page table int32 [n_seq, max_pages], len int32 [n_seq] and, for float8 pages,
    scales fp32 [n_layer, n_kv_head] (or None: 1); all on one CUDA device.  Holds references to
    the tensors only."""

    def __init__(self, k, v, page_table, len, k_scale=None, v_scale=None):
        torch = _torch()
        if k.dim() != 5 or page_table.dim() != 2:
            raise ValueError("k must be [n_layer, n_page, n_kv_head, page_size, head_dim], page_table "
                             "[n_seq, max_pages]")
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            raise TypeError(f"k must be torch.bfloat16 or torch.float8_e4m3fn, got {k.dtype}")
        self.k, self.v, self.page_table, self.len = k, v, page_table, len
        self.k_scale, self.v_scale = k_scale, v_scale
        (self.n_layer, self.n_page, self.n_kv_head, self.page_size,
         self.head_dim) = (int(x) for x in k.shape)
        self.n_seq, self.max_pages = (int(x) for x in page_table.shape)
        self.device = k.device
        self.type = VD_PAGED_BF16 if k.dtype == torch.bfloat16 else VD_PAGED_E4M3
        if v.dtype != k.dtype:
            raise TypeError(f"v must be {k.dtype}, got {v.dtype}")
        if v.device != k.device:
            raise ValueError(f"v must live on {k.device}, got {v.device}")
        if v.shape != k.shape:
            raise ValueError(f"v must have shape {tuple(k.shape)}, got {tuple(v.shape)}")
        for d, (n, sk, sv) in enumerate(zip(k.shape, k.stride(), v.stride())):
            if n > 1 and (sk != sv or (d == 4 and sk != 1)):
                raise ValueError("k and v must have equal strides, and rows that lie together")
        _ptr(page_table, torch.int32, page_table.shape, "page_table", self.device)
        _ptr(len, torch.int32, (self.n_seq,), "len", self.device)
        scales = (self.n_layer, self.n_kv_head)
        s = [_ptr(x, torch.float32, scales, name, self.device)
             for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale"))]
        self._s = _VdPagedCache(k.data_ptr(), v.data_ptr(), s[0], s[1], page_table.data_ptr(),
                                len.data_ptr(), *k.stride()[:4], self.type, self.n_seq,
                                self.n_layer, self.n_kv_head, self.head_dim, self.page_size,
                                self.n_page, self.max_pages)
        self._ref = ctypes.byref(self._s)
        self._gpu = self.device.type == "cuda"
        self._vector = (self.n_seq,)

    @classmethod
    def empty(cls, n_seq, n_layer, n_kv_head, head_dim, n_page, page_size, max_pages, dtype=None,
              device="cuda"):
        """A cache of zeros without a page: page_table is all -1."""
        torch = _torch()
        shape = (n_layer, n_page, n_kv_head, page_size, head_dim)
        k, v = (torch.zeros(shape, dtype=dtype or torch.bfloat16, device=device) for _ in range(2))
        return cls(k, v, torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_seq, dtype=torch.int32, device=device))

    def ref(self):
        """What a call hands to the library; a cache that is not on a GPU is refused."""
        if not self._gpu:
            _on_gpu(self.device)
        return self._ref


# ---------------------------------------------------------------------------
# the C ABI, same names
# ---------------------------------------------------------------------------
def vd_score(cache: Cache, variant: int, scores_out, stream=None) -> None:
    torch = _torch()
    sc = _ptr(scores_out, torch.float32, cache.unit_shape() + (cache.capacity,), "scores_out", cache.device)
    _check(load_library().vd_score(cache.ref(), int(variant), sc, _stream(stream)), "vd_score")


def vd_evict_block(cache: Cache, N: int, N_dev=None, B: int = 0, variant: int = VD_SCORE_L2,
                   mu: int = VD_MU_RECOMPUTE, running_sum=None, kept_idx_out=None,
                   scores_out=None, stream=None) -> None:
    torch = _torch()
    us = cache.unit_shape()
    args = (
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
    )
    _check(load_library().vd_evict_block(cache.ref(), int(N), args[0], int(B), int(variant), int(mu),
                                         args[1], args[2], args[3], _stream(stream)),
           "vd_evict_block")


def vd_append_evict_block(cache: Cache, k_new, v_new, B: int, N: int, N_dev=None,
                          variant: int = VD_SCORE_L2, mu: int = VD_MU_RECOMPUTE,
                          running_sum=None, kept_idx_out=None, scores_out=None,
                          stream=None, pos=None, pos_first_new=None) -> None:
    """vd_append followed by vd_evict_block (or, with pos and pos_first_new,
    vd_evict_block_holefill) in one launch; k_new, v_new: bf16
    [n_seq, n_layer, n_kv_head, B, head_dim], read straight from the caller's
    buffers (only surviving rows are written into the cache)."""
    torch = _torch()
    us = cache.unit_shape()
    shape = us + (int(B), cache.head_dim)
    args = (
        _ptr(k_new, torch.bfloat16, shape, "k_new", cache.device),
        _ptr(v_new, torch.bfloat16, shape, "v_new", cache.device),
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
        _ptr(pos, torch.int32, us + (cache.capacity,), "pos", cache.device),
        _ptr(pos_first_new, torch.int32, (cache.n_seq,), "pos_first_new", cache.device),
    )
    _check(load_library().vd_append_evict_block(cache.ref(), args[0], args[1], int(B), int(N),
                                                args[2], int(variant), int(mu), args[3],
                                                args[6], args[7], args[4], args[5],
                                                _stream(stream)),
           "vd_append_evict_block")


def vd_append_evict_decode(cache: Cache, k_new, v_new, N: int, N_dev=None,
                           variant: int = VD_SCORE_L2, mu: int = VD_MU_RECOMPUTE,
                           running_sum=None, evicted_out=None, kept_idx_out=None,
                           scores_out=None, stream=None, pos=None, pos_first_new=None) -> None:
    """vd_append of one token followed by vd_evict_decode (or, with pos and
    pos_first_new, vd_evict_decode_holefill) in one launch; k_new, v_new:
    bf16 [n_seq, n_layer, n_kv_head, 1, head_dim]."""
    torch = _torch()
    us = cache.unit_shape()
    shape = us + (1, cache.head_dim)
    args = (
        _ptr(k_new, torch.bfloat16, shape, "k_new", cache.device),
        _ptr(v_new, torch.bfloat16, shape, "v_new", cache.device),
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(pos, torch.int32, us + (cache.capacity,), "pos", cache.device),
        _ptr(pos_first_new, torch.int32, (cache.n_seq,), "pos_first_new", cache.device),
        _ptr(evicted_out, torch.int32, us, "evicted_out", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
    )
    _check(load_library().vd_append_evict_decode(cache.ref(), args[0], args[1], int(N), args[2],
                                                 int(variant), int(mu), args[3], args[4],
                                                 args[5], args[6], args[7], args[8],
                                                 _stream(stream)),
           "vd_append_evict_decode")


def vd_evict_decode(cache: Cache, N: int, N_dev=None, variant: int = VD_SCORE_L2,
                    mu: int = VD_MU_RECOMPUTE, running_sum=None, evicted_out=None,
                    kept_idx_out=None, scores_out=None, stream=None) -> None:
    torch = _torch()
    us = cache.unit_shape()
    args = (
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(evicted_out, torch.int32, us, "evicted_out", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
    )
    _check(load_library().vd_evict_decode(cache.ref(), int(N), args[0], int(variant), int(mu),
                                          args[1], args[2], args[3], args[4], _stream(stream)),
           "vd_evict_decode")


def vd_score_ex(cache: Cache, variant: int, score_keys: bool = False, scores_out=None,
                dispersion_out=None, stream=None, mu: int = VD_MU_RECOMPUTE,
                running_sum=None) -> None:
    """Scores of V (or K) rows and/or the per-unit dispersion sigma; with
    mu=VD_MU_RUNNING the mean is running_sum / len (fp64 [n_seq, n_layer,
    n_kv_head, head_dim], read only), so the rows are read once."""
    torch = _torch()
    us = cache.unit_shape()
    sc = _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device)
    dp = _ptr(dispersion_out, torch.float32, us, "dispersion_out", cache.device)
    rs = _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device)
    _check(load_library().vd_score_ex(cache.ref(), int(variant), int(mu), rs,
                                      int(bool(score_keys)), sc, dp, _stream(stream)),
           "vd_score_ex")


def vd_evict_block_ex(cache: Cache, N: int, N_dev=None, B: int = 0, variant: int = VD_SCORE_L2,
                      mu: int = VD_MU_RECOMPUTE, running_sum=None, score_keys: bool = False,
                      attn=None, kept_idx_out=None, scores_out=None, dispersion_out=None,
                      stream=None) -> None:
    """Block eviction on the K-side rule and/or with attention weights;
    dispersion_out: fp32 [n_seq, n_layer, n_kv_head], sigma of the
    pre-eviction rows from the same score pass (units that evicted)."""
    torch = _torch()
    us = cache.unit_shape()
    args = (
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(attn, torch.float32, us + (cache.capacity,), "attn", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
        _ptr(dispersion_out, torch.float32, us, "dispersion_out", cache.device),
    )
    _check(load_library().vd_evict_block_ex(cache.ref(), int(N), args[0], int(B), int(variant),
                                            int(mu), args[1], int(bool(score_keys)), args[2],
                                            args[3], args[4], args[5], _stream(stream)),
           "vd_evict_block_ex")


def vd_append_evict_block_ex(cache: Cache, k_new, v_new, B: int, N: int, N_dev=None,
                             variant: int = VD_SCORE_L2, mu: int = VD_MU_RECOMPUTE,
                             running_sum=None, score_keys: bool = False, attn=None,
                             kept_idx_out=None, scores_out=None, dispersion_out=None,
                             stream=None) -> None:
    """vd_append followed by vd_evict_block_ex in one launch; k_new, v_new:
    bf16 [n_seq, n_layer, n_kv_head, B, head_dim], read straight from the
    caller's buffers (attn covers the new rows at slots len .. len + B - 1)."""
    torch = _torch()
    us = cache.unit_shape()
    shape = us + (int(B), cache.head_dim)
    args = (
        _ptr(k_new, torch.bfloat16, shape, "k_new", cache.device),
        _ptr(v_new, torch.bfloat16, shape, "v_new", cache.device),
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(attn, torch.float32, us + (cache.capacity,), "attn", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
        _ptr(dispersion_out, torch.float32, us, "dispersion_out", cache.device),
    )
    _check(load_library().vd_append_evict_block_ex(
        cache.ref(), args[0], args[1], int(B), int(N), args[2], int(variant), int(mu), args[3],
        int(bool(score_keys)), args[4], args[5], args[6], args[7], _stream(stream)),
        "vd_append_evict_block_ex")


def vd_evict_block_holefill(cache: Cache, N: int, pos, pos_first_new, N_dev=None, B: int = 0,
                            variant: int = VD_SCORE_L2, mu: int = VD_MU_RECOMPUTE,
                            running_sum=None, kept_idx_out=None, scores_out=None,
                            stream=None) -> None:
    """Block eviction in the hole-fill layout (kept appended rows move into the
    evicted slots; ties by token position).  pos: int32 [.., capacity]
    positions of the cached rows; pos_first_new: int32 [n_seq]."""
    torch = _torch()
    us = cache.unit_shape()
    args = (
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(pos, torch.int32, us + (cache.capacity,), "pos", cache.device),
        _ptr(pos_first_new, torch.int32, (cache.n_seq,), "pos_first_new", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
    )
    _check(load_library().vd_evict_block_holefill(cache.ref(), int(N), args[0], int(B), int(variant),
                                                  int(mu), args[1], args[2], args[3], args[4],
                                                  args[5], _stream(stream)),
           "vd_evict_block_holefill")


def vd_evict_decode_holefill(cache: Cache, N: int, pos, pos_first_new, N_dev=None,
                             variant: int = VD_SCORE_L2, mu: int = VD_MU_RECOMPUTE,
                             running_sum=None, evicted_out=None, kept_idx_out=None,
                             scores_out=None, stream=None) -> None:
    """Decode eviction in the hole-fill layout: the appended token moves into
    the evicted slot (at most one row moves)."""
    torch = _torch()
    us = cache.unit_shape()
    args = (
        _ptr(N_dev, torch.int32, (cache.n_seq,), "N_dev", cache.device),
        _ptr(running_sum, torch.float64, us + (cache.head_dim,), "running_sum", cache.device),
        _ptr(pos, torch.int32, us + (cache.capacity,), "pos", cache.device),
        _ptr(pos_first_new, torch.int32, (cache.n_seq,), "pos_first_new", cache.device),
        _ptr(evicted_out, torch.int32, us, "evicted_out", cache.device),
        _ptr(kept_idx_out, torch.int32, us + (int(N),), "kept_idx_out", cache.device),
        _ptr(scores_out, torch.float32, us + (cache.capacity,), "scores_out", cache.device),
    )
    _check(load_library().vd_evict_decode_holefill(cache.ref(), int(N), args[0], int(variant),
                                                   int(mu), args[1], args[2], args[3], args[4],
                                                   args[5], args[6], _stream(stream)),
           "vd_evict_decode_holefill")


def vd_append(cache: Cache, k_new, v_new, B: int, stream=None) -> None:
    torch = _torch()
    shape = cache.unit_shape() + (int(B), cache.head_dim)
    kp = _ptr(k_new, torch.bfloat16, shape, "k_new", cache.device)
    vp = _ptr(v_new, torch.bfloat16, shape, "v_new", cache.device)
    _check(load_library().vd_append(cache.ref(), kp, vp, int(B), _stream(stream)), "vd_append")


def vd_running_sum_init_ex(cache: Cache, of_keys: bool, running_sum, stream=None) -> None:
    """fp64 column sums of the cached K rows (of_keys) or V rows, per unit."""
    torch = _torch()
    rp = _ptr(running_sum, torch.float64, cache.unit_shape() + (cache.head_dim,), "running_sum",
              cache.device)
    _check(load_library().vd_running_sum_init_ex(cache.ref(), int(bool(of_keys)), rp,
                                                 _stream(stream)), "vd_running_sum_init_ex")


def vd_running_sum_init(cache: Cache, running_sum, stream=None) -> None:
    torch = _torch()
    rp = _ptr(running_sum, torch.float64, cache.unit_shape() + (cache.head_dim,), "running_sum",
              cache.device)
    _check(load_library().vd_running_sum_init(cache.ref(), rp, _stream(stream)), "vd_running_sum_init")


def _launch_stream(device, stream):
    """The stream handle of a call.  Kernels launch on the current device: tensors of
    another one are refused."""
    torch = _torch()
    if device.type != "cuda" or not torch.cuda.is_initialized():
        return None  # CPU tensors: refused once the call's arguments are checked
    index = torch._C._cuda_getDevice()
    if device.index != index:
        raise ValueError(f"the tensors live on {device}, the current device is cuda:{index}")
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if stream is None and raw is not None else _stream(stream)


def vd_q4_append(cache: Q4Cache, k_new, v_new, B: int, stream=None) -> None:
    """vd_append into a 4-bit cache; k_new, v_new: bf16
    [n_seq, n_layer, n_kv_head, B, head_dim]."""
    torch = _torch()
    s = _launch_stream(cache.device, stream)
    shape = cache.unit_shape() + (int(B), cache.head_dim)
    kp = _ptr(k_new, torch.bfloat16, shape, "k_new", cache.device)
    vp = _ptr(v_new, torch.bfloat16, shape, "v_new", cache.device)
    _check(load_library().vd_q4_append(cache.ref(), kp, vp, int(B), s),
           "vd_q4_append")


def _same_device(stored, cache: Cache, stream):
    if stored.device != cache.device:
        raise ValueError(f"cache must live on {stored.device}, got {cache.device}")
    return _launch_stream(stored.device, stream)


def vd_q4_pack(dst: Q4Cache, src: Cache, layer0: int = 0, stream=None) -> None:
    """Rows [0, src.len) of a bf16 cache into layers [layer0, layer0 + src.n_layer)
    of a 4-bit one; the call that writes the last layer also sets dst.len."""
    s = _same_device(dst, src, stream)
    _check(load_library().vd_q4_pack(dst.ref(), int(layer0), src.ref(), s),
           "vd_q4_pack")


def vd_q4_unpack(src: Q4Cache, dst: Cache, layer0: int = 0, stream=None) -> None:
    """Rows [0, src.len) of layers [layer0, layer0 + dst.n_layer) of a 4-bit cache to
    bf16 (exact) in dst, and dst.len = src.len."""
    s = _same_device(src, dst, stream)
    _check(load_library().vd_q4_unpack(src.ref(), int(layer0), dst.ref(), s),
           "vd_q4_unpack")


def vd_q4_attend(cache: Q4Cache, q, out, k_new=None, v_new=None, layer: int = 0, scale=None,
                 lse_out=None, stream=None) -> None:
    """Attention of new tokens over one layer of a 4-bit cache and, causally, over their
    own rows.  q, out: bf16 [n_seq, B, n_q_head, head_dim]; k_new, v_new: bf16
    [n_seq, n_layer, n_kv_head, B, head_dim], the buffers of vd_q4_append, or both None
    (every token sees the cached rows alone); scale: 1 / sqrt(head_dim) unless given;
    lse_out: fp32 [n_seq, B, n_q_head]."""
    torch = _torch()
    s = _launch_stream(cache.device, stream)
    if q.dim() != 4:
        raise ValueError("q must be [n_seq, B, n_q_head, head_dim]")
    _, B, n_q, _ = q.shape
    shape = (cache.n_seq, B, n_q, cache.head_dim)
    new = cache.unit_shape() + (B, cache.head_dim)
    args = (
        _ptr(q, torch.bfloat16, shape, "q", cache.device),
        _ptr(k_new, torch.bfloat16, new, "k_new", cache.device),
        _ptr(v_new, torch.bfloat16, new, "v_new", cache.device),
        _ptr(out, torch.bfloat16, shape, "out", cache.device),
        _ptr(lse_out, torch.float32, shape[:3], "lse_out", cache.device),
    )
    scale = cache.head_dim ** -0.5 if scale is None else float(scale)
    _check(load_library().vd_q4_attend(cache.ref(), int(layer), args[0], n_q, args[1], args[2], B,
                                       scale, args[3], args[4], s),
           "vd_q4_attend")


def vd_qkv_norm_rope(qkv, q_out, k_new, v_new, layer: int = 0, q_weight=None, k_weight=None,
                     eps: float = 1e-6, inv_freq=None, pos_first_new=None,
                     interleaved: bool = False, stream=None) -> None:
    """Queries and one layer's new rows from projections, in one pass: per-head RMS norm
    of queries and keys (weights bf16 [head_dim], or None: no norm), rotation of their
    first 2 * len(inv_freq) values by position (inv_freq fp32, or None: no rotation;
    pos_first_new int32 [n_seq]), values copied.  qkv: bf16
    [n_seq, B, n_q_head + 2 * n_kv_head, head_dim]; q_out: bf16
    [n_seq, B, n_q_head, head_dim]; k_new, v_new: bf16
    [n_seq, n_layer, n_kv_head, B, head_dim], of which `layer` is written."""
    torch = _torch()
    if qkv.dim() != 4 or q_out.dim() != 4 or k_new.dim() != 5:
        raise ValueError("qkv and q_out must have 4 dimensions, k_new 5")
    dev = qkv.device
    s = _launch_stream(dev, stream)
    n_seq, B, heads, d = qkv.shape
    n_q, n_layer = q_out.shape[2], k_new.shape[1]
    n_kv = (heads - n_q) // 2
    new = (n_seq, n_layer, n_kv, B, d)
    pairs = 0 if inv_freq is None else inv_freq.numel()
    if heads != n_q + 2 * n_kv:
        raise ValueError(f"qkv has {heads} heads, which are not {n_q} query heads and as many "
                         "key as value heads")
    args = (
        _ptr(qkv, torch.bfloat16, (n_seq, B, heads, d), "qkv", dev),
        _ptr(q_weight, torch.bfloat16, (d,), "q_weight", dev),
        _ptr(k_weight, torch.bfloat16, (d,), "k_weight", dev),
        _ptr(inv_freq, torch.float32, (pairs,), "inv_freq", dev),
        _ptr(pos_first_new, torch.int32, (n_seq,), "pos_first_new", dev),
        _ptr(q_out, torch.bfloat16, (n_seq, B, n_q, d), "q_out", dev),
        _ptr(k_new, torch.bfloat16, new, "k_new", dev),
        _ptr(v_new, torch.bfloat16, new, "v_new", dev),
    )
    _on_gpu(dev)
    _check(load_library().vd_qkv_norm_rope(args[0], n_seq, B, n_q, n_kv, d, args[1], args[2],
                                           float(eps), args[3], 2 * pairs, int(bool(interleaved)),
                                           args[4], args[5], args[6], args[7], int(layer), n_layer, s),
           "vd_qkv_norm_rope")


def _paged_stream(cache: PagedCache, stream):
    """_launch_stream for a cache that is on a GPU, where CUDA is up."""
    if not cache._gpu:
        return None
    C = _torch()._C
    index = C._cuda_getDevice()
    if cache.device.index != index:
        raise ValueError(f"the tensors live on {cache.device}, the current device is cuda:{index}")
    raw = getattr(C, "_cuda_getCurrentRawStream", None)
    return raw(index) if stream is None and raw is not None else _stream(stream)


def vd_paged_append(cache: PagedCache, qkv, q_out, layer: int = 0, q_weight=None, k_weight=None,
                    eps: float = 1e-6, inv_freq=None, pos_first_new=None,
                    interleaved: bool = False, n_new=None, stream=None) -> None:
    """vd_qkv_norm_rope whose keys and values go to slots [len, len + n_new) of one layer of a
    paged cache (n_new int32 [n_seq], or None: all B); without pos_first_new a token's
    position is its slot.  len stays until vd_paged_advance."""
    torch = _torch()
    shape = qkv.shape
    if len(shape) != 4 or q_out.dim() != 4:
        raise ValueError("qkv and q_out must have 4 dimensions")
    dev, n_seq, d, bf16 = cache.device, cache.n_seq, cache.head_dim, torch.bfloat16
    s = _paged_stream(cache, stream)
    B, heads = shape[1], shape[2]
    n_q = heads - 2 * cache.n_kv_head
    pairs = 0 if inv_freq is None else inv_freq.numel()
    args = (
        _ptr(qkv, bf16, (n_seq, B, heads, d), "qkv", dev),
        None if n_new is None else _ptr(n_new, torch.int32, cache._vector, "n_new", dev),
        None if q_weight is None else _ptr(q_weight, bf16, (d,), "q_weight", dev),
        None if k_weight is None else _ptr(k_weight, bf16, (d,), "k_weight", dev),
        None if inv_freq is None else _ptr(inv_freq, torch.float32, (pairs,), "inv_freq", dev),
        None if pos_first_new is None else _ptr(pos_first_new, torch.int32, cache._vector,
                                                "pos_first_new", dev),
        _ptr(q_out, bf16, (n_seq, B, n_q, d), "q_out", dev),
    )
    code = load_library().vd_paged_append(cache.ref(), int(layer), args[0], B, n_q, args[1], args[2],
                                          args[3], float(eps), args[4], 2 * pairs, bool(interleaved),
                                          args[5], args[6], s)
    if code:
        raise VdError(code, "vd_paged_append")


def vd_paged_attend_workspace(cache: PagedCache, n_q_head: int, B: int) -> int:
    """Bytes of workspace that vd_paged_attend takes on the current device: one size for all calls
    over caches of this type and head_dim, whatever their sequences, tokens, heads and lengths."""
    return int(load_library().vd_paged_attend_workspace(cache._ref, int(n_q_head), int(B)))


def vd_paged_attend(cache: PagedCache, q, out, workspace, layer: int = 0, causal: bool = True,
                    scale=None, n_new=None, lse_out=None, stream=None) -> None:
    """Attention of new tokens over one layer of a paged cache: token i over slots
    [0, len + i + 1) (causal: its own row is in the pages, vd_paged_append) or over
    [0, len).  q, out: bf16 [n_seq, B, n_q_head, head_dim]; workspace: uint8, at least
    vd_paged_attend_workspace bytes, one for each stream and graph that may run at the same
    time; n_new int32 [n_seq], or None: all B; scale: 1 / sqrt(head_dim) unless given; lse_out:
    fp32 [n_seq, B, n_q_head]."""
    torch = _torch()
    dev = cache.device
    s = _paged_stream(cache, stream)
    if q.dim() != 4:
        raise ValueError("q must be [n_seq, B, n_q_head, head_dim]")
    _, B, n_q, _ = q.shape
    shape, size = (cache.n_seq, B, n_q, cache.head_dim), workspace.numel()
    args = (
        _ptr(q, torch.bfloat16, shape, "q", dev),
        None if n_new is None else _ptr(n_new, torch.int32, cache._vector, "n_new", dev),
        _ptr(out, torch.bfloat16, shape, "out", dev),
        None if lse_out is None else _ptr(lse_out, torch.float32, shape[:3], "lse_out", dev),
        _ptr(workspace, torch.uint8, (size,), "workspace", dev),
    )
    scale = cache.head_dim ** -0.5 if scale is None else float(scale)
    code = load_library().vd_paged_attend(cache.ref(), int(layer), args[0], B, n_q, args[1],
                                          bool(causal), scale, args[2], args[3], args[4], size, s)
    if code:
        raise VdError(code, "vd_paged_attend")


def vd_paged_advance(cache: PagedCache, B: int = 1, n_new=None, stream=None) -> None:
    """len += n_new (int32 [n_seq], at most B each; None: B), at the end of a step."""
    torch = _torch()
    s = _launch_stream(cache.device, stream)
    n = _ptr(n_new, torch.int32, (cache.n_seq,), "n_new", cache.device)
    _check(load_library().vd_paged_advance(cache.ref(), n, int(B), s), "vd_paged_advance")


def vd_paged_pack(dst: PagedCache, src: Cache, layer0: int = 0, stream=None) -> None:
    """Rows [0, src.len) of a bf16 cache into layers [layer0, layer0 + src.n_layer) of a
    paged one; the call that writes the last layer also sets dst.len."""
    s = _same_device(dst, src, stream)
    _check(load_library().vd_paged_pack(dst.ref(), int(layer0), src.ref(), s), "vd_paged_pack")


def vd_paged_unpack(src: PagedCache, dst: Cache, layer0: int = 0, stream=None) -> None:
    """Rows [0, src.len) of layers [layer0, layer0 + dst.n_layer) of a paged cache to bf16
    in dst, and dst.len = src.len."""
    s = _same_device(src, dst, stream)
    _check(load_library().vd_paged_unpack(src.ref(), int(layer0), dst.ref(), s), "vd_paged_unpack")


def vd_workspace_size(cache: Cache) -> int:
    return int(load_library().vd_workspace_size(cache._ref))  # no launch: any device


def vd_status_string(code: int) -> str:
    return load_library().vd_status_string(int(code)).decode()


def vd_get_device_status(stream=None) -> int:
    """Synchronises the stream and returns (and clears) the device status."""
    return int(load_library().vd_get_device_status(_stream(stream)))
