"""ctypes binding of libworldkv.so: the same calls as include/wk.h, argument marshalling only (that of the token-level cache's
calls, which a program makes for every token, is compiled: csrc/pages_binding.cc).

PyTorch supplies device memory and streams; every step of the path runs in the library's kernels.
There is no fallback: if the shared library is missing or no sm_100 device is present, loading or
``wk_create`` fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libworldkv.so")

WK_OK = 0
WK_ERR_ARG, WK_ERR_SHAPE, WK_ERR_POOL_FULL, WK_ERR_BAD_SLOT = -1, -2, -3, -4
WK_ERR_CUDA, WK_ERR_TIMEOUT, WK_ERR_NONFINITE, WK_ERR_UNBOUND, WK_ERR_NO_DEVICE = -5, -6, -7, -8, -9
WK_DEV_BAD_SLOT, WK_DEV_TIMEOUT, WK_DEV_NONFINITE, WK_DEV_POOL_FULL = 1, 2, 4, 8


class wk_config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("tokens_per_frame", C.c_int32), ("frames_per_chunk", C.c_int32), ("n_keep", C.c_int32),
                ("pool_slots", C.c_int32), ("max_k", C.c_int32), ("max_dense_segments", C.c_int32),
                ("device", C.c_int32), ("softmax_scale", C.c_float), ("score_mode", C.c_int32)]


class wk_dense_seg(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("n_tokens", C.c_int32), ("reserved", C.c_int32)]


class wk_paged_kv(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("K_exp", C.c_void_p), ("V_exp", C.c_void_p),
                ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_pages", C.c_int32), ("page_tokens", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("type", C.c_int32), ("reserved", C.c_int32)]


SCORE_WHOLE_KEY, SCORE_PER_HEAD = 0, 2     # wk_config.score_mode
WK_BF16, WK_F16, WK_E4M3 = 0, 1, 2         # wk_paged_kv.type
_TYPES = {torch.bfloat16: WK_BF16, torch.float16: WK_F16, torch.float8_e4m3fn: WK_E4M3}


class WkError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)} ({status})")
        self.status = status


_lib = None


def load_library() -> C.CDLL:
    """Loads libworldkv.so (built in-tree by paper_2605_22718_b200.build) and declares its symbols."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2605_22718_b200.build` (needs nvcc); "
                           "there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    cfgp = C.POINTER(wk_config)
    sigs = {
        "wk_create": (i32, [cfgp, C.POINTER(vp)]),
        "wk_destroy": (None, [vp]),
        "wk_pool_bytes": (sz, [cfgp]),
        "wk_scratch_bytes": (sz, [cfgp, i32, i32, i32]),
        "wk_bind": (i32, [vp, vp, sz, vp, sz, i32, i32, i32]),
        "wk_compress_chunk": (i32, [vp, vp, i64, i32, vp, vp, vp]),
        "wk_pool_append": (i32, [vp, i32, i32, vp, vp, i64, vp, C.POINTER(C.c_float), i64, C.POINTER(i32), vp]),
        "wk_pool_compress_append": (i32, [vp, i32, i32, vp, vp, i64, vp, C.POINTER(C.c_float), i64, i32, C.POINTER(i32),
                                          C.POINTER(i32), vp]),
        "wk_pool_evict": (i32, [vp, i32, vp]),
        "wk_pool_oldest": (i32, [vp]),
        "wk_pool_count": (i32, [vp]),
        "wk_pool_tag": (i64, [vp, i32]),
        "wk_retrieve": (i32, [vp, C.POINTER(C.c_float), i32, vp, vp, C.POINTER(i32), vp]),
        "wk_retrieve_query": (i32, [vp, i32, vp, i32, i32, vp, vp, C.POINTER(i32), vp]),
        "wk_host_chunk_bytes": (C.c_size_t, [vp]),
        "wk_pool_store_host": (i32, [vp, i32, vp, vp]),
        "wk_pool_load_host": (i32, [vp, i32, i32, vp, C.POINTER(C.c_float), C.c_int64, C.POINTER(i32), vp]),
        "wk_retrieve_scan_scratch_bytes": (C.c_size_t, []),
        "wk_retrieve_scan": (i32, [vp, vp, vp, C.c_int64, C.POINTER(C.c_float), i32, vp, vp, i32, vp, C.c_size_t, vp]),
        "wk_retrieve_noalloc": (i32, [vp, vp, i32, C.POINTER(C.c_float), i32, i32, vp, vp, vp]),
        "wk_memory_attention": (i32, [vp, i32, vp, i32, C.POINTER(wk_dense_seg), i32, vp, i32, vp, vp, i32, vp]),
        "wk_page_plan": (i32, [vp, i32, i32, i32, vp, vp, vp, vp, i32, i64, vp, vp, vp, i32, vp, vp, vp]),
        "wk_page_store": (i32, [vp, vp, vp, vp, i32, i32, i64, vp, vp]),
        "wk_paged_scratch_bytes": (sz, [vp]),
        "wk_paged_attention": (i32, [vp, vp, vp, i32, i64, i32, i32, vp, i32, i64, vp, i32, i32, C.c_float, vp, vp, vp, sz,
                                     vp]),
        "wk_poll_status": (i32, [vp, C.POINTER(C.c_uint32), vp]),
        "wk_status_string": (C.c_char_p, [i32]),
        "wk_last_cuda_error": (i32, [vp]),
        "wk_launch_count": (i64, [vp]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


EXPORTED_SYMBOLS = ("wk_create", "wk_destroy", "wk_pool_bytes", "wk_scratch_bytes", "wk_bind", "wk_compress_chunk",
                    "wk_pool_append", "wk_pool_compress_append", "wk_pool_evict", "wk_pool_oldest", "wk_pool_count", "wk_pool_tag", "wk_retrieve",
                    "wk_retrieve_noalloc", "wk_retrieve_query", "wk_retrieve_scan", "wk_retrieve_scan_scratch_bytes",
                    "wk_host_chunk_bytes", "wk_pool_store_host", "wk_pool_load_host",
                    "wk_memory_attention", "wk_page_plan", "wk_page_store", "wk_paged_scratch_bytes", "wk_paged_attention",
                    "wk_poll_status", "wk_status_string", "wk_last_cuda_error",
                    "wk_launch_count")


def status_string(status: int) -> str:
    return load_library().wk_status_string(status).decode()


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    # torch's own raw getters: building a Stream object for the current stream takes 3.2 us of a 10 us call, this 0.2
    if not stream:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _made(stream: Optional[torch.cuda.Stream], make, *args, **kw) -> torch.Tensor:
    """What a call allocates.  It belongs to the stream that the call runs on: a block of another stream's could be given to work
    (or come from work) that does not wait for the call."""
    if not stream:
        return make(*args, **kw)
    if not isinstance(stream, torch.cuda.Stream):     # any object that has a cuda_stream
        stream = torch.cuda.ExternalStream(stream.cuda_stream)
    with torch.cuda.stream(stream):
        return make(*args, **kw)


_Pose = C.c_float * 8


def _pose_arg(pose):
    """The eight numbers of a pose as a C array (arrays and tensors hand over all of them in one call)."""
    if hasattr(pose, "tolist"):
        try:
            return _Pose(*pose.tolist())
        except TypeError:    # not plain numbers: elements that only float() converts
            pass
    return _Pose(*[float(x) for x in pose])


def retrieve_noalloc(poses: torch.Tensor, valid: torch.Tensor, cur_pose: Sequence[float], k: int, max_k: int,
                     slots_out: torch.Tensor, dist_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """wk_retrieve_noalloc: pose retrieval for callers that may not allocate device memory (no context, scratch built
    into the library).  poses [n_slots, 8] fp32, valid [n_slots] int32, slots_out [max_k] int32, dist_out [max_k] fp64 -- all
    preallocated by the caller; this wrapper allocates nothing either."""
    pose_arr = _pose_arg(cur_pose)
    st = load_library().wk_retrieve_noalloc(poses.data_ptr(), valid.data_ptr(), poses.shape[0], pose_arr, k, max_k,
                                            slots_out.data_ptr(), _ptr(dist_out), _stream(stream))
    if st != WK_OK:
        raise WkError(st, "wk_retrieve_noalloc")


class WorldKV:
    """One library context plus the two device buffers it needs (allocated through torch).

    Method names and arguments mirror include/wk.h.  Tensors are CUDA tensors: bf16 [tokens, H, 128]
    (or [tokens, D]) contiguous; index tensors int32.  A call runs on ``stream``, or on the current one; what it
    allocates belongs to that stream, as with ``torch.cuda.stream``.
    """

    def __init__(self, n_layers: int, n_heads: int, tokens_per_frame: int, n_keep: int, pool_slots: int, max_k: int,
                 frames_per_chunk: int = 3, max_dense_segments: int = 4, device: int = 0, softmax_scale: float = 0.0,
                 max_batch: int = 1, max_lq: int = 0, max_splits: int = 1, score_mode: int = 0):
        self.lib = load_library()
        self.cfg = wk_config(n_layers, n_heads, 128, tokens_per_frame, frames_per_chunk, n_keep, pool_slots, max_k,
                             max_dense_segments, device, softmax_scale, score_mode)
        self.score_mode, self.n_heads = score_mode, n_heads
        self.T, self.F, self.H, self.D = tokens_per_frame, frames_per_chunk, n_heads, n_heads * 128
        self.C = tokens_per_frame + n_keep
        self.NA = (frames_per_chunk - 1) * tokens_per_frame
        self.n_layers, self.pool_slots, self.max_k = n_layers, pool_slots, max_k
        self.max_lq = max_lq if max_lq > 0 else frames_per_chunk * tokens_per_frame
        handle = C.c_void_p()
        st = self.lib.wk_create(C.byref(self.cfg), C.byref(handle))
        if st != WK_OK:
            raise WkError(st, "wk_create")
        self.ctx = handle
        self.device = torch.device("cuda", device)
        pool_bytes = self.lib.wk_pool_bytes(C.byref(self.cfg))
        scratch_bytes = self.lib.wk_scratch_bytes(C.byref(self.cfg), max_batch, self.max_lq, max_splits)
        self.pool = torch.zeros(pool_bytes, dtype=torch.uint8, device=self.device)
        self.scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=self.device)
        torch.cuda.synchronize(self.device)
        st = self.lib.wk_bind(self.ctx, self.pool.data_ptr(), pool_bytes, self.scratch.data_ptr(), scratch_bytes,
                              max_batch, self.max_lq, max_splits)
        if st != WK_OK:
            raise WkError(st, "wk_bind")

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.lib.wk_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        self.close()

    # ---- World Compression --------------------------------------------------------------------
    def compress_chunk(self, K_chunks: torch.Tensor, keep_idx_out: Optional[torch.Tensor] = None,
                       scores_out: Optional[torch.Tensor] = None, batch: Optional[int] = None,
                       batch_stride_elems: Optional[int] = None, stream=None) -> torch.Tensor:
        """K_chunks: [batch, F*T, D] bf16.  Returns keep_idx [batch, T + n_keep] int32 ([batch, H, T + n_keep] with
        per-head keep-sets)."""
        if batch is None:
            batch = K_chunks.shape[0] if K_chunks.dim() == 3 else 1
        if batch_stride_elems is None:
            batch_stride_elems = K_chunks.stride(0) if K_chunks.dim() == 3 else self.F * self.T * self.D
        if keep_idx_out is None:
            shape = (batch, self.n_heads, self.C) if self.score_mode == SCORE_PER_HEAD else (batch, self.C)
            keep_idx_out = _made(stream, torch.empty, shape, dtype=torch.int32, device=self.device)
        st = self.lib.wk_compress_chunk(self.ctx, K_chunks.data_ptr(), batch_stride_elems, batch,
                                        keep_idx_out.data_ptr(), _ptr(scores_out), _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_compress_chunk")
        return keep_idx_out

    # ---- chunk pool ---------------------------------------------------------------------------
    def pool_append(self, layer0: int, n: int, K_chunks: torch.Tensor, V_chunks: torch.Tensor, keep_idx: torch.Tensor,
                    pose: Sequence[float], chunk_tag: int = 0, slot: int = -1,
                    batch_stride_elems: Optional[int] = None, stream=None) -> int:
        if batch_stride_elems is None:
            batch_stride_elems = K_chunks.stride(0) if K_chunks.dim() == 3 else self.F * self.T * self.D
        pose_arr = _pose_arg(pose)
        slot_io = C.c_int32(slot)
        st = self.lib.wk_pool_append(self.ctx, layer0, n, K_chunks.data_ptr(), V_chunks.data_ptr(), batch_stride_elems,
                                     keep_idx.data_ptr(), pose_arr, chunk_tag, C.byref(slot_io), _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_pool_append")
        return slot_io.value

    def pool_compress_append(self, layer0: int, n: int, K_chunks: torch.Tensor, V_chunks: torch.Tensor,
                             pose: Sequence[float], chunk_tag: int = 0, slot: int = -1, evict_oldest_if_full: bool = False,
                             keep_idx: Optional[torch.Tensor] = None, batch_stride_elems: Optional[int] = None,
                             stream=None) -> Tuple[int, int, torch.Tensor]:
        """wk_pool_compress_append: returns (slot, evicted slot or -1, keep_idx)."""
        if batch_stride_elems is None:
            batch_stride_elems = K_chunks.stride(0) if K_chunks.dim() == 3 else self.F * self.T * self.D
        if keep_idx is None:
            shape = (n, self.n_heads, self.C) if self.score_mode == SCORE_PER_HEAD else (n, self.C)
            keep_idx = _made(stream, torch.empty, shape, dtype=torch.int32, device=self.device)
        pose_arr = _pose_arg(pose)
        slot_io, evicted = C.c_int32(slot), C.c_int32(-1)
        st = self.lib.wk_pool_compress_append(self.ctx, layer0, n, K_chunks.data_ptr(), V_chunks.data_ptr(),
                                              batch_stride_elems, keep_idx.data_ptr(), pose_arr, chunk_tag,
                                              1 if evict_oldest_if_full else 0, C.byref(slot_io), C.byref(evicted),
                                              _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_pool_compress_append")
        return slot_io.value, evicted.value, keep_idx

    def pool_evict(self, slot: int, stream=None) -> None:
        st = self.lib.wk_pool_evict(self.ctx, slot, _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_pool_evict")

    def pool_oldest(self) -> int:
        return self.lib.wk_pool_oldest(self.ctx)

    def pool_count(self) -> int:
        return self.lib.wk_pool_count(self.ctx)

    def pool_tag(self, slot: int) -> int:
        return self.lib.wk_pool_tag(self.ctx, slot)

    # ---- World Retrieval ----------------------------------------------------------------------
    def retrieve(self, cur_pose: Sequence[float], k: int, slots_out: Optional[torch.Tensor] = None,
                 dist_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, int]:
        """Returns (slots_out int32[max_k] on the device, count = min(k, M))."""
        if slots_out is None:
            slots_out = _made(stream, torch.empty, max(1, self.max_k), dtype=torch.int32, device=self.device)
        pose_arr, n_out = _pose_arg(cur_pose), C.c_int32(0)
        st = self.lib.wk_retrieve(self.ctx, pose_arr, k, slots_out.data_ptr(), _ptr(dist_out), C.byref(n_out),
                                  _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_retrieve")
        return slots_out, n_out.value

    # ---- host-memory tier ----------------------------------------------------------------------
    def host_chunk_bytes(self) -> int:
        return self.lib.wk_host_chunk_bytes(self.ctx)

    def pool_store_host(self, slot: int, host_dst: torch.Tensor, stream=None) -> None:
        """Copies the chunk in `slot` into a (page-locked) host tensor of host_chunk_bytes() bytes."""
        assert not host_dst.is_cuda and host_dst.numel() * host_dst.element_size() >= self.host_chunk_bytes()
        st = self.lib.wk_pool_store_host(self.ctx, slot, host_dst.data_ptr(), _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_pool_store_host")

    def pool_load_host(self, layer0: int, n: int, host_src: torch.Tensor, pose: Sequence[float], chunk_tag: int = -1,
                       slot: int = -1, stream=None) -> int:
        """Loads layers [layer0, layer0 + n) of a host chunk image into the pool; returns the slot."""
        assert not host_src.is_cuda and host_src.numel() * host_src.element_size() >= self.host_chunk_bytes()
        pose_arr = _pose_arg(pose)
        slot_io = C.c_int32(slot)
        st = self.lib.wk_pool_load_host(self.ctx, layer0, n, host_src.data_ptr(), pose_arr, chunk_tag, C.byref(slot_io),
                                        _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_pool_load_host")
        return slot_io.value

    def retrieve_scan(self, poses: torch.Tensor, cur_pose: Sequence[float], k: int, valid: Optional[torch.Tensor] = None,
                      ids_out: Optional[torch.Tensor] = None, dist_out: Optional[torch.Tensor] = None,
                      scratch: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Retrieval over a plain pose array [n, 8] fp32 of any length; returns ids_out int32 (-1 past the count)."""
        if ids_out is None:
            ids_out = _made(stream, torch.empty, max(1, k), dtype=torch.int32, device=self.device)
        if scratch is None:
            scratch = _made(stream, torch.empty, self.lib.wk_retrieve_scan_scratch_bytes(), dtype=torch.uint8, device=self.device)
        pose_arr = _pose_arg(cur_pose)
        st = self.lib.wk_retrieve_scan(self.ctx, poses.data_ptr(), _ptr(valid), poses.shape[0], pose_arr, k,
                                       ids_out.data_ptr(), _ptr(dist_out), ids_out.numel(), scratch.data_ptr(),
                                       scratch.numel(), _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_retrieve_scan")
        return ids_out

    def retrieve_query(self, layer: int, Q: torch.Tensor, k: int, slots_out: Optional[torch.Tensor] = None,
                       score_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, int]:
        """Query-based retrieval: returns (slots_out int32[max_k] on the device, count = min(k, M))."""
        if slots_out is None:
            slots_out = _made(stream, torch.empty, max(1, self.max_k), dtype=torch.int32, device=self.device)
        n_out = C.c_int32(0)
        st = self.lib.wk_retrieve_query(self.ctx, layer, Q.data_ptr(), Q.shape[0], k, slots_out.data_ptr(), _ptr(score_out),
                                        C.byref(n_out), _stream(stream))
        if st != WK_OK:
            raise WkError(st, "wk_retrieve_query")
        return slots_out, n_out.value

    # ---- memory attention ---------------------------------------------------------------------
    def memory_attention(self, layer: int, Q: torch.Tensor, segs: Sequence[Tuple[torch.Tensor, torch.Tensor]],
                         slots: Optional[torch.Tensor], n_slots: int, O: Optional[torch.Tensor] = None,
                         lse_out: Optional[torch.Tensor] = None, kv_splits: int = 0, stream=None) -> torch.Tensor:
        lq = Q.size(0)
        if O is None:
            O = _made(stream, torch.empty_like, Q)
        n_segs = len(segs)
        arr = (wk_dense_seg * max(1, n_segs))()
        for i, (k, v) in enumerate(segs):
            seg = arr[i]
            seg.K, seg.V, seg.n_tokens = k.data_ptr(), v.data_ptr(), k.size(0)
        st = self.lib.wk_memory_attention(self.ctx, layer, Q.data_ptr(), lq, arr, n_segs, _ptr(slots), n_slots,
                                          O.data_ptr(), _ptr(lse_out), kv_splits, _stream(stream))
        if st != WK_OK:
            raise WkError(st, f"wk_memory_attention (last CUDA error {self.last_cuda_error()})")
        return O

    # ---- status -------------------------------------------------------------------------------
    def poll_status(self, stream=None) -> Tuple[int, int]:
        flags = C.c_uint32(0)
        st = self.lib.wk_poll_status(self.ctx, C.byref(flags), _stream(stream))
        return st, flags.value

    def launch_count(self) -> int:
        return self.lib.wk_launch_count(self.ctx)

    def last_cuda_error(self) -> int:
        return self.lib.wk_last_cuda_error(self.ctx)


class PagedKV:
    """One layer's token-level cache in pages, on the device of a WorldKV context.

    K, V: [n_pages, page_tokens, n_kv_heads, head_dim] CUDA tensors of bf16, fp16 or float8_e4m3fn, head_dim 64 or 128, any
    strides that are multiples of 16 bytes (last axis contiguous; K and V alike).  In 8 bits K_exp and V_exp are uint8
    [n_pages, n_kv_heads, page_tokens], contiguous.  ``PagedKV.empty`` allocates them.  A cache made from n_pages and
    page_tokens alone only plans.  Method names and arguments mirror include/wk.h.

    A call runs on ``stream``, or on the current one.  What it allocates (slots, starts, O) belongs to that stream, as with
    ``torch.cuda.stream``: to use it on another stream, let that wait, and ``record_stream`` it there.
    """

    def __init__(self, kv: WorldKV, K: Optional[torch.Tensor] = None, V: Optional[torch.Tensor] = None,
                 K_exp: Optional[torch.Tensor] = None, V_exp: Optional[torch.Tensor] = None,
                 n_pages: Optional[int] = None, page_tokens: Optional[int] = None):
        self.kv, self.lib, self.device = kv, kv.lib, kv.device
        self._index, self._native = kv.device.index, _pages()
        self.K, self.V, self.K_exp, self.V_exp = K, V, K_exp, V_exp
        self._desc, self._desc_at = None, 0
        if K is None:
            _need(n_pages is not None and page_tokens is not None, "PagedKV: K and V, or n_pages and page_tokens")
            self.n_pages, self.page_tokens = n_pages, page_tokens
            return
        _need(V is not None and K.dim() == 4 and K.shape == V.shape and K.stride() == V.stride() and K.dtype == V.dtype
              and K.dtype in _TYPES and K.stride(3) == 1, "PagedKV: K and V of one shape, type and layout")
        self.n_pages, self.page_tokens, self.n_kv_heads, self.head_dim = K.shape
        self.type = _TYPES[K.dtype]
        self._on_device("PagedKV", K, V, K_exp, V_exp)
        if self.type == WK_E4M3:
            for e in (K_exp, V_exp):
                _need(e is not None and e.dtype == torch.uint8 and e.is_contiguous()
                      and e.shape == (self.n_pages, self.n_kv_heads, self.page_tokens), "PagedKV: K_exp and V_exp")
        else:
            _need(K_exp is None and V_exp is None, "PagedKV: exponents belong to a cache in 8 bits")
        self._desc = wk_paged_kv(K.data_ptr(), V.data_ptr(), _ptr(K_exp), _ptr(V_exp), K.stride(0), K.stride(1), K.stride(2),
                                 self.n_pages, self.page_tokens, self.n_kv_heads, self.head_dim, self.type, 0)
        self._desc_at = C.addressof(self._desc)
        if getattr(kv, "paged_scratch", None) is None:     # shared by the caches of a context, like its other scratch
            kv.paged_scratch = torch.zeros(self.lib.wk_paged_scratch_bytes(kv.ctx), dtype=torch.uint8, device=self.device)
            torch.cuda.synchronize(self.device)

    @classmethod
    def empty(cls, kv: WorldKV, n_pages: int, page_tokens: int, n_kv_heads: int, head_dim: int = 128,
              dtype: torch.dtype = torch.bfloat16) -> "PagedKV":
        shape = (n_pages, page_tokens, n_kv_heads, head_dim)
        pages = [torch.empty(shape, dtype=dtype, device=kv.device) for _ in range(2)]
        exps = [torch.full((n_pages, n_kv_heads, page_tokens), 127, dtype=torch.uint8, device=kv.device)
                if dtype == torch.float8_e4m3fn else None for _ in range(2)]
        return cls(kv, *pages, *exps)

    def _on_device(self, what: str, *tensors) -> None:
        for x in tensors:
            _need(x is None or (x.is_cuda and x.get_device() == self._index), what + ": tensors on the context's device")

    def free_pages(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(ring, state) for page_plan with every page free."""
        ring = torch.arange(self.n_pages, dtype=torch.int32, device=self.device)
        return ring, torch.tensor([0, self.n_pages, 0, 0], dtype=torch.int32, device=self.device)

    def page_plan(self, lens: torch.Tensor, new_tokens: torch.Tensor, tables: torch.Tensor, ring: torch.Tensor,
                  state: torch.Tensor, max_tokens: int, lens_out: Optional[torch.Tensor] = None,
                  state_out: Optional[torch.Tensor] = None, slots_out: Optional[torch.Tensor] = None,
                  starts_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Pages and slots for the next step's tokens; lens and state are advanced in place unless lens_out, state_out are
        given.  Returns (slots [max_tokens], starts [n_req + 1]) int32, on the device."""
        kv = self.kv
        r = self._native.page_plan(kv.ctx.value if kv.ctx else 0, self._index, self.n_pages, self.page_tokens, lens, new_tokens,
                                   lens_out, tables, ring, state, state_out, max_tokens, slots_out, starts_out,
                                   stream.cuda_stream if stream else None)
        return r if r.__class__ is tuple else _failed(r, "wk_page_plan", kv)

    def page_store(self, K_new: torch.Tensor, V_new: torch.Tensor, slots: torch.Tensor, stream=None) -> None:
        """Rows K_new, V_new [n, n_kv_heads, head_dim] (heads contiguous, any row stride, both alike) into slots [>= n]."""
        kv = self.kv
        if self._desc is None:
            raise WkError(WK_ERR_ARG, "page_store: a cache that only plans (made without K and V)")
        r = self._native.page_store(kv.ctx.value if kv.ctx else 0, self._index, self._desc_at, K_new, V_new, slots,
                                    stream.cuda_stream if stream else None)
        if r is not None:
            _failed(r, "wk_page_store", kv)

    def paged_attention(self, Q: torch.Tensor, tables: torch.Tensor, lens: torch.Tensor, window: int = 0, sink: int = 0,
                        softmax_scale: float = 0.0, O: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                        scratch: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """O [n_req, n_heads, head_dim] of one new token per request: Q [n_req, n_heads, head_dim] (heads contiguous, any
        row stride) over the tokens that tables and lens name.  scratch: as WorldKV's, shared by the calls of a context unless
        given.  Calls that may overlap on the GPU (on several streams, or replayed from several graphs) need one each, zero-filled once:
        where two have overlapped on one, all later results on it are undefined until it is zero-filled again
        (``kv.paged_scratch.zero_()``)."""
        kv = self.kv
        if self._desc is None:
            raise WkError(WK_ERR_ARG, "paged_attention: a cache that only plans (made without K and V)")
        r = self._native.paged_attention(kv.ctx.value if kv.ctx else 0, self._index, self._desc_at, Q, tables, lens, window, sink,
                                         softmax_scale, O, lse_out, scratch if scratch is not None else kv.paged_scratch,
                                         stream.cuda_stream if stream else None)
        return r if r.__class__ is not int and r.__class__ is not str else _failed(r, "wk_paged_attention", kv)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise WkError(WK_ERR_ARG, what)


def _failed(r, what: str, kv: WorldKV):
    """Raises for what the marshalling returned in place of tensors: what is wrong with an argument, or a call's status."""
    if isinstance(r, str):
        raise WkError(WK_ERR_ARG, r)
    raise WkError(r, f"{what} (last CUDA error {kv.last_cuda_error() if kv.ctx else 0})")


_marshalling = None


def _pages():
    """The compiled marshalling of the three calls (csrc/pages_binding.cc), told where the library has them."""
    global _marshalling
    if _marshalling is None:
        lib = load_library()
        try:
            from . import _pages as native
        except ImportError as e:
            raise RuntimeError("_pages.so is missing or does not fit this PyTorch: run `python -m paper_2605_22718_b200.build`; "
                               "there is no fallback path") from e
        native.use(*[C.cast(f, C.c_void_p).value for f in (lib.wk_page_plan, lib.wk_page_store, lib.wk_paged_attention)])
        _marshalling = native
    return _marshalling
