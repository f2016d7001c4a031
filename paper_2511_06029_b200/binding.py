"""Thin ctypes binding of liblethe.so: same names as the C ABI (include/lethe.h), argument marshalling only.

Every step of the path runs in the CUDA library; nothing here computes.  torch supplies device memory and
streams.  If the library has not been built (``python -m paper_2511_06029_b200.build``) loading fails loudly —
there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("LETHE_LIB", os.path.join(_HERE, "liblethe.so"))   # LETHE_LIB: an alternative build

OK, ERR_INVALID_ARG, ERR_CAPACITY, ERR_BUDGET, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED, ERR_PAGE, ERR_TOO_LARGE = range(9)
STATIC_PRUNE_MAX_ENTRIES = 4 * 1024 * 1024
F32, BF16, FP8_E4M3, FP8_E5M2 = 0, 1, 2, 3
CONTIG, PAGED = 0, 1
VARIANT_AUTO, VARIANT_SIMT, VARIANT_MMA4, VARIANT_MMA8 = 0, 1, 2, 3

EXPORTS = ["lethe_create", "lethe_destroy", "lethe_last_error", "lethe_poll_status", "lethe_set_tuning", "lethe_set_wait_limit",
           "lethe_decode_attend", "lethe_decode_attend_host", "lethe_estimate_sparsity", "lethe_alloc_budgets",
           "lethe_rasr_prune", "lethe_rasr_prune_static", "lethe_segment_prune", "lethe_prefill_seed",
           "lethe_collapsed_prune", "lethe_chunk_attend", "lethe_rotate", "lethe_append", "lethe_block_append", "lethe_block_read",
           "lethe_block_select", "lethe_block_attend"]


class LetheError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"lethe status {status}: {msg}")
        self.status = status


class lethe_cache(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("layout", ctypes.c_int32), ("capacity", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("rel", ctypes.c_void_p), ("pos", ctypes.c_void_p),
        ("len", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
        ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
    ]


class lethe_score_mod(ctypes.Structure):
    _fields_ = [("softcap", ctypes.c_float), ("window", ctypes.c_int32), ("slopes", ctypes.c_void_p),
                ("doc_start", ctypes.c_void_p), ("prefix_len", ctypes.c_void_p)]


class lethe_rotary(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("style", ctypes.c_int32), ("n_axes", ctypes.c_int32),
                ("pair_axis", ctypes.POINTER(ctypes.c_int32)), ("pair_freq", ctypes.POINTER(ctypes.c_double)),
                ("axis_pos", ctypes.c_void_p)]


class lethe_block_cache(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
        ("capacity", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("k_range", ctypes.c_void_p), ("k_open", ctypes.c_void_p), ("v_open", ctypes.c_void_p), ("len", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
    ]


_lib = None


def load() -> ctypes.CDLL:
    """Load liblethe.so and declare the prototypes of include/lethe.h."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_06029_b200.build` "
                           "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, cp = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(lethe_cache)
    lib.lethe_create.restype = ctypes.c_int
    lib.lethe_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int, ctypes.c_size_t]
    lib.lethe_destroy.restype = None
    lib.lethe_destroy.argtypes = [vp]
    lib.lethe_last_error.restype = ctypes.c_char_p
    lib.lethe_last_error.argtypes = [vp]
    lib.lethe_poll_status.restype = ctypes.c_int
    lib.lethe_poll_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
    lib.lethe_set_tuning.restype = ctypes.c_int
    lib.lethe_set_tuning.argtypes = [vp, ctypes.c_int, ctypes.c_int]
    lib.lethe_set_wait_limit.restype = ctypes.c_int
    lib.lethe_set_wait_limit.argtypes = [vp, i32]
    attend_args = [vp, cp, ctypes.c_int, ctypes.c_int, vp, vp, vp, vp, ctypes.POINTER(ctypes.c_float),
                   ctypes.c_float, vp, vp, vp]
    lib.lethe_decode_attend.restype = ctypes.c_int
    lib.lethe_decode_attend.argtypes = attend_args
    lib.lethe_decode_attend_host.restype = ctypes.c_int
    lib.lethe_decode_attend_host.argtypes = attend_args
    lib.lethe_estimate_sparsity.restype = ctypes.c_int
    lib.lethe_estimate_sparsity.argtypes = [vp, cp, vp, vp]
    lib.lethe_alloc_budgets.restype = ctypes.c_int
    lib.lethe_alloc_budgets.argtypes = [vp, ctypes.c_int, ctypes.c_int, vp, vp, i32, vp, vp]
    lib.lethe_rasr_prune.restype = ctypes.c_int
    lib.lethe_rasr_prune.argtypes = [vp, cp, vp, i32, i32, vp, i32, vp]
    lib.lethe_collapsed_prune.restype = ctypes.c_int
    lib.lethe_collapsed_prune.argtypes = [vp, cp, vp, i32, i32, i32, vp, i32, vp]
    lib.lethe_segment_prune.restype = ctypes.c_int
    lib.lethe_segment_prune.argtypes = [vp, cp, i32, ctypes.c_float, i32, i32, vp, vp, i32, vp]
    lib.lethe_prefill_seed.restype = ctypes.c_int
    lib.lethe_prefill_seed.argtypes = [vp, cp, vp, i32, ctypes.POINTER(ctypes.c_float), ctypes.c_float, vp]
    lib.lethe_chunk_attend.restype = ctypes.c_int
    lib.lethe_chunk_attend.argtypes = [vp, cp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, ctypes.c_int, vp, vp, vp, vp,
                                       ctypes.POINTER(ctypes.c_float), ctypes.c_double, ctypes.POINTER(lethe_score_mod),
                                       ctypes.POINTER(lethe_rotary), vp, vp, vp]
    lib.lethe_rotate.restype = ctypes.c_int
    lib.lethe_rotate.argtypes = [vp, ctypes.POINTER(lethe_rotary), i32, i32, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                 ctypes.c_int, vp, vp, i32, vp, vp, vp]
    bp, rp, fp = ctypes.POINTER(lethe_block_cache), ctypes.POINTER(lethe_rotary), ctypes.POINTER(ctypes.c_float)
    lib.lethe_append.restype = ctypes.c_int
    lib.lethe_append.argtypes = [vp, cp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, ctypes.c_int, vp, vp, vp, vp, rp, vp, vp]
    lib.lethe_block_append.restype = ctypes.c_int
    lib.lethe_block_append.argtypes = [vp, bp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, ctypes.c_int, vp, vp, vp, rp, vp, vp]
    lib.lethe_block_read.restype = ctypes.c_int
    lib.lethe_block_read.argtypes = [vp, bp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, vp, vp, vp]
    lib.lethe_block_select.restype = ctypes.c_int
    lib.lethe_block_select.argtypes = [vp, bp, ctypes.c_int, ctypes.c_int, vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp]
    lib.lethe_block_attend.restype = ctypes.c_int
    lib.lethe_block_attend.argtypes = [vp, bp, ctypes.c_int, ctypes.c_int, vp, fp, vp, ctypes.c_int, vp, vp, vp]
    lib.lethe_rasr_prune_static.restype = ctypes.c_int
    lib.lethe_rasr_prune_static.argtypes = [cp, vp, i32, i32, vp, i32, vp, vp]
    _lib = lib
    return lib


def _dp(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _raw_stream(device: int) -> int:
    """The current stream's handle (without the Stream object around it, which takes longer to make than a small call)."""
    return torch._C._cuda_getCurrentRawStream(device)


class Cache:
    """Device tensors of the cache plus the C descriptor that points at them (the tensors stay owned here)."""

    def __init__(self, n_q_heads: int, k: torch.Tensor, v: torch.Tensor, rel: torch.Tensor, pos: torch.Tensor,
                 len_: torch.Tensor, page_table: Optional[torch.Tensor] = None, k_scale=None, v_scale=None):
        """k_scale, v_scale: per-layer scales of a float8_e4m3fn / float8_e5m2 cache (sequences of L floats; None = 1)."""
        self.k, self.v, self.rel, self.pos, self.len, self.page_table = k, v, rel, pos, len_, page_table
        for t in (k, v, rel, pos, len_) + ((page_table,) if page_table is not None else ()):
            assert t.is_cuda and t.is_contiguous()
        assert rel.dtype == torch.float32 and pos.dtype == torch.int32 and len_.dtype == torch.int32
        L, B, Hkv = len_.shape
        dt = {torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: FP8_E4M3, torch.float8_e5m2: FP8_E5M2}[k.dtype]
        if page_table is None:
            assert k.dim() == 5 and tuple(k.shape[:3]) == (L, B, Hkv)
            cap, D, layout, pt, npages = k.shape[3], k.shape[4], CONTIG, 0, 0
            assert tuple(rel.shape) == (L, B, Hkv, cap)
        else:
            assert k.dim() == 3 and page_table.dtype == torch.int32
            npages, pt, D = k.shape
            cap, layout = page_table.shape[3], PAGED
            assert tuple(rel.shape) == (L, B, Hkv, cap * pt)
        self.n_layers, self.batch, self.n_kv_heads, self.n_q_heads, self.head_dim = L, B, Hkv, n_q_heads, D
        self.capacity, self.page_tokens = cap, pt
        self.c = lethe_cache(L, B, n_q_heads, Hkv, D, dt, layout, cap, pt, k.data_ptr(), v.data_ptr(),
                             rel.data_ptr(), pos.data_ptr(), len_.data_ptr(),
                             page_table.data_ptr() if page_table is not None else None, npages, None, None)
        # host arrays of the per-layer scales, kept alive here
        self._k_scale = self._v_scale = None
        if dt in (FP8_E4M3, FP8_E5M2):
            for name, sc in (("k_scale", k_scale), ("v_scale", v_scale)):
                if sc is None:
                    continue
                vals = [float(x) for x in (sc.tolist() if isinstance(sc, torch.Tensor) else sc)]
                assert len(vals) == L
                arr = (ctypes.c_float * L)(*vals)
                setattr(self, "_" + name, arr)
                setattr(self.c, name, ctypes.cast(arr, ctypes.c_void_p))
        else:
            assert k_scale is None and v_scale is None, "scales belong to quantised caches"

    @property
    def act_dtype(self) -> torch.dtype:
        """Type of q, k_new, v_new and out."""
        return torch.bfloat16 if self.k.dtype in (torch.float8_e4m3fn, torch.float8_e5m2) else self.k.dtype

    @property
    def device(self):
        return self.k.device

    @property
    def cap_tokens(self) -> int:
        return self.capacity * self.page_tokens if self.page_table is not None else self.capacity


class BlockCache:
    """Device tensors of a cache in 8 bits with a scale for each block of tokens, plus the C descriptor that points at them (the
    tensors stay owned here)."""

    def __init__(self, n_q_heads: int, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                 k_range: Optional[torch.Tensor], k_open: torch.Tensor, v_open: torch.Tensor, len_: torch.Tensor,
                 page_table: Optional[torch.Tensor] = None):
        """k, v int8 [L][B][Hkv][capacity][block_tokens][D], or pools [pages][block_tokens][D] with page_table [L][B][Hkv][capacity]
        int32; k_scale, v_scale float32 and k_range int8 [..][2][D] (or None) by block likewise; k_open, v_open bfloat16
        [L][B][Hkv][block_tokens][D]; len_ int32 [L][B][Hkv]."""
        self.k, self.v, self.k_scale, self.v_scale, self.k_range = k, v, k_scale, v_scale, k_range
        self.k_open, self.v_open, self.len, self.page_table = k_open, v_open, len_, page_table
        for t in (k, v, k_scale, v_scale, k_range, k_open, v_open, len_, page_table):
            assert t is None or (t.is_cuda and t.is_contiguous() and t.device == k.device)
        assert k.dtype == v.dtype == torch.int8 and k.shape == v.shape and (k_range is None or k_range.dtype == torch.int8)
        assert k_scale.dtype == v_scale.dtype == torch.float32 and k_open.dtype == v_open.dtype == torch.bfloat16
        assert len_.dtype == torch.int32 and len_.dim() == 3
        L, B, Hkv = len_.shape
        lead, (T, D) = tuple(k.shape[:-2]), k.shape[-2:]
        if page_table is None:
            assert len(lead) == 4 and lead[:3] == (L, B, Hkv)
            cap, layout, n_pages = lead[3], CONTIG, 0
        else:
            assert len(lead) == 1 and page_table.dtype == torch.int32 and page_table.dim() == 4 and tuple(page_table.shape[:3]) == (L, B, Hkv)
            cap, layout, n_pages = page_table.shape[3], PAGED, lead[0]
        assert tuple(k_scale.shape) == tuple(v_scale.shape) == lead and (k_range is None or tuple(k_range.shape) == lead + (2, D))
        assert tuple(k_open.shape) == tuple(v_open.shape) == (L, B, Hkv, T, D)
        self.n_layers, self.batch, self.n_kv_heads, self.n_q_heads, self.head_dim = L, B, Hkv, n_q_heads, D
        self.capacity, self.block_tokens = cap, T
        ptr = [None if t is None else t.data_ptr() for t in (k, v, k_scale, v_scale, k_range, k_open, v_open, len_, page_table)]
        self.c = lethe_block_cache(L, B, n_q_heads, Hkv, D, layout, cap, T, *ptr, n_pages)
        self.ref = ctypes.byref(self.c)

    @property
    def device(self):
        return self.k.device

    @property
    def cap_tokens(self) -> int:
        return self.capacity * self.block_tokens


class ScoreMod:
    """lethe_score_mod: softcap, window, and device tensors slopes [Hq] fp32, doc_start [n_tokens] int32, prefix_len [B] int32
    (each may be None).  The tensors stay owned here."""

    def __init__(self, softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
                 doc_start: Optional[torch.Tensor] = None, prefix_len: Optional[torch.Tensor] = None):
        self.slopes, self.doc_start, self.prefix_len = slopes, doc_start, prefix_len
        for t, dt in ((slopes, torch.float32), (doc_start, torch.int32), (prefix_len, torch.int32)):
            assert t is None or (t.is_cuda and t.is_contiguous() and t.dim() == 1 and t.dtype == dt)
        ptr = [None if t is None else t.data_ptr() for t in (slopes, doc_start, prefix_len)]
        self.c = lethe_score_mod(float(softcap), int(window), *ptr)


ROT_HALVES, ROT_PAIRS = 0, 1


class Rotary:
    """lethe_rotary: pair_axis and pair_freq (one entry per pair; host sequences) and axis_pos, a device int32 tensor
    [n_axes][n_tokens].  The rotated part of a row is twice as long as pair_axis."""

    def __init__(self, pair_axis: Sequence[int], pair_freq: Sequence[float], axis_pos: torch.Tensor, style: int = ROT_HALVES):
        assert len(pair_axis) == len(pair_freq)
        assert axis_pos.is_cuda and axis_pos.is_contiguous() and axis_pos.dim() == 2 and axis_pos.dtype == torch.int32
        n = len(pair_axis)
        self.axis_pos = axis_pos
        self.pair_axis = (ctypes.c_int32 * n)(*[int(x) for x in pair_axis])
        self.pair_freq = (ctypes.c_double * n)(*[float(x) for x in pair_freq])
        self.c = lethe_rotary(2 * n, int(style), axis_pos.shape[0], ctypes.cast(self.pair_axis, ctypes.POINTER(ctypes.c_int32)),
                              ctypes.cast(self.pair_freq, ctypes.POINTER(ctypes.c_double)), axis_pos.data_ptr())
        self.ref = ctypes.byref(self.c)
        self.n_tokens = axis_pos.shape[1]


def rasr_prune_static(cache: "Cache", budgets: torch.Tensor, recent: int, sink: int,
                      keep_idx: Optional[torch.Tensor] = None, status_out: Optional[torch.Tensor] = None) -> int:
    """lethe_rasr_prune_static: the prune step for callers that may not allocate device memory (no context, fixed
    in-library scratch).  Runs on the current device and the current torch stream; returns the host-side status
    (OK, or ERR_TOO_LARGE / ERR_INVALID_ARG / ... when nothing was enqueued).  status_out: device int32[2]."""
    assert budgets.dtype == torch.int32 and budgets.is_cuda
    max_k = 0
    if keep_idx is not None:
        assert keep_idx.dtype == torch.int32 and keep_idx.is_cuda
        max_k = keep_idx.shape[-1]
    if status_out is not None:
        assert status_out.dtype == torch.int32 and status_out.is_cuda and status_out.numel() >= 2
    return int(load().lethe_rasr_prune_static(ctypes.byref(cache.c), _dp(budgets), recent, sink, _dp(keep_idx), max_k,
                                              _dp(status_out), _stream(cache.device)))


COLLAPSE_HEADS, COLLAPSE_HEADS_BATCH = 0, 1


class Context:
    """Owns one lethe_ctx.  Methods carry the C names without the prefix and raise LetheError on failure."""

    def __init__(self, device: int = 0, scratch_bytes_hint: int = 0):
        self.lib = load()
        self.device = device
        h = ctypes.c_void_p()
        st = self.lib.lethe_create(ctypes.byref(h), device, scratch_bytes_hint)
        if st != OK:
            raise LetheError(st, "lethe_create failed (needs an sm_100 GPU)")
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.lethe_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def last_error(self) -> str:
        return self.lib.lethe_last_error(self.h).decode()

    def _check(self, st: int):
        if st != OK:
            raise LetheError(st, self.last_error())

    def set_tuning(self, variant: int = 0, splits: int = 0):
        self._check(self.lib.lethe_set_tuning(self.h, variant, splits))

    def set_wait_limit(self, polls: int = 0):
        self._check(self.lib.lethe_set_wait_limit(self.h, polls))

    def poll_status(self):
        """Synchronise the current stream and return (status, item) of the first device-side error since last poll."""
        info = (ctypes.c_int32 * 2)()
        st = self.lib.lethe_poll_status(self.h, _stream(self.device), info)
        return st, int(info[1])

    @staticmethod
    def _scale(scale: Sequence[float]):
        arr = (ctypes.c_float * len(scale))(*[float(x) for x in scale])
        return arr

    def decode_attend(self, cache: Cache, layer_begin: int, layer_end: int, q, k_new, v_new, token_pos, scale, gamma,
                      out, lse=None, scale_c=None):
        sc = scale_c if scale_c is not None else self._scale(scale)
        self._check(self.lib.lethe_decode_attend(self.h, ctypes.byref(cache.c), layer_begin, layer_end, _dp(q),
                                                 _dp(k_new), _dp(v_new), _dp(token_pos), sc, gamma, _dp(out), _dp(lse),
                                                 _stream(self.device)))

    def decode_attend_host(self, cache: Cache, layer_begin: int, layer_end: int, q, k_new, v_new, token_pos, scale,
                           gamma, out, lse=None, scale_c=None):
        """q, k_new, v_new, token_pos, out, lse are HOST tensors (pinned for asynchronous copies)."""
        for t in (q, k_new, v_new, token_pos, out, lse):
            assert t is None or (not t.is_cuda and t.is_contiguous())
        sc = scale_c if scale_c is not None else self._scale(scale)
        self._check(self.lib.lethe_decode_attend_host(self.h, ctypes.byref(cache.c), layer_begin, layer_end, _dp(q),
                                                      _dp(k_new), _dp(v_new), _dp(token_pos), sc, gamma, _dp(out),
                                                      _dp(lse), _stream(self.device)))

    def estimate_sparsity(self, cache: Cache, sparsity: torch.Tensor):
        assert sparsity.is_cuda and sparsity.dtype == torch.float32
        self._check(self.lib.lethe_estimate_sparsity(self.h, ctypes.byref(cache.c), _dp(sparsity),
                                                     _stream(self.device)))

    def alloc_budgets(self, sparsity: torch.Tensor, total_budget: torch.Tensor, k_min: int, budgets: torch.Tensor):
        assert sparsity.dtype == torch.float32 and total_budget.dtype == torch.int64 and budgets.dtype == torch.int32
        L, B = sparsity.shape
        self._check(self.lib.lethe_alloc_budgets(self.h, L, B, _dp(sparsity), _dp(total_budget), k_min, _dp(budgets),
                                                 _stream(self.device)))

    def rasr_prune(self, cache: Cache, budgets: torch.Tensor, recent: int, sink: int,
                   keep_idx: Optional[torch.Tensor] = None):
        assert budgets.dtype == torch.int32 and budgets.is_cuda
        max_k = 0
        if keep_idx is not None:
            assert keep_idx.dtype == torch.int32 and keep_idx.is_cuda
            max_k = keep_idx.shape[-1]
        self._check(self.lib.lethe_rasr_prune(self.h, ctypes.byref(cache.c), _dp(budgets), recent, sink,
                                              _dp(keep_idx), max_k, _stream(self.device)))

    def segment_prune(self, cache: Cache, n_segments: int, tau: float, recent: int, sink: int, l_evict: torch.Tensor,
                      keep_idx: Optional[torch.Tensor] = None):
        assert l_evict.dtype == torch.int32 and l_evict.is_cuda and l_evict.is_contiguous()
        max_k = 0
        if keep_idx is not None:
            assert keep_idx.dtype == torch.int32 and keep_idx.is_cuda
            max_k = keep_idx.shape[-1]
        self._check(self.lib.lethe_segment_prune(self.h, ctypes.byref(cache.c), n_segments, tau, recent, sink,
                                                 _dp(l_evict), _dp(keep_idx), max_k, _stream(self.device)))

    def collapsed_prune(self, cache: Cache, budgets: torch.Tensor, recent: int, sink: int, scope: int,
                        keep_idx: Optional[torch.Tensor] = None):
        """scope COLLAPSE_HEADS: budgets [L][B]; COLLAPSE_HEADS_BATCH: budgets [L]; keep_idx [groups][max_k]."""
        assert budgets.dtype == torch.int32 and budgets.is_cuda and budgets.is_contiguous()
        max_k = 0
        if keep_idx is not None:
            assert keep_idx.dtype == torch.int32 and keep_idx.is_cuda
            max_k = keep_idx.shape[-1]
        self._check(self.lib.lethe_collapsed_prune(self.h, ctypes.byref(cache.c), _dp(budgets), recent, sink, scope,
                                                   _dp(keep_idx), max_k, _stream(self.device)))

    def prefill_seed(self, cache: Cache, q_prompt: torch.Tensor, scale, gamma: float):
        """q_prompt [L][B][P][Hq][D] on the device, cache dtype; overwrites rel[0..P) of every item."""
        assert q_prompt.is_cuda and q_prompt.is_contiguous() and q_prompt.dim() == 5
        self._check(self.lib.lethe_prefill_seed(self.h, ctypes.byref(cache.c), _dp(q_prompt), q_prompt.shape[2],
                                                self._scale(scale), gamma, _stream(self.device)))

    def rotate(self, rotary: Rotary, q: torch.Tensor, k: Optional[torch.Tensor], q_out: torch.Tensor,
               k_out: Optional[torch.Tensor], inverse: bool = False):
        """q [nl][n_tokens][Hq][D] and k [nl][n_tokens][Hkv][D] (or None), float32 or bfloat16, into q_out, k_out (which may be
        q, k themselves)."""
        shape, dt = q.shape, q.dtype
        assert q.is_cuda and q_out.is_cuda and q.is_contiguous() and q_out.is_contiguous() and q_out.shape == shape and q_out.dtype == dt
        nl, n, hq, d = shape
        assert rotary.n_tokens == n and (k is None) == (k_out is None)
        hkv, kp, ko = 0, None, None
        if k is not None:
            ks = k.shape
            assert k.is_cuda and k_out.is_cuda and k.is_contiguous() and k_out.is_contiguous() and k_out.shape == ks and k.dtype == k_out.dtype == dt
            assert ks[0] == nl and ks[1] == n and ks[3] == d
            hkv, kp, ko = ks[2], k.data_ptr(), k_out.data_ptr()
        code = F32 if dt == torch.float32 else BF16 if dt == torch.bfloat16 else -1
        self._check(self.lib.lethe_rotate(self.h, rotary.ref, code, d, nl, n, hq, hkv, q.data_ptr(), kp, 1 if inverse else 0, q_out.data_ptr(), ko,
                                          torch.cuda.current_stream(self.device).cuda_stream))

    def chunk_attend(self, cache: Cache, layer_begin: int, layer_end: int, chunk_start: torch.Tensor, max_chunk: int, q, k_new,
                     v_new, token_pos, scale, gamma, out, lse=None, mod: Optional[ScoreMod] = None,
                     rotary: Optional[Rotary] = None, scale_c=None):
        """q, out [nl][n_tokens][Hq][D]; k_new, v_new [nl][n_tokens][Hkv][D] or None; chunk_start [B + 1] int32 and token_pos
        [n_tokens] int32 on the device; lse [nl][n_tokens][Hq] float32 or None.  All contiguous."""
        nl, n_tokens = layer_end - layer_begin, q.shape[1]
        act, head = cache.act_dtype, (cache.n_q_heads, cache.head_dim)
        assert chunk_start.is_cuda and chunk_start.is_contiguous() and chunk_start.dtype == torch.int32 and chunk_start.numel() == cache.batch + 1
        for t in (q, out):
            assert t.is_cuda and t.is_contiguous() and t.dtype == act and tuple(t.shape) == (nl, n_tokens) + head
        for t in (k_new, v_new):
            assert t is None or (t.is_cuda and t.is_contiguous() and t.dtype == act and tuple(t.shape) == (nl, n_tokens, cache.n_kv_heads, cache.head_dim))
        assert token_pos is None or (token_pos.is_cuda and token_pos.is_contiguous() and token_pos.dtype == torch.int32 and token_pos.numel() == n_tokens)
        assert lse is None or (lse.is_cuda and lse.is_contiguous() and lse.dtype == torch.float32 and tuple(lse.shape) == (nl, n_tokens, cache.n_q_heads))
        if mod is not None:
            assert mod.slopes is None or mod.slopes.numel() == cache.n_q_heads
            assert mod.doc_start is None or mod.doc_start.numel() == n_tokens
            assert mod.prefix_len is None or mod.prefix_len.numel() == cache.batch
        assert rotary is None or rotary.n_tokens == n_tokens
        sc = scale_c if scale_c is not None else self._scale(scale)
        self._check(self.lib.lethe_chunk_attend(self.h, ctypes.byref(cache.c), layer_begin, layer_end, _dp(chunk_start), n_tokens,
                                                max_chunk, _dp(q), _dp(k_new), _dp(v_new), _dp(token_pos), sc, gamma,
                                                None if mod is None else ctypes.byref(mod.c),
                                                None if rotary is None else ctypes.byref(rotary.c), _dp(out), _dp(lse),
                                                _stream(self.device)))

    # get_device() is -1 for a host tensor: one comparison says that a tensor is where the context's kernels run.
    def _append_args(self, cache, nl, chunk_start, act, k_new, v_new, rotary, q, q_out):
        """Checks what append and block_append have in common; the number of tokens."""
        n, dev = k_new.shape[1], self.device
        assert cache.len.get_device() == dev and chunk_start.get_device() == dev and chunk_start.is_contiguous() and chunk_start.dtype == torch.int32 and chunk_start.numel() == cache.batch + 1
        want = (nl, n, cache.n_kv_heads, cache.head_dim)
        for t in (k_new, v_new):
            assert t.get_device() == dev and t.dtype == act and t.shape == want and t.is_contiguous()
        assert (q is None) == (q_out is None) and (rotary is None or (rotary.n_tokens == n and rotary.axis_pos.get_device() == dev))
        if q is not None:
            want = (nl, n, cache.n_q_heads, cache.head_dim)
            assert q.get_device() == dev and q.dtype == act and q.shape == want and q.is_contiguous()
            assert q_out is q or (q_out.get_device() == dev and q_out.dtype == act and q_out.shape == want and q_out.is_contiguous())
        return n

    def append(self, cache: Cache, layer_begin: int, layer_end: int, chunk_start: torch.Tensor, max_chunk: int, k_new, v_new, token_pos,
               rotary: Optional[Rotary] = None, q=None, q_out=None):
        """k_new, v_new [nl][n_tokens][Hkv][D]; chunk_start [B + 1] and token_pos [n_tokens] int32; q, q_out [nl][n_tokens][Hq][D] (with
        rotary) or None.  All contiguous device tensors."""
        n = self._append_args(cache, layer_end - layer_begin, chunk_start, cache.act_dtype, k_new, v_new, rotary, q, q_out)
        assert token_pos.get_device() == self.device and token_pos.is_contiguous() and token_pos.dtype == torch.int32 and token_pos.numel() == n
        self._check(self.lib.lethe_append(self.h, ctypes.byref(cache.c), layer_begin, layer_end, chunk_start.data_ptr(), n, max_chunk,
                                          None if q is None else q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), token_pos.data_ptr(),
                                          None if rotary is None else rotary.ref, None if q is None else q_out.data_ptr(),
                                          _raw_stream(self.device)))

    def block_append(self, cache: BlockCache, layer_begin: int, layer_end: int, chunk_start: torch.Tensor, max_chunk: int, k_new, v_new,
                     rotary: Optional[Rotary] = None, q=None, q_out=None):
        """As append, all bfloat16."""
        n = self._append_args(cache, layer_end - layer_begin, chunk_start, torch.bfloat16, k_new, v_new, rotary, q, q_out)
        self._check(self.lib.lethe_block_append(self.h, cache.ref, layer_begin, layer_end, chunk_start.data_ptr(), n, max_chunk,
                                                None if q is None else q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(),
                                                None if rotary is None else rotary.ref, None if q is None else q_out.data_ptr(),
                                                _raw_stream(self.device)))

    def block_read(self, cache: BlockCache, layer_begin: int, layer_end: int, slot_begin: Optional[torch.Tensor], k_out, v_out):
        """k_out, v_out bfloat16 [nl][B][Hkv][n_slots][D]; slot_begin [B] int32 on the device, or None for slot 0."""
        lead = (layer_end - layer_begin, cache.batch, cache.n_kv_heads, k_out.shape[3], cache.head_dim)
        assert cache.len.get_device() == self.device
        for t in (k_out, v_out):
            assert t.get_device() == self.device and t.dtype == torch.bfloat16 and t.shape == lead and t.is_contiguous()
        assert slot_begin is None or (slot_begin.get_device() == self.device and slot_begin.is_contiguous() and slot_begin.dtype == torch.int32 and slot_begin.numel() == cache.batch)
        self._check(self.lib.lethe_block_read(self.h, cache.ref, layer_begin, layer_end, None if slot_begin is None else slot_begin.data_ptr(),
                                              k_out.shape[3], k_out.data_ptr(), v_out.data_ptr(), _raw_stream(self.device)))

    def _block_query(self, cache, layer_begin, layer_end, selected, *tensors):
        want = (layer_end - layer_begin, cache.batch, cache.n_q_heads, cache.head_dim)
        assert cache.len.get_device() == self.device
        for t in tensors:
            assert t.get_device() == self.device and t.dtype == torch.bfloat16 and t.shape == want and t.is_contiguous()
        if selected is not None:
            assert selected.get_device() == self.device and selected.dtype == torch.int32 and selected.is_contiguous() and selected.dim() == 4
            assert selected.shape[:3] == (want[0], cache.batch, cache.n_kv_heads) and selected.shape[3] > 0

    def block_select(self, cache: BlockCache, layer_begin: int, layer_end: int, q, sink: int, recent: int, selected: torch.Tensor):
        """selected [nl][B][Hkv][n_select] int32 is written: the chosen blocks in ascending order, then -1."""
        self._block_query(cache, layer_begin, layer_end, selected, q)
        self._check(self.lib.lethe_block_select(self.h, cache.ref, layer_begin, layer_end, q.data_ptr(), selected.shape[3], sink, recent,
                                                selected.data_ptr(), _raw_stream(self.device)))

    def block_attend(self, cache: BlockCache, layer_begin: int, layer_end: int, q, scale, out, lse=None, selected: Optional[torch.Tensor] = None,
                     scale_c=None):
        """q, out [nl][B][Hq][D] bfloat16; scale one float per layer of the cache; lse [nl][B][Hq] float32 or None; selected as
        block_select leaves it, or None for all blocks."""
        self._block_query(cache, layer_begin, layer_end, selected, q, out)
        assert lse is None or (lse.get_device() == self.device and lse.dtype == torch.float32 and lse.shape == q.shape[:3] and lse.is_contiguous())
        sc = scale_c if scale_c is not None else self._scale(scale)
        self._check(self.lib.lethe_block_attend(self.h, cache.ref, layer_begin, layer_end, q.data_ptr(), sc,
                                                None if selected is None else selected.data_ptr(), 0 if selected is None else selected.shape[3],
                                                out.data_ptr(), None if lse is None else lse.data_ptr(),
                                                _raw_stream(self.device)))
