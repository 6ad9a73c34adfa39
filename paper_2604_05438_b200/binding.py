"""Binding of libtkphi.so: same names as the C entry points, marshalling only (ctypes; the paged calls, whose GPU time can
be a few microseconds, through a CPython module)."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtkphi.so")
_lib = None

WS_BUILD, WS_TOPK_DECODE, WS_DECODE_STEP, WS_MLP_KEY_FEATURES = 0, 1, 2, 3
WS_PAGED_ATTENTION, WS_PAGED_BLOCK_ATTENTION = 4, 5
FLAG_NONE, FLAG_NOSUB, FLAG_FULL_CONTEXT = 0, 1, 2

EXPORTED_SYMBOLS = (
    "tkphi_workspace_bytes", "tkphi_build_summaries", "tkphi_topk_decode", "tkphi_decode_step",
    "tkphi_device_status", "tkphi_last_error", "tkphi_version",
    "tkphi_kernel_timing_enable", "tkphi_kernel_timing_read",
    "tkphi_build_summaries_static", "tkphi_static_last_error", "tkphi_static_device_status",
    "tkphi_selftest_timeout",
    "tkphi_mlp_key_features", "tkphi_build_summaries_cached", "tkphi_decode_step_mlp",
    "tkphi_paged_workspace_bytes", "tkphi_paged_append", "tkphi_paged_attention", "tkphi_paged_block_attention",
    "tkphi_paged_append_norm", "tkphi_coded_append", "tkphi_coded_read", "tkphi_coded_workspace_bytes",
    "tkphi_coded_attention", "tkphi_coded_block_attention",
)
STATIC_SCRATCH_BYTES = 8 << 20
KERNEL_KINDS = ("score", "select", "exact_residual", "build", "memset", "cached_z", "mlp", "paged_append", "paged_select",
                "paged_rows", "paged_tiles", "paged_read")
ERR_TIMEOUT = -5


class TkphiError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"tkphi status {status}: {message}")
        self.status = status


class _KvDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("n_feat", C.c_int32), ("n_sink", C.c_int32),
                ("n_tail", C.c_int32), ("cu_seqlens_host", C.c_void_p), ("cu_seqlens_dev", C.c_void_p),
                ("k", C.c_void_p), ("v", C.c_void_p), ("kv_stride_head", C.c_int64),
                ("kv_stride_token", C.c_int64), ("n_tail_seq_host", C.c_void_p), ("n_tail_seq_dev", C.c_void_p)]


class _PhiDesc(C.Structure):
    _fields_ = [("w_q", C.c_void_p), ("b_q", C.c_void_p), ("w_k", C.c_void_p), ("b_k", C.c_void_p),
                ("gamma_q", C.c_float), ("gamma_k", C.c_float), ("phi_k_cache", C.c_void_p)]


class _MlpDesc(C.Structure):
    _fields_ = [("d_emb", C.c_int32), ("n_heads", C.c_int32), ("w_s", C.c_void_p), ("b_s", C.c_void_p),
                ("w_1", C.c_void_p), ("b_1", C.c_void_p), ("w_2", C.c_void_p), ("b_2", C.c_void_p),
                ("alpha", C.c_void_p), ("w_o", C.c_void_p), ("b_o", C.c_void_p)]


class _PagedDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("stride_page", C.c_int64), ("stride_head", C.c_int64),
                ("stride_token", C.c_int64), ("page_table", C.c_void_p), ("kv_lens_host", C.c_void_p),
                ("kv_lens_dev", C.c_void_p), ("cu_q_host", C.c_void_p), ("cu_q_dev", C.c_void_p),
                ("key_bounds", C.c_void_p), ("status", C.c_void_p)]


class _CodedDesc(C.Structure):
    _fields_ = [("step", _PagedDesc), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p)]


class _NormDesc(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("q_stride_head", C.c_int64), ("k_weight", C.c_void_p), ("k_stride_head", C.c_int64),
                ("eps", C.c_float)]


class _ReadDesc(C.Structure):
    _fields_ = [("cu_rows_host", C.c_void_p), ("cu_rows_dev", C.c_void_p), ("first_host", C.c_void_p), ("first_dev", C.c_void_p),
                ("k_out", C.c_void_p), ("k_stride_row", C.c_int64), ("k_stride_head", C.c_int64),
                ("v_out", C.c_void_p), ("v_stride_row", C.c_int64), ("v_stride_head", C.c_int64)]


class _AppendDesc(C.Structure):
    _fields_ = [("k_new", C.c_void_p), ("k_stride_token", C.c_int64), ("k_stride_head", C.c_int64),
                ("v_new", C.c_void_p), ("v_stride_token", C.c_int64), ("v_stride_head", C.c_int64),
                ("q", C.c_void_p), ("q_stride_token", C.c_int64), ("q_stride_head", C.c_int64),
                ("q_out", C.c_void_p), ("o_stride_token", C.c_int64), ("o_stride_head", C.c_int64),
                ("inv_freq", C.c_void_p), ("rot_dim", C.c_int32), ("pairs", C.c_int32), ("positions", C.c_void_p)]


class _PageSelection(C.Structure):
    _fields_ = [("n_sink_pages", C.c_int32), ("n_tail_pages", C.c_int32), ("topk_pages", C.c_int32)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libtkphi.so (built in-tree by ``paper_2604_05438_b200.build``); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                           "`python -m paper_2604_05438_b200.build` (there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    lib.tkphi_workspace_bytes.restype = C.c_size_t
    lib.tkphi_workspace_bytes.argtypes = [C.POINTER(_KvDesc), C.c_void_p, C.c_int32, C.c_int]
    lib.tkphi_build_summaries.restype = C.c_int
    lib.tkphi_build_summaries.argtypes = [C.POINTER(_KvDesc), C.POINTER(_PhiDesc), C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_build_summaries_static.restype = C.c_int
    lib.tkphi_build_summaries_static.argtypes = [C.POINTER(_KvDesc), C.POINTER(_PhiDesc), C.c_void_p, C.c_void_p,
                                                 C.c_void_p]
    lib.tkphi_static_last_error.restype = C.c_char_p
    lib.tkphi_static_device_status.restype = C.c_int
    lib.tkphi_static_device_status.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
    lib.tkphi_selftest_timeout.restype = C.c_int
    lib.tkphi_selftest_timeout.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_topk_decode.restype = C.c_int
    lib.tkphi_topk_decode.argtypes = [C.POINTER(_KvDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_decode_step.restype = C.c_int
    lib.tkphi_decode_step.argtypes = [C.POINTER(_KvDesc), C.POINTER(_PhiDesc), C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_mlp_key_features.restype = C.c_int
    lib.tkphi_mlp_key_features.argtypes = [C.POINTER(_KvDesc), C.POINTER(_MlpDesc), C.c_void_p, C.c_void_p, C.c_size_t,
                                           C.c_void_p]
    lib.tkphi_build_summaries_cached.restype = C.c_int
    lib.tkphi_build_summaries_cached.argtypes = [C.POINTER(_KvDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                 C.c_size_t, C.c_void_p]
    lib.tkphi_decode_step_mlp.restype = C.c_int
    lib.tkphi_decode_step_mlp.argtypes = [C.POINTER(_KvDesc), C.POINTER(_MlpDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_paged_workspace_bytes.restype = C.c_size_t
    lib.tkphi_paged_workspace_bytes.argtypes = [C.POINTER(_PagedDesc), C.POINTER(_PageSelection), C.c_int]
    lib.tkphi_paged_append.restype = C.c_int
    lib.tkphi_paged_append.argtypes = [C.POINTER(_PagedDesc), C.POINTER(_AppendDesc), C.c_void_p]
    lib.tkphi_paged_attention.restype = C.c_int
    lib.tkphi_paged_attention.argtypes = [C.POINTER(_PagedDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                          C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_paged_block_attention.restype = C.c_int
    lib.tkphi_paged_block_attention.argtypes = [C.POINTER(_PagedDesc), C.POINTER(_PageSelection), C.c_void_p, C.c_void_p,
                                                C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_paged_append_norm.restype = C.c_int
    lib.tkphi_paged_append_norm.argtypes = [C.POINTER(_PagedDesc), C.POINTER(_AppendDesc), C.POINTER(_NormDesc), C.c_void_p]
    lib.tkphi_coded_append.restype = C.c_int
    lib.tkphi_coded_append.argtypes = [C.POINTER(_CodedDesc), C.POINTER(_AppendDesc), C.POINTER(_NormDesc), C.c_void_p]
    lib.tkphi_coded_read.restype = C.c_int
    lib.tkphi_coded_read.argtypes = [C.POINTER(_CodedDesc), C.POINTER(_ReadDesc), C.c_void_p]
    lib.tkphi_coded_workspace_bytes.restype = C.c_size_t
    lib.tkphi_coded_workspace_bytes.argtypes = [C.POINTER(_CodedDesc), C.POINTER(_PageSelection), C.c_int]
    lib.tkphi_coded_attention.restype = C.c_int
    lib.tkphi_coded_attention.argtypes = [C.POINTER(_CodedDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_float,
                                           C.c_uint32, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_coded_block_attention.restype = C.c_int
    lib.tkphi_coded_block_attention.argtypes = [C.POINTER(_CodedDesc), C.POINTER(_PageSelection), C.c_void_p, C.c_void_p,
                                                 C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.tkphi_device_status.restype = C.c_int
    lib.tkphi_device_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
    lib.tkphi_kernel_timing_enable.restype = None
    lib.tkphi_kernel_timing_enable.argtypes = [C.c_int32]
    lib.tkphi_kernel_timing_read.restype = C.c_int
    lib.tkphi_kernel_timing_read.argtypes = [C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.tkphi_last_error.restype = C.c_char_p
    lib.tkphi_version.restype = C.c_int32
    _lib = lib
    return lib


def _check(status: int):
    if status != 0:
        raise TkphiError(status, load_library().tkphi_last_error().decode())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream, kv: Optional["KVCache"] = None) -> Optional[int]:
    """The stream's handle; what kv made itself is marked as used there."""
    if stream is None:      # (the raw handle: building a Stream object for it takes longer than a kernel launch)
        raw = torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    else:
        raw = stream.cuda_stream
    if kv is not None and kv._made and raw != kv._made_on:
        for t in kv._made:
            t.record_stream(torch.cuda.current_stream() if stream is None else stream)
    return raw or None


@dataclass
class KVCache:
    """One layer's ragged K/V cache as the library sees it (no copies are made).

    k, v: bf16 device tensors addressed as [head, row, dim] through the strides
    (any layout whose innermost dim is contiguous).  cu_seqlens: int64 host array
    [batch+1]; a device copy is kept alongside (its memory is not handed out again
    before calls on other streams that read it are complete).
    """
    k: torch.Tensor
    v: torch.Tensor
    cu_seqlens: np.ndarray
    n_q_heads: int
    n_feat: int
    n_sink: int
    n_tail: int
    cu_seqlens_dev: Optional[torch.Tensor] = None
    n_tail_seq: Optional[np.ndarray] = None        # int32 [batch]: per-sequence tail-anchor counts (replace n_tail)
    n_tail_seq_dev: Optional[torch.Tensor] = None

    def __post_init__(self):
        self.cu_seqlens = np.ascontiguousarray(self.cu_seqlens, dtype=np.int64)
        self._made = []                            # device tensors that the caller does not know
        if self.cu_seqlens_dev is None:
            self.cu_seqlens_dev = torch.from_numpy(self.cu_seqlens).to(self.k.device)
            self._made.append(self.cu_seqlens_dev)
        if self.n_tail_seq is not None:
            self.n_tail_seq = np.ascontiguousarray(self.n_tail_seq, dtype=np.int32)
            assert self.n_tail_seq.shape == (len(self.cu_seqlens) - 1,)
            if self.n_tail_seq_dev is None:
                self.n_tail_seq_dev = torch.from_numpy(self.n_tail_seq).to(self.k.device)
                self._made.append(self.n_tail_seq_dev)
        self._made_on = torch._C._cuda_getCurrentRawStream(self.k.get_device()) if self.k.is_cuda else None

    @property
    def batch(self) -> int:
        return len(self.cu_seqlens) - 1

    def desc(self) -> _KvDesc:
        k, v = self.k, self.v
        assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16 and k.dim() == 3
        assert k.stride() == v.stride() and k.stride(2) == 1
        return _KvDesc(self.batch, self.n_q_heads, k.shape[0], k.shape[2], self.n_feat, self.n_sink,
                       self.n_tail, self.cu_seqlens.ctypes.data, self.cu_seqlens_dev.data_ptr(),
                       k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1),
                       None if self.n_tail_seq is None else self.n_tail_seq.ctypes.data,
                       None if self.n_tail_seq is None else self.n_tail_seq_dev.data_ptr())


@dataclass
class PhiMaps:
    """fp32 device parameters of phi(x) = exp(W x + b - gamma |x|^2)."""
    w_q: torch.Tensor
    b_q: torch.Tensor
    w_k: torch.Tensor
    b_k: torch.Tensor
    gamma_q: float
    gamma_k: float
    phi_k_cache: Optional[torch.Tensor] = None   # optional fp32 [n_kv_heads][T_total][n_feat]: written by the build, read by decode_step

    def desc(self) -> _PhiDesc:
        for t in (self.w_q, self.b_q, self.w_k, self.b_k):
            assert t.dtype == torch.float32 and t.is_contiguous()
        cache = None
        if self.phi_k_cache is not None:
            assert self.phi_k_cache.dtype == torch.float32 and self.phi_k_cache.is_contiguous()
            cache = self.phi_k_cache.data_ptr()
        return _PhiDesc(self.w_q.data_ptr(), self.b_q.data_ptr(), self.w_k.data_ptr(), self.b_k.data_ptr(),
                        float(self.gamma_q), float(self.gamma_k), cache)


@dataclass
class MlpMaps:
    """fp32 device parameters of one side's ReZero-MLP feature maps (App. C.2): phi(x) =
    exp(W_o (g0 + alpha (W_2 GeLU(W_1 g0 + b_1) + b_2)) + b_o), g0 = W_s x + b_s; leading dim = heads."""
    w_s: torch.Tensor
    b_s: torch.Tensor
    w_1: torch.Tensor
    b_1: torch.Tensor
    w_2: torch.Tensor
    b_2: torch.Tensor
    alpha: torch.Tensor
    w_o: torch.Tensor
    b_o: torch.Tensor

    def desc(self) -> _MlpDesc:
        ts = (self.w_s, self.b_s, self.w_1, self.b_1, self.w_2, self.b_2, self.alpha, self.w_o, self.b_o)
        for t in ts:
            assert t.dtype == torch.float32 and t.is_contiguous()
        return _MlpDesc(self.w_1.shape[1], self.w_s.shape[0], *[t.data_ptr() for t in ts])


_native_module = None


def _native():
    """The CPython module of the paged calls (built in-tree beside libtkphi.so); raises if absent or built for another torch."""
    global _native_module
    if _native_module is None:
        load_library()
        try:
            from . import _paged_binding
        except ImportError as e:
            raise RuntimeError("_paged_binding.so is missing or does not load: build it with "
                               "`python -m paper_2604_05438_b200.build`") from e
        if _paged_binding.torch_version != torch.__version__:
            raise RuntimeError(f"_paged_binding.so was built for torch {_paged_binding.torch_version}, this is "
                               f"{torch.__version__}: build it again with `python -m paper_2604_05438_b200.build`")
        _native_module = _paged_binding
    return _native_module


_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


class PagedKVCache:
    """One step of a batch of sequences over a paged K/V cache, as the library sees it (no copies of the cache are made).

    k, v: device tensors of one 16-bit type addressed as [page, head, slot, dim] through their (equal) strides; a cache
    stored [page, slot, head, dim] is passed as its ``transpose(1, 2)``.  page_table: int32 device [batch, max_pages].
    kv_lens: int64 host [batch], cache lengths with this step's new tokens; cu_q: int64 host [batch+1], the new tokens'
    rows; device copies are kept alongside.  key_bounds: [n_pages, n_kv_heads, 2, head_dim] or None.  status: device
    int32 word in which the kernels leave errors (made here, zero, unless given); ``device_status()`` reads it.

    What is made here may be used on any stream: a call on another stream than the one that was current here waits for it
    there, and its memory is not handed out again before that call is complete.  The caller's own tensors are the caller's to
    order and keep, here and in the calls.  With kv_lens_dev and cu_q_dev given nothing is copied and nothing waited for.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, kv_lens, cu_q, n_q_heads: int,
                 key_bounds: Optional[torch.Tensor] = None, kv_lens_dev: Optional[torch.Tensor] = None,
                 cu_q_dev: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
        assert k.dtype in _DTYPES
        self.dtype = k.dtype
        self._set(k, v, page_table, kv_lens, cu_q, n_q_heads, key_bounds, kv_lens_dev, cu_q_dev, status)

    def _set(self, k, v, page_table, kv_lens, cu_q, n_q_heads, key_bounds, kv_lens_dev, cu_q_dev, status):
        dev = k.device
        self.k, self.v, self.page_table, self.key_bounds, self.n_q_heads = k, v, page_table, key_bounds, n_q_heads
        # the descriptor points to these copies, and calls are checked against them: they do not change any more
        self.kv_lens, self.cu_q = np.array(kv_lens, dtype=np.int64), np.array(cu_q, dtype=np.int64)
        self.kv_lens.setflags(write=False)
        self.cu_q.setflags(write=False)
        assert v.dtype == k.dtype and k.dim() == 4 and v.shape == k.shape
        assert k.stride() == v.stride() and k.stride(3) == 1
        assert self.kv_lens.ndim == 1 and self.cu_q.shape == (len(self.kv_lens) + 1,)
        assert page_table.dtype == torch.int32 and page_table.dim() == 2 and page_table.is_contiguous()
        assert page_table.shape[0] == len(self.kv_lens)
        if key_bounds is not None:
            assert key_bounds.dtype == self.dtype and key_bounds.is_contiguous()
            assert key_bounds.shape == (k.shape[0], k.shape[1], 2, k.shape[3])
        made = ()
        if kv_lens_dev is None or cu_q_dev is None:
            # lengths, cu_q and status in one copy, which is complete when it returns
            made = (torch.from_numpy(np.concatenate([self.kv_lens, self.cu_q, [0]])).to(dev),)
            lens, cu, word = made[0].split([len(self.kv_lens), len(self.cu_q), 1])
            kv_lens_dev = lens if kv_lens_dev is None else kv_lens_dev
            cu_q_dev = cu if cu_q_dev is None else cu_q_dev
            status = word.view(torch.int32)[:1] if status is None else status
            pending = False
        elif status is None:
            status = torch.zeros(1, dtype=torch.int32, device=dev)
            made, pending = (status,), True
        self.kv_lens_dev, self.cu_q_dev, self.status = kv_lens_dev, cu_q_dev, status
        for t, a in ((self.kv_lens_dev, self.kv_lens), (self.cu_q_dev, self.cu_q)):
            assert t.dtype == torch.int64 and t.shape == a.shape and t.is_contiguous()
        assert self.status.dtype == torch.int32 and self.status.numel() == 1
        for t in (v, page_table, key_bounds, self.kv_lens_dev, self.cu_q_dev, self.status):
            assert t is None or t.device == dev, "the cache, its page table and its lengths must be on one device"
        self.total_q = int(self.cu_q[-1])
        step = _PagedDesc(len(self.kv_lens), n_q_heads, k.shape[1], k.shape[3], _DTYPES[self.dtype], k.shape[2],
                          k.shape[0], page_table.shape[1], k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1),
                          k.stride(2), page_table.data_ptr(), self.kv_lens.ctypes.data, self.kv_lens_dev.data_ptr(),
                          self.cu_q.ctypes.data, self.cu_q_dev.data_ptr(),
                          None if key_bounds is None else key_bounds.data_ptr(), self.status.data_ptr())
        self._desc = self._descriptor(step)
        self._handle = _native().handle(C.addressof(self._desc), k.get_device(), made, bool(made) and pending, self.held8)

    held8 = False            # the cache is in 8 bits

    def _descriptor(self, step: _PagedDesc):
        return step

    @property
    def batch(self) -> int:
        return len(self.kv_lens)

    def desc(self):
        return self._desc

    def device_status(self) -> int:
        """0, or the error that a call on this descriptor's status word left there (waits for all streams of the device)."""
        if self.status.is_cuda:
            torch.cuda.synchronize(self.status.device)
        return int(self.status.item())


class PagedKVCache8(PagedKVCache):
    """One step of a batch of sequences over a paged K/V cache in 8 bits: the paged calls take it as they take a PagedKVCache.

    k, v: float8_e4m3fn codes, addressed [page, head, slot, dim] as there; k_scales, v_scales: float8_e8m0fnu
    [n_pages, n_kv_heads, page_size], a power of two for each row (0 for codes and 0 for scales is an empty cache).  dtype:
    bfloat16 or float16, the type of queries, outputs, new tokens, key_bounds and rows read back.  Everything else as there.
    """

    held8 = True

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scales: torch.Tensor, v_scales: torch.Tensor, page_table: torch.Tensor,
                 kv_lens, cu_q, n_q_heads: int, dtype: torch.dtype, key_bounds: Optional[torch.Tensor] = None,
                 kv_lens_dev: Optional[torch.Tensor] = None, cu_q_dev: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None):
        assert k.dtype == torch.float8_e4m3fn and dtype in _DTYPES
        for t in (k_scales, v_scales):
            assert t.dtype == torch.float8_e8m0fnu and t.is_contiguous() and t.shape == k.shape[:3]
            assert t.device == k.device, "the cache, its page table and its lengths must be on one device"
        self.dtype, self.k_scales, self.v_scales = dtype, k_scales, v_scales
        self._set(k, v, page_table, kv_lens, cu_q, n_q_heads, key_bounds, kv_lens_dev, cu_q_dev, status)

    def _descriptor(self, step: _PagedDesc):
        return _CodedDesc(step, self.k_scales.data_ptr(), self.v_scales.data_ptr())


class CacheRows:
    """Rows of an 8-bit cache that paged_read takes: output row cu_rows[b] + i gets position first[b] + i of sequence b (first
    None: 0).  Device copies are made here (one copy, which is complete when it returns) unless given."""

    def __init__(self, cu_rows, first=None, device=None, cu_rows_dev: Optional[torch.Tensor] = None,
                 first_dev: Optional[torch.Tensor] = None):
        self.cu_rows = np.array(cu_rows, dtype=np.int64)
        self.first = None if first is None else np.array(first, dtype=np.int64)
        assert self.cu_rows.ndim == 1 and len(self.cu_rows) > 1
        assert self.first is None or self.first.shape == (len(self.cu_rows) - 1,)
        assert first_dev is None or first is not None, "first_dev is a device copy of first"
        made = ()
        if cu_rows_dev is None or (first is not None and first_dev is None):
            both = self.cu_rows if first is None else np.concatenate([self.cu_rows, self.first])
            made = (torch.from_numpy(both).to(device),)
            parts = made[0].split([len(self.cu_rows), len(both) - len(self.cu_rows)])
            cu_rows_dev = parts[0] if cu_rows_dev is None else cu_rows_dev
            first_dev = parts[1] if first is not None and first_dev is None else first_dev
        for t, a in ((cu_rows_dev, self.cu_rows), (first_dev, self.first)):
            assert t is None or (t.dtype == torch.int64 and t.shape == a.shape and t.is_contiguous() and t.device == cu_rows_dev.device)
        self.cu_rows_dev, self.first_dev = cu_rows_dev, first_dev
        for a in (self.cu_rows, self.first):
            if a is not None:
                a.setflags(write=False)
        self._desc = _ReadDesc(self.cu_rows.ctypes.data, cu_rows_dev.data_ptr(), None if first is None else self.first.ctypes.data,
                               None if first is None else first_dev.data_ptr())
        self._handle = _native().rows(C.addressof(self._desc), cu_rows_dev.get_device(), len(self.cu_rows) - 1, int(self.cu_rows[-1]), made)

    @property
    def total(self) -> int:
        return int(self.cu_rows[-1])


@dataclass
class HeadNorms:
    """Root-mean-square norms of the new tokens' heads before the rotation: x * weight / sqrt(mean(x^2) + eps), each head on
    its own.  Weights: fp32 device [head_dim] (for all heads) or [heads, head_dim]; a None side is not normed."""
    q_weight: Optional[torch.Tensor]
    k_weight: Optional[torch.Tensor]
    eps: float = 1e-6

    def __post_init__(self):
        for w in (self.q_weight, self.k_weight):
            assert w is None or (w.dtype == torch.float32 and w.dim() in (1, 2) and w.is_contiguous())


@dataclass
class RotaryMap:
    """Position rotation: fp32 device inv_freq [rot_dim / 2] (angle per position); pairs: neighbouring dims are partners
    (otherwise dim c and dim c + rot_dim / 2)."""
    inv_freq: torch.Tensor
    pairs: bool = False

    def __post_init__(self):
        assert self.inv_freq.dtype == torch.float32 and self.inv_freq.dim() == 1 and self.inv_freq.is_contiguous()


@dataclass
class PageSelection:
    """Pages that paged_block_attention reads: the first n_sink_pages, the last n_tail_pages, topk_pages between."""
    n_sink_pages: int
    n_tail_pages: int
    topk_pages: int

    @property
    def n_pages(self) -> int:
        return self.n_sink_pages + self.n_tail_pages + self.topk_pages

    def desc(self) -> _PageSelection:
        return _PageSelection(self.n_sink_pages, self.n_tail_pages, self.topk_pages)


def _topk_host(topk) -> np.ndarray:
    return np.ascontiguousarray(topk, dtype=np.int32)


def workspace_bytes(kv: KVCache, topk_host, topk_max: int, which: int) -> int:
    lib = load_library()
    d = kv.desc()
    th = None if topk_host is None else _topk_host(topk_host)
    n = lib.tkphi_workspace_bytes(C.byref(d), None if th is None else th.ctypes.data, int(topk_max), which)
    if n == 0:
        raise TkphiError(-1, lib.tkphi_last_error().decode())
    return int(n)


def build_summaries(kv: KVCache, phi: PhiMaps, S: torch.Tensor, u: torch.Tensor,
                    workspace: torch.Tensor, stream=None) -> None:
    lib = load_library()
    d, ph = kv.desc(), phi.desc()
    _check(lib.tkphi_build_summaries(C.byref(d), C.byref(ph), S.data_ptr(), u.data_ptr(),
                                     workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                     _stream_ptr(stream, kv)))


def build_summaries_static(kv: KVCache, phi: PhiMaps, S: torch.Tensor, u: torch.Tensor, stream=None) -> None:
    """Summary build on the library's built-in scratch: for callers that may not
    allocate device memory.  Problems needing more than STATIC_SCRATCH_BYTES of
    scratch raise TkphiError (status -3).  Calls that overlap on the GPU race."""
    lib = load_library()
    d, ph = kv.desc(), phi.desc()
    st = lib.tkphi_build_summaries_static(C.byref(d), C.byref(ph), S.data_ptr(), u.data_ptr(), _stream_ptr(stream, kv))
    if st != 0:
        raise TkphiError(st, lib.tkphi_static_last_error().decode())


def static_device_status(stream=None) -> int:
    """Status word of the last build_summaries_static call on the current device (0 = fine)."""
    lib = load_library()
    out = C.c_int32(0)
    st = lib.tkphi_static_device_status(_stream_ptr(stream), C.byref(out))
    if st != 0:
        raise TkphiError(st, lib.tkphi_static_last_error().decode())
    return int(out.value)


def selftest_timeout(workspace: torch.Tensor, stream=None) -> None:
    """Runs the library's bounded-wait self-test kernel; device_status(workspace) then reads ERR_TIMEOUT."""
    lib = load_library()
    _check(lib.tkphi_selftest_timeout(workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                      _stream_ptr(stream)))


def mlp_key_features(kv: KVCache, mlp_k: MlpMaps, phi_k_cache: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    lib = load_library()
    d, m = kv.desc(), mlp_k.desc()
    _check(lib.tkphi_mlp_key_features(C.byref(d), C.byref(m), phi_k_cache.data_ptr(), workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), _stream_ptr(stream, kv)))


def build_summaries_cached(kv: KVCache, phi_k_cache: torch.Tensor, S: torch.Tensor, u: torch.Tensor,
                           workspace: torch.Tensor, stream=None) -> None:
    lib = load_library()
    d = kv.desc()
    _check(lib.tkphi_build_summaries_cached(C.byref(d), phi_k_cache.data_ptr(), S.data_ptr(), u.data_ptr(),
                                            workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                            _stream_ptr(stream, kv)))


def decode_step_mlp(kv: KVCache, mlp_q: MlpMaps, phi_k_cache: Optional[torch.Tensor], q: torch.Tensor, topk_host,
                    topk_dev: torch.Tensor, topk_max: int, S: torch.Tensor, u: torch.Tensor,
                    idx_out: Optional[torch.Tensor], y_out: torch.Tensor, dbg_out: Optional[torch.Tensor], flags: int,
                    workspace: torch.Tensor, stream=None) -> None:
    lib = load_library()
    d, m = kv.desc(), mlp_q.desc()
    th = _topk_host(topk_host)
    _check(lib.tkphi_decode_step_mlp(C.byref(d), C.byref(m), _ptr(phi_k_cache), q.data_ptr(), th.ctypes.data,
                                     topk_dev.data_ptr(), int(topk_max), S.data_ptr(), u.data_ptr(), _ptr(idx_out),
                                     y_out.data_ptr(), _ptr(dbg_out), int(flags), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), _stream_ptr(stream, kv)))


def topk_decode(kv: KVCache, q: torch.Tensor, topk_host, topk_dev: torch.Tensor, topk_max: int,
                idx_out: Optional[torch.Tensor], y_out: torch.Tensor, workspace: torch.Tensor,
                stream=None) -> None:
    lib = load_library()
    d = kv.desc()
    th = _topk_host(topk_host)
    _check(lib.tkphi_topk_decode(C.byref(d), q.data_ptr(), th.ctypes.data, topk_dev.data_ptr(), int(topk_max),
                                 _ptr(idx_out), y_out.data_ptr(), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream_ptr(stream, kv)))


def decode_step(kv: KVCache, phi: PhiMaps, q: torch.Tensor, topk_host, topk_dev: torch.Tensor,
                topk_max: int, S: torch.Tensor, u: torch.Tensor, idx_out: Optional[torch.Tensor],
                y_out: torch.Tensor, dbg_out: Optional[torch.Tensor], flags: int,
                workspace: torch.Tensor, stream=None) -> None:
    lib = load_library()
    d, ph = kv.desc(), phi.desc()
    th = _topk_host(topk_host)
    _check(lib.tkphi_decode_step(C.byref(d), C.byref(ph), q.data_ptr(), th.ctypes.data, topk_dev.data_ptr(),
                                 int(topk_max), S.data_ptr(), u.data_ptr(), _ptr(idx_out), y_out.data_ptr(),
                                 _ptr(dbg_out), int(flags), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream_ptr(stream, kv)))


def paged_workspace_bytes(kv: PagedKVCache, which: int, selection: Optional[PageSelection] = None) -> int:
    lib = load_library()
    sel = None if selection is None else C.byref(selection.desc())
    ask = lib.tkphi_coded_workspace_bytes if kv.held8 else lib.tkphi_paged_workspace_bytes
    with torch.cuda.device(kv.k.device):          # the plan goes by the device's multiprocessors
        n = ask(C.byref(kv.desc()), sel, which)
    if n == 0:
        raise TkphiError(-1, lib.tkphi_last_error().decode())
    return int(n)


def paged_append(kv: PagedKVCache, k_new: torch.Tensor, v_new: torch.Tensor, rotary: Optional[RotaryMap] = None,
                 q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 positions: Optional[torch.Tensor] = None, stream=None, norms: Optional[HeadNorms] = None) -> None:
    """Rotates the new keys (and q into q_out) by their positions and writes keys and values into the cache's pages, rounded to
    8 bits where kv is a PagedKVCache8; key bounds of the touched pages follow.  norms: the heads' norms before the rotation.
    k_new, v_new, q, q_out: [total_q, heads, head_dim], any token and head strides; positions: int64 [total_q] or None for
    the cache positions."""
    inv, pairs = (None, False) if rotary is None else (rotary.inv_freq, rotary.pairs)
    if norms is None:
        st = _native().append(kv._handle, k_new, v_new, inv, pairs, q, q_out, positions, stream)
    else:
        st = _native().append_norm(kv._handle, k_new, v_new, inv, pairs, q, q_out, positions, norms.q_weight, norms.k_weight,
                                   norms.eps, stream)
    if st:
        _check(st)


def paged_read(kv: PagedKVCache8, rows: CacheRows, k_out: Optional[torch.Tensor], v_out: Optional[torch.Tensor], stream=None) -> None:
    """What rows of an 8-bit cache stand for, as 16-bit rows: k_out, v_out [rows.total, n_kv_heads, head_dim] of kv's dtype, any
    row and head strides (a [head, row, dim] array is passed as its transpose(0, 1)), either may be None."""
    st = _native().read(kv._handle, rows._handle, k_out, v_out, stream)
    if st:
        _check(st)


def paged_attention(kv: PagedKVCache, q: torch.Tensor, y_out: torch.Tensor, lse_out: Optional[torch.Tensor],
                    scale: Optional[float], flags: int, workspace: torch.Tensor, stream=None) -> None:
    """Attention of the step's new tokens over their sequences' whole caches (of 16 or of 8 bits); q, y_out [total_q, n_q_heads, head_dim],
    lse_out fp32 [total_q, n_q_heads] or None, scale None for 1/sqrt(head_dim), flags FLAG_NONE or FLAG_FULL_CONTEXT."""
    st = _native().attention(kv._handle, q, y_out, lse_out, scale, flags, workspace, stream)
    if st:
        _check(st)


def paged_block_attention(kv: PagedKVCache, selection: PageSelection, q: torch.Tensor, y_out: torch.Tensor,
                          lse_out: Optional[torch.Tensor], page_idx_out: Optional[torch.Tensor], scale: Optional[float],
                          workspace: torch.Tensor, stream=None) -> None:
    """Attention over the pages that ``selection`` takes for each new token and KV head; page_idx_out int32
    [total_q, n_kv_heads, selection.n_pages] or None gets them."""
    st = _native().block_attention(kv._handle, selection.n_sink_pages, selection.n_tail_pages, selection.topk_pages, q,
                                   y_out, lse_out, page_idx_out, scale, workspace, stream)
    if st:
        _check(st)


def device_status(workspace: torch.Tensor, stream=None) -> int:
    lib = load_library()
    out = C.c_int32(0)
    _check(lib.tkphi_device_status(workspace.data_ptr(), _stream_ptr(stream), C.byref(out)))
    return int(out.value)


def kernel_timing(fn) -> dict:
    """Run ``fn()`` with the library's per-kernel event timing on; returns
    {kind: {"ms": total, "launches": n, "avg_ms": ms/n}} for the kinds that ran."""
    lib = load_library()
    lib.tkphi_kernel_timing_enable(1)
    try:
        fn()
        torch.cuda.synchronize()
        ms = (C.c_float * len(KERNEL_KINDS))()
        cnt = (C.c_int32 * len(KERNEL_KINDS))()
        _check(lib.tkphi_kernel_timing_read(ms, cnt))
    finally:
        lib.tkphi_kernel_timing_enable(0)
    return {k: {"ms": float(ms[i]), "launches": int(cnt[i]), "avg_ms": float(ms[i]) / cnt[i]}
            for i, k in enumerate(KERNEL_KINDS) if cnt[i] > 0}
