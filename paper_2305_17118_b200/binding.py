"""ctypes binding of libscissorhands.so: argument marshalling only.

Every function mirrors one entry point of ``include/scissorhands.h``.  Device
buffers are torch CUDA tensors (PyTorch is used for device memory and streams
only); the kernels do all of the method's work.  There is no CPU fallback: if
the library cannot be loaded this module raises at import.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Tuple

import numpy as np
import torch

from . import build as _build

SH_OK, SH_EINVAL, SH_EFULL, SH_ESTATE, SH_ECUDA, SH_ENOMEM, SH_ETOOBIG, SH_EDEVICE = 0, -1, -2, -3, -4, -5, -6, -7
SH_STATIC_SCRATCH_MAX_ENTRIES = 1 << 20
SH_F32, SH_F16, SH_BF16, SH_INT4_G64_F16 = 0, 1, 2, 3
SH_OPT_SOFTMAX_SCALE, SH_OPT_SPLIT, SH_OPT_AUTO_COMPRESS, SH_OPT_DECODE_KERNEL, SH_OPT_PREFILL_CHUNK, SH_OPT_RECORD_MODE = 0, 1, 2, 3, 4, 5
SH_OPT_COMPACTION = 6
SH_OPT_SELFTEST_SKIP_TILE = 7
SH_SELECT_MAX_N = 40000

DTYPE_CODE = {"f32": SH_F32, "f16": SH_F16, "bf16": SH_BF16, "int4": SH_INT4_G64_F16}
INPUT_TORCH_DTYPE = {SH_F32: torch.float32, SH_F16: torch.float16, SH_BF16: torch.bfloat16,
                     SH_INT4_G64_F16: torch.float16}

EXPORTS = ["sh_create", "sh_destroy", "sh_workspace_bytes", "sh_bind", "sh_set_option", "sh_decode_step",
           "sh_decode_step_host", "sh_prefill", "sh_prefill_chunk", "sh_prefill_chunk_max", "sh_export_record", "sh_recompute_record", "sh_prefill_ragged",
           "sh_sequence_state",
           "sh_compress", "sh_compress_static", "sh_scores", "sh_select", "sh_state", "sh_export_unit",
           "sh_restore", "sh_launch_count", "sh_decode_kernel_choice", "sh_import_compressed", "sh_prefill_bulk",
           "sh_prefill_bulk_scratch_bytes", "sh_strerror", "sh_last_cuda_error",
           "sh_qk_norm_rope", "sh_window_prefill", "sh_window_append", "sh_window_decode", "sh_window_decode_workspace_bytes", "sh_window_prefill_workspace_bytes", "sh_window_status",
           "sh_context_attention", "sh_context_attention_workspace_bytes", "sh_mass_prefill", "sh_mass_prefill_workspace_bytes", "sh_mass_decode",
           "sh_mass_decode_workspace_bytes", "sh_mass_evict", "sh_mass_evict_workspace_bytes"]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_longlong), ("head_stride", C.c_longlong)]


class _WindowCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("sequence_stride", C.c_longlong), ("head_stride", C.c_longlong),
                ("slot_stride", C.c_longlong)]


class _Window(C.Structure):
    _fields_ = [("dtype", C.c_int), ("head_dim", C.c_int), ("q_heads", C.c_int), ("kv_heads", C.c_int), ("window", C.c_int),
                ("sinks", C.c_int), ("scale", C.c_double)]


class _Rope(C.Structure):
    _fields_ = [("dtype", C.c_int), ("head_dim", C.c_int), ("rot_dim", C.c_int), ("axes", C.c_int), ("sections", C.c_int * 3),
                ("spread", C.c_int), ("adjacent_pairs", C.c_int), ("eps", C.c_float), ("inv_freq_dev", C.c_void_p),
                ("q_weight_dev", C.c_void_p), ("k_weight_dev", C.c_void_p)]


class _Attention(C.Structure):
    _fields_ = [("dtype", C.c_int), ("head_dim", C.c_int), ("q_heads", C.c_int), ("kv_heads", C.c_int), ("slots", C.c_int), ("scale", C.c_double)]


class _Records(C.Structure):
    _fields_ = [("mass", C.c_void_p), ("positions", C.c_void_p), ("sequence_stride", C.c_longlong), ("head_stride", C.c_longlong)]


def _load() -> C.CDLL:
    path = _build.LIB
    if _build.stale():
        try:
            path = _build.build()
        except Exception as e:  # no nvcc here: use what was shipped, if anything
            if not os.path.exists(_build.LIB):
                raise ImportError(f"libscissorhands.so is not built and cannot be built: {e}") from e
    return declare(C.CDLL(path))


def declare(lib: C.CDLL) -> C.CDLL:
    """Argument and result types of every entry point, on a loaded build of the library."""
    vp, ip, llp = C.c_void_p, C.POINTER(C.c_int), C.POINTER(C.c_longlong)
    lib.sh_create.argtypes = [C.c_int] * 7 + [C.POINTER(vp)]
    lib.sh_destroy.argtypes = [vp]
    lib.sh_destroy.restype = None
    lib.sh_workspace_bytes.argtypes = [vp]
    lib.sh_workspace_bytes.restype = C.c_size_t
    lib.sh_bind.argtypes = [vp, vp, C.c_size_t, vp]
    lib.sh_set_option.argtypes = [vp, C.c_int, C.c_double]
    lib.sh_scores.argtypes = [vp, vp, vp, vp]
    lib.sh_decode_step.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.sh_decode_step_host.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.sh_prefill.argtypes = [vp, vp, vp, vp, C.c_int, vp, vp]
    lib.sh_prefill_chunk.argtypes = [vp, vp, vp, vp, C.c_int, vp, vp]
    lib.sh_prefill_chunk_max.argtypes = [vp]
    lib.sh_export_record.argtypes = [vp, C.c_int, vp, vp]
    lib.sh_recompute_record.argtypes = [vp, vp]
    lib.sh_prefill_ragged.argtypes = [vp, vp, vp, vp, C.c_int, ip, C.c_int, vp, vp]
    lib.sh_sequence_state.argtypes = [vp, ip, llp, C.c_int]
    lib.sh_compress.argtypes = [vp, vp, ip]
    lib.sh_compress_static.argtypes = [vp, vp, ip]
    lib.sh_select.argtypes = [vp, C.c_int, C.c_int, C.c_int, C.c_int, vp, vp]
    lib.sh_state.argtypes = [vp, vp, ip, llp, vp, vp, vp]
    lib.sh_export_unit.argtypes = [vp, C.c_int, vp, vp, vp]
    lib.sh_restore.argtypes = [vp, C.c_int, C.c_longlong]
    lib.sh_launch_count.argtypes = [vp]
    lib.sh_launch_count.restype = C.c_longlong
    lib.sh_decode_kernel_choice.argtypes = [vp]
    lib.sh_import_compressed.argtypes = [vp, vp, vp]
    lib.sh_prefill_bulk.argtypes = [vp, vp, vp, vp, C.c_int, vp, vp, C.c_size_t, vp]
    lib.sh_prefill_bulk_scratch_bytes.argtypes = [vp, C.c_int]
    lib.sh_prefill_bulk_scratch_bytes.restype = C.c_size_t
    lib.sh_strerror.argtypes = [C.c_int]
    lib.sh_strerror.restype = C.c_char_p
    lib.sh_last_cuda_error.argtypes = [vp]
    lib.sh_last_cuda_error.restype = C.c_char_p
    rows = cache = window = rope = vp      # (structs arrive as packed bytes or by reference)
    lib.sh_qk_norm_rope.argtypes = [rope, C.c_int, C.c_int, C.c_int, rows, rows, vp, C.c_longlong, rows, rows, vp]
    lib.sh_window_prefill.argtypes = [window, C.c_int, C.c_int, rows, rows, rows, vp, vp, cache, rows, vp, C.c_size_t, vp]
    lib.sh_window_prefill_workspace_bytes.argtypes = [window, C.c_int, C.c_int, C.c_int]
    lib.sh_window_prefill_workspace_bytes.restype = C.c_size_t
    lib.sh_window_append.argtypes = [window, C.c_int, C.c_int, rows, rows, vp, vp, cache, vp]
    lib.sh_window_status.argtypes = [vp]
    lib.sh_window_decode.argtypes = [window, C.c_int, rows, rows, rows, vp, cache, rope, vp, C.c_longlong, rows, vp, C.c_size_t, vp]
    lib.sh_window_decode_workspace_bytes.argtypes = [window, C.c_int]
    lib.sh_window_decode_workspace_bytes.restype = C.c_size_t
    attention = records = vp
    lib.sh_context_attention.argtypes = [attention, C.c_int, C.c_int, rows, cache, vp, vp, rows, C.c_int, vp, C.c_int, vp, C.c_size_t, vp]
    lib.sh_context_attention_workspace_bytes.argtypes = [attention, C.c_int, C.c_int, C.c_int]
    lib.sh_mass_prefill.argtypes = [attention, C.c_int, C.c_int, rows, rows, rows, vp, vp, vp, cache, records, rows, C.c_int, vp, rows, vp, C.c_size_t, vp]
    lib.sh_mass_prefill_workspace_bytes.argtypes = [attention, C.c_int, C.c_int]
    lib.sh_mass_decode.argtypes = [attention, C.c_int, rows, rows, rows, vp, vp, cache, records, rows, C.c_int, vp, rows, vp, C.c_size_t, vp]
    lib.sh_mass_decode_workspace_bytes.argtypes = [attention, C.c_int]
    lib.sh_mass_evict.argtypes = [attention, C.c_int, vp, cache, records, C.c_int, C.c_int, cache, records, C.c_int, vp, vp, C.c_size_t, vp]
    lib.sh_mass_evict_workspace_bytes.argtypes = [attention, C.c_int, C.c_int, C.c_int]
    for fn in (lib.sh_context_attention_workspace_bytes, lib.sh_mass_prefill_workspace_bytes, lib.sh_mass_decode_workspace_bytes,
               lib.sh_mass_evict_workspace_bytes):
        fn.restype = C.c_size_t
    return lib


lib = _load()


class ShError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        msg = lib.sh_strerror(status).decode()
        super().__init__(f"libscissorhands: {msg} ({status})" + (f": {detail}" if detail else ""))


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    return (stream or torch.cuda.current_stream()).cuda_stream


def _dev(t: torch.Tensor, dtype: torch.dtype, numel: int, what: str) -> int:
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype and t.numel() == numel):
        raise ValueError(f"{what}: need a contiguous CUDA tensor of {numel} x {dtype}, got "
                         f"{tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


class Handle:
    """One budgeted KV cache: ``heads`` independent units of one layer.

    Mirrors ``sh_create`` + ``sh_bind``; the workspace is a torch uint8 tensor
    owned by this object.
    """

    def __init__(self, B: int, r: int, w: int, m: int, heads: int, head_dim: int, dtype, device="cuda:0",
                 split: Optional[int] = None, scale: Optional[float] = None, auto_compress: bool = True,
                 kernel: Optional[int] = None, prefill_chunk: Optional[bool] = None, recompute_record: bool = False,
                 unordered: Optional[bool] = None):
        self.dtype = DTYPE_CODE[dtype] if isinstance(dtype, str) else int(dtype)
        self.B, self.r, self.w, self.m, self.U, self.D = B, r, w, m, heads, head_dim
        self.Bw = (B + 31) // 32
        self.device = torch.device(device)
        self.in_dtype = INPUT_TORCH_DTYPE.get(self.dtype, torch.float16)
        h = C.c_void_p()
        rc = lib.sh_create(B, r, w, m, heads, head_dim, self.dtype, C.byref(h))
        if rc:
            raise ShError(rc)
        self._h = h
        if scale is not None:
            self.set_option(SH_OPT_SOFTMAX_SCALE, scale)
        if split is not None:
            self.set_option(SH_OPT_SPLIT, split)
        if kernel is not None:
            self.set_option(SH_OPT_DECODE_KERNEL, kernel)
        if recompute_record:
            self.set_option(SH_OPT_RECORD_MODE, 1.0)
        if unordered is not None:
            self.set_option(SH_OPT_COMPACTION, 1.0 if unordered else 0.0)
        if prefill_chunk is not None:
            self.set_option(SH_OPT_PREFILL_CHUNK, float(int(prefill_chunk)))
        self.set_option(SH_OPT_AUTO_COMPRESS, 1.0 if auto_compress else 0.0)
        self.workspace_bytes = int(lib.sh_workspace_bytes(h))
        with torch.cuda.device(self.device):
            self.slab = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
            off = (-self.slab.data_ptr()) % 256
            self._slab_ptr = self.slab.data_ptr() + off
            self._slab_off = off
            self._check(lib.sh_bind(h, self._slab_ptr, self.workspace_bytes, _stream_ptr(None)))

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        if h and lib is not None:      # at interpreter shutdown the module globals may already be gone
            lib.sh_destroy(h)

    def _check(self, rc: int):
        if rc:
            raise ShError(rc, lib.sh_last_cuda_error(self._h).decode() if rc == SH_ECUDA else "")

    # -- sh_set_option -------------------------------------------------------
    def set_option(self, key: int, value: float):
        self._check(lib.sh_set_option(self._h, key, float(value)))

    # -- sh_decode_step ------------------------------------------------------
    def decode_step(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                    out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        n = self.U * self.D
        if out is None:
            out = torch.empty(self.U, self.D, dtype=torch.float32, device=self.device)
        self._check(lib.sh_decode_step(self._h, _dev(q, self.in_dtype, n, "q"), _dev(k_new, self.in_dtype, n, "k_new"),
                                       _dev(v_new, self.in_dtype, n, "v_new"), _dev(out, torch.float32, n, "out"),
                                       _stream_ptr(stream)))
        return out

    # -- sh_decode_step_host ---------------------------------------------------
    def decode_step_host(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor,
                         stream=None) -> torch.Tensor:
        n = self.U * self.D
        for t, dt, what in ((q, self.in_dtype, "q"), (k_new, self.in_dtype, "k_new"), (v_new, self.in_dtype, "v_new"),
                            (out, torch.float32, "out")):
            if t.is_cuda or not t.is_contiguous() or t.dtype != dt or t.numel() != n:
                raise ValueError(f"{what}: need a contiguous host tensor of {n} x {dt}")
        self._check(lib.sh_decode_step_host(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr(),
                                            _stream_ptr(stream)))
        return out

    def decode_step_host_raw(self, q_ptr: int, k_ptr: int, v_ptr: int, out_ptr: int, stream_ptr: int = 0):
        """sh_decode_step_host on raw host addresses the caller has validated once (contiguous rows of
        the handle's dtype, [heads, head_dim]; out fp32): no per-call tensor checks."""
        rc = lib.sh_decode_step_host(self._h, q_ptr, k_ptr, v_ptr, out_ptr, stream_ptr)
        if rc:
            self._check(rc)

    # -- sh_prefill ------------------------------------------------------------
    def prefill(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: Optional[torch.Tensor] = None,
                stream=None):
        p = q.shape[0]
        n = p * self.U * self.D
        optr = _dev(out, torch.float32, n, "out") if out is not None else None
        self._check(lib.sh_prefill(self._h, _dev(q, self.in_dtype, n, "q"), _dev(k, self.in_dtype, n, "k"),
                                   _dev(v, self.in_dtype, n, "v"), p, optr, _stream_ptr(stream)))
        return out

    # -- sh_import_compressed / sh_prefill_bulk -------------------------------------
    def import_compressed(self, src: "Handle", stream=None):
        self._check(lib.sh_import_compressed(self._h, src._h, _stream_ptr(stream)))

    def prefill_bulk(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: Optional[torch.Tensor] = None,
                     stream=None):
        p = q.shape[0]
        n = p * self.U * self.D
        need = int(lib.sh_prefill_bulk_scratch_bytes(self._h, p))
        if not need:
            raise ShError(SH_EINVAL, "prompt length outside 1..32767")
        with torch.cuda.device(self.device):
            scratch = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        sptr = scratch.data_ptr() + (-scratch.data_ptr()) % 256
        optr = _dev(out, torch.float32, n, "out") if out is not None else None
        self._check(lib.sh_prefill_bulk(self._h, _dev(q, self.in_dtype, n, "q"), _dev(k, self.in_dtype, n, "k"),
                                        _dev(v, self.in_dtype, n, "v"), p, optr, sptr, need, _stream_ptr(stream)))
        scratch.record_stream(stream or torch.cuda.current_stream())
        return out

    # -- sh_prefill_ragged / sh_sequence_state -----------------------------------
    def prefill_ragged(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lengths, out: Optional[torch.Tensor] = None,
                       stream=None):
        p = q.shape[0]
        n = p * self.U * self.D
        lens = (C.c_int * len(lengths))(*[int(x) for x in lengths])
        optr = _dev(out, torch.float32, n, "out") if out is not None else None
        self._check(lib.sh_prefill_ragged(self._h, _dev(q, self.in_dtype, n, "q"), _dev(k, self.in_dtype, n, "k"),
                                          _dev(v, self.in_dtype, n, "v"), p, lens, len(lengths), optr,
                                          _stream_ptr(stream)))
        return out

    def sequence_state(self):
        """(n [sequences], t [sequences]) host counters."""
        ns = lib.sh_sequence_state(self._h, None, None, 0)
        n_a, t_a = (C.c_int * ns)(), (C.c_longlong * ns)()
        lib.sh_sequence_state(self._h, n_a, t_a, ns)
        return np.array(n_a[:], dtype=np.int64), np.array(t_a[:], dtype=np.int64)

    def state_full(self, stream=None):
        """sh_state without trimming to a common n: (pos [U,B], counters [U,B], low [U,B] bool)."""
        pos_a = np.zeros((self.U, self.B), dtype=np.int32)
        cnt_a = np.zeros((self.U, self.B), dtype=np.uint16)
        low_a = np.zeros((self.U, self.Bw), dtype=np.uint32)
        self._check(lib.sh_state(self._h, _stream_ptr(stream), None, None, pos_a.ctypes.data, cnt_a.ctypes.data,
                                 low_a.ctypes.data))
        bits = np.unpackbits(low_a.view(np.uint8), axis=1, bitorder="little")[:, : self.B].astype(bool)
        return pos_a, cnt_a, bits

    # -- sh_prefill_chunk --------------------------------------------------------
    @property
    def prefill_chunk_max(self) -> int:
        return int(lib.sh_prefill_chunk_max(self._h))

    def prefill_chunk(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: Optional[torch.Tensor] = None,
                      stream=None):
        c = q.shape[0]
        n = c * self.U * self.D
        optr = _dev(out, torch.float32, n, "out") if out is not None else None
        self._check(lib.sh_prefill_chunk(self._h, _dev(q, self.in_dtype, n, "q"), _dev(k, self.in_dtype, n, "k"),
                                         _dev(v, self.in_dtype, n, "v"), c, optr, _stream_ptr(stream)))
        return out

    # -- sh_recompute_record --------------------------------------------------------
    def recompute_record(self, stream=None):
        self._check(lib.sh_recompute_record(self._h, _stream_ptr(stream)))

    # -- sh_export_record -----------------------------------------------------------
    def export_record(self, unit: int, stream=None) -> np.ndarray:
        """Bit-planes of one unit as a bool array [w, B]: entry (s mod w, j) is step s's comparison for slot j."""
        planes = np.zeros((self.w, self.Bw), dtype=np.uint32)
        self._check(lib.sh_export_record(self._h, unit, planes.ctypes.data, _stream_ptr(stream)))
        return np.unpackbits(planes.view(np.uint8), axis=1, bitorder="little")[:, : self.B].astype(bool)

    # -- sh_scores ---------------------------------------------------------------
    def scores(self, q: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention scores of ``q`` [U, d] over each unit's present cache: fp32 [U, B], 0 beyond the live slots."""
        if out is None:
            out = torch.empty(self.U, self.B, dtype=torch.float32, device=self.device)
        self._check(lib.sh_scores(self._h, _dev(q, self.in_dtype, self.U * self.D, "q"),
                                  _dev(out, torch.float32, self.U * self.B, "out"), _stream_ptr(stream)))
        return out

    # -- sh_compress -------------------------------------------------------------
    def compress(self, stream=None) -> int:
        ev = C.c_int(0)
        self._check(lib.sh_compress(self._h, _stream_ptr(stream), C.byref(ev)))
        return ev.value

    # -- sh_compress_static ----------------------------------------------------------
    def compress_static(self, stream=None) -> int:
        """sh_compress without any device allocation or workspace scratch: for
        callers that cannot cudaMalloc (all HBM already pooled, or inside a
        latency-critical loop).  Needs heads * B <= SH_STATIC_SCRATCH_MAX_ENTRIES;
        calls on one device must not overlap."""
        ev = C.c_int(0)
        self._check(lib.sh_compress_static(self._h, _stream_ptr(stream), C.byref(ev)))
        return ev.value

    # -- sh_state ------------------------------------------------------------------
    def state(self, pos: bool = True, counters: bool = True, low: bool = True, stream=None):
        """Returns ``(n, t, pos [U,n] int32 | None, counters [U,n] uint16 | None,
        low [U,n] bool | None)`` on the host."""
        n, t = C.c_int(0), C.c_longlong(0)
        pos_a = np.zeros((self.U, self.B), dtype=np.int32) if pos else None
        cnt_a = np.zeros((self.U, self.B), dtype=np.uint16) if counters else None
        low_a = np.zeros((self.U, self.Bw), dtype=np.uint32) if low else None
        ptr = lambda a: a.ctypes.data if a is not None else None
        self._check(lib.sh_state(self._h, _stream_ptr(stream), C.byref(n), C.byref(t), ptr(pos_a), ptr(cnt_a),
                                 ptr(low_a)))
        nn = n.value
        low_b = None
        if low:
            bits = np.unpackbits(low_a.view(np.uint8), axis=1, bitorder="little")
            low_b = bits[:, :nn].astype(bool)
            assert not bits[:, nn:].any(), "record bits set beyond the live slots"
        return (nn, t.value, pos_a[:, :nn] if pos else None, cnt_a[:, :nn] if counters else None, low_b)

    @property
    def n(self) -> int:
        n = C.c_int(0)
        self._check(lib.sh_state(self._h, _stream_ptr(None), C.byref(n), None, None, None, None))
        return n.value

    # -- sh_export_unit ---------------------------------------------------------------
    def export_unit(self, unit: int, stream=None) -> Tuple[np.ndarray, np.ndarray]:
        K = np.zeros((self.B, self.D), dtype=np.float32)
        V = np.zeros((self.B, self.D), dtype=np.float32)
        self._check(lib.sh_export_unit(self._h, unit, K.ctypes.data, V.ctypes.data, _stream_ptr(stream)))
        return K, V

    # -- checkpoint / sh_restore -------------------------------------------------------
    def snapshot(self):
        """Copy of the whole workspace plus the host counters that go with it."""
        n, t, *_ = self.state(pos=False, counters=False, low=False)
        return self.slab.clone(), n, t

    def restore(self, snap):
        slab, n, t = snap
        self.slab.copy_(slab)
        self._check(lib.sh_restore(self._h, n, t))

    @property
    def launch_count(self) -> int:
        return int(lib.sh_launch_count(self._h))

    @property
    def decode_kernel(self) -> str:
        """Name of the fused decode kernel sh_decode_step launches for this handle."""
        return {1: "sh_decode_kernel", 2: "sh_decode_tma_kernel", 3: "sh_decode_int4_mma_kernel"}[int(lib.sh_decode_kernel_choice(self._h))]


def select(counters: torch.Tensor, r: int, m: int, stream=None) -> torch.Tensor:
    """``sh_select``: counters ``[units, n]`` (CUDA, any integer dtype, values
    <= 16384) -> dropped indices ``[units, m]`` int32, ascending."""
    units, n = counters.shape
    c16 = counters.to(torch.int16).contiguous()   # values <= 16384: same bits as uint16
    out = torch.empty(units, m, dtype=torch.int32, device=counters.device)
    rc = lib.sh_select(c16.data_ptr(), units, n, r, m, out.data_ptr(), _stream_ptr(stream))
    if rc:
        raise ShError(rc)
    return out


# -- query/key preparation and the window cache (no handle: tensors in, tensors out) ---------------------------------
# The wrappers sit on the path of every decoded token, so they look at each tensor once and hand the structs over as bytes packed
# in C layout (the layout of _Rows, _WindowCache, _Window and _Rope above).
_CODE_OF = {torch.float32: SH_F32, torch.float16: SH_F16, torch.bfloat16: SH_BF16}
_pack_rows, _pack_cache = struct.Struct("Pqq").pack, struct.Struct("PPqqq").pack
_pack_window, _pack_rope = struct.Struct("iiiiiid").pack, struct.Struct("9ifPPP").pack
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device


def _fail(what: str, need: str, t) -> None:
    got = f"{tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}" if isinstance(t, torch.Tensor) else repr(t)
    raise ValueError(f"{what}: need {need}, got {got}")


def _head_rows(t, what: str):
    """Shape, type, device and packed sh_rows of rows [tokens, heads, head_dim]."""
    if isinstance(t, torch.Tensor) and t.dim() == 3:
        shape, dtype, device = t.shape, t.dtype, t.get_device()
        ts, hs, es = t.stride()
        if device >= 0 and dtype in _CODE_OF and (shape[2] == 64 or shape[2] == 128) and (es == 1 or t.numel() == 0):
            return shape, dtype, device, _pack_rows(t.data_ptr(), ts, hs)
    _fail(what, "a CUDA tensor [tokens, heads, 64 or 128] of f32, f16 or bf16 with contiguous rows", t)


def _more_rows(t, what: str, shape, dtype, device):
    """Packed sh_rows of a tensor that must look like the first one."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == shape):
        _fail(what, f"{tuple(shape)} of {dtype} on cuda:{device}", t)
    ts, hs, es = t.stride()
    if es != 1 and t.numel():
        _fail(what, "contiguous rows", t)
    return _pack_rows(t.data_ptr(), ts, hs)


def _key_rows(k, what: str, tokens: int, d: int, dtype, device):
    """The same for keys, whose number of heads is free: (shape, packed sh_rows)."""
    if not (isinstance(k, torch.Tensor) and k.dim() == 3):
        _fail(what, "a tensor [tokens, heads, head_dim]", k)
    shape = k.shape
    if shape[0] != tokens or shape[2] != d:
        _fail(what, f"[{tokens}, heads, {d}]", k)
    return shape, _more_rows(k, what, shape, dtype, device)


def _ints(t, what: str, n: int, device: int) -> int:
    """Address of an int32 vector of n entries."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.get_device() == device and t.shape == (n,) and (n <= 1 or t.stride(0) == 1)):
        _fail(what, f"a contiguous int32 vector of {n} entries on cuda:{device}", t)
    return t.data_ptr()


def _sequences(starts) -> int:
    if not (isinstance(starts, torch.Tensor) and starts.dim() == 1 and starts.numel() >= 1):
        _fail("starts", "an int32 vector of sequences + 1 entries", starts)
    return starts.numel() - 1


def _positions(positions, axes: int, tokens: int, device: int):
    """(address, stride between axes) of [tokens] or [axes, tokens] positions."""
    if axes == 1 and isinstance(positions, torch.Tensor) and positions.dim() == 1:
        return _ints(positions, "positions", tokens, device), 0
    if not (isinstance(positions, torch.Tensor) and positions.dtype is torch.int32 and positions.get_device() == device
            and positions.shape == (axes, tokens) and (tokens <= 1 or positions.stride(1) == 1)):
        _fail("positions", f"an int32 tensor [{axes}, {tokens}] on cuda:{device}, contiguous along its last dimension", positions)
    return positions.data_ptr(), positions.stride(0)


def _new(like: torch.Tensor, shape, stream, zero: bool, dtype=None) -> torch.Tensor:
    """A tensor for a call on ``stream``: allocated (and zeroed) in that stream's order."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return like.new_zeros(shape, dtype=dtype) if zero else like.new_empty(shape, dtype=dtype)
    if dtype is None:
        return like.new_zeros(shape) if zero else like.new_empty(shape)
    return like.new_zeros(shape, dtype=dtype) if zero else like.new_empty(shape, dtype=dtype)


def _launch(what: str, fn, device: int, stream, *args) -> None:
    """Call a library entry on the tensors' device and the given (or that device's current) stream."""
    if device == _current_device():
        rc = fn(*args, _raw_stream(device) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _raw_stream(device) if stream is None else stream.cuda_stream)
    if rc:
        raise ShError(rc, f"{what}: strides and addresses must be multiples of 16 bytes, outputs must not overlap themselves, "
                          f"and sizes must lie in the ranges the header states" if rc == SH_EINVAL else what)


class Rope:
    """Norm and rotation of query and key rows (``sh_rope``): what a model keeps for ``qk_norm_rope`` and ``window_decode``.

    ``inv_freq``: fp32 CUDA tensor of rot_dim / 2 frequencies (rot_dim a multiple of 16, at most head_dim; empty: no rotation).
    ``q_weight`` / ``k_weight``: [head_dim] in the rows' type, or None (those rows are not normalised).
    ``sections``: pairs per position axis, one to three of them (default: one axis); ``spread``: the pairs of three axes are
    dealt out in turn instead of in blocks.  ``adjacent``: pairs (2i, 2i+1) instead of (i, i + rot_dim/2)."""

    def __init__(self, inv_freq: torch.Tensor, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, sections=None, spread: bool = False, adjacent: bool = False):
        if not (isinstance(inv_freq, torch.Tensor) and inv_freq.is_cuda and inv_freq.dim() == 1 and inv_freq.dtype == torch.float32
                and (inv_freq.numel() <= 1 or inv_freq.stride(0) == 1)):
            _fail("inv_freq", "a contiguous fp32 CUDA vector", inv_freq)
        pairs = inv_freq.numel()
        sections = (pairs,) if sections is None else tuple(int(x) for x in sections)
        if pairs % 8 or not 1 <= len(sections) <= 3 or min(sections) < 0 or sum(sections) != pairs:
            raise ValueError(f"sections {sections}: need one to three sizes that add up to the {pairs} pairs, a multiple of 8")
        if spread and len(sections) != 3:
            raise ValueError("spread needs three sections")
        for w, what in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if w is not None and not (isinstance(w, torch.Tensor) and w.dim() == 1 and w.device == inv_freq.device and w.dtype in _CODE_OF
                                      and w.numel() in (64, 128) and w.stride(0) == 1 and 2 * pairs <= w.numel()):
                _fail(what, f"a contiguous [head_dim] vector on {inv_freq.device}", w)
        self.inv_freq, self.q_weight, self.k_weight = inv_freq, q_weight, k_weight
        self.eps, self.sections, self.spread, self.adjacent = float(eps), sections, bool(spread), bool(adjacent)
        self.axes = len(sections)
        # what does not change from call to call (addresses are looked up each time: parameters can be moved)
        self._head = (2 * pairs, self.axes, *(sections + (0, 0))[:3], int(self.spread), int(self.adjacent), self.eps)

    def _packed(self, d: int, dtype, device: int) -> bytes:
        f, qw, kw = self.inv_freq, self.q_weight, self.k_weight
        if f.get_device() != device or f.dtype is not torch.float32 or f.shape != (self._head[0] // 2,) or (f.numel() > 1 and f.stride(0) != 1):
            _fail("rope", f"a contiguous vector of {self._head[0] // 2} fp32 frequencies on cuda:{device}", f)
        for w in (qw, kw):
            if w is not None and (w.dtype is not dtype or w.shape != (d,) or w.get_device() != device or w.stride(0) != 1):
                _fail("weight", f"contiguous [{d}] of {dtype} on cuda:{device}", w)
        return _pack_rope(_CODE_OF[dtype], d, *self._head, f.data_ptr(), 0 if qw is None else qw.data_ptr(), 0 if kw is None else kw.data_ptr())


def qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, rope: Rope, q_out: Optional[torch.Tensor] = None,
                 k_out: Optional[torch.Tensor] = None, stream=None):
    """``sh_qk_norm_rope``: rows ``q`` [tokens, q_heads, head_dim] and ``k`` [tokens, k_heads, head_dim] (or None), views of a packed
    projection included, normalised and rotated in one pass.  ``positions``: int32 [tokens], or [axes, tokens].
    Outputs default to new contiguous tensors; ``q_out=q`` works in place.  Returns (q_out, k_out)."""
    shape, dtype, device, qr = _head_rows(q, "q")
    tokens, q_heads, d = shape
    kshape, kr, kor = (0, 0), None, None
    if k is not None:
        kshape, kr = _key_rows(k, "k", tokens, d, dtype, device)
    elif k_out is not None:
        raise ValueError("k_out without k")
    ro = rope._packed(d, dtype, device)
    pos, axis_stride = _positions(positions, rope.axes, tokens, device)
    q_out = _new(q, shape, stream, False) if q_out is None else q_out
    qor = _more_rows(q_out, "q_out", shape, dtype, device)
    if k is not None:
        k_out = _new(k, kshape, stream, False) if k_out is None else k_out
        kor = _more_rows(k_out, "k_out", kshape, dtype, device)
    _launch("qk_norm_rope", lib.sh_qk_norm_rope, device, stream, ro, tokens, q_heads, kshape[1], qr, kr, pos, axis_stride, qor, kor)
    return q_out, k_out


def _window_packed(dtype, d: int, q_heads: int, kv_heads: int, window: int, sinks: int, scale: Optional[float]) -> bytes:
    if window < 1 or sinks < 0 or window + sinks >= 1 << 30:
        raise ValueError(f"window {window}, sinks {sinks}: need window >= 1, sinks >= 0, together below 2^30")
    if kv_heads < 1 or q_heads < 1 or q_heads % kv_heads:
        raise ValueError(f"{q_heads} query heads, {kv_heads} key heads: the first must be a multiple of the second")
    if scale is not None and not (1e-30 < scale < 1e30):
        raise ValueError(f"scale {scale}: need a number between 1e-30 and 1e30")
    return _pack_window(_CODE_OF[dtype], d, q_heads, kv_heads, window, sinks, 0.0 if scale is None else scale)


def _cache_packed(k_cache, v_cache, shape, dtype, device: int) -> bytes:
    if not (isinstance(k_cache, torch.Tensor) and k_cache.dtype is dtype and k_cache.get_device() == device and k_cache.shape == shape):
        _fail("k_cache", f"[sequences, key heads, slots, head_dim] = {tuple(shape)} of {dtype} on cuda:{device}", k_cache)
    if not (isinstance(v_cache, torch.Tensor) and v_cache.dtype is dtype and v_cache.get_device() == device and v_cache.shape == shape):
        _fail("v_cache", f"[sequences, key heads, slots, head_dim] = {tuple(shape)} of {dtype} on cuda:{device}", v_cache)
    ks, vs = k_cache.stride(), v_cache.stride()
    if ks[3] != 1 and k_cache.numel():
        _fail("k_cache", "contiguous rows", k_cache)
    if ks != vs and any(ks[i] != vs[i] for i in range(4) if shape[i] > 1):
        _fail("v_cache", f"the strides of k_cache, {ks}", v_cache)
    return _pack_cache(k_cache.data_ptr(), v_cache.data_ptr(), ks[0], ks[1], ks[2])


def window_prefill(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, *, window: int, sinks: int = 0,
                   lengths: Optional[torch.Tensor] = None, k_cache: Optional[torch.Tensor] = None, v_cache: Optional[torch.Tensor] = None,
                   scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``sh_window_prefill``: attention of prompt chunks with a sliding window and sink tokens.

    ``q`` [tokens, q_heads, head_dim], ``k``/``v`` [tokens, kv_heads, head_dim]; the tokens ``starts[i] .. starts[i+1] - 1`` (int32, on the
    device) continue sequence i, which holds ``lengths[i]`` tokens in ``k_cache``/``v_cache`` [sequences, kv_heads, sinks + window, head_dim]
    (all three None: fresh prompts).  A token sees those before it among the first ``sinks`` positions and the last ``window``, itself
    included.  Rows of ``out`` that belong to no sequence are left as they were (a new ``out`` is zeroed).  ``out`` must not overlap the
    inputs.  16-bit types: the weights are rounded once to the type.  A broken device shows in ``window_status`` alone."""
    shape, dtype, device, qr = _head_rows(q, "q")
    tokens, q_heads, d = shape
    kshape, kr = _key_rows(k, "k", tokens, d, dtype, device)
    vr = _more_rows(v, "v", kshape, dtype, device)
    win = _window_packed(dtype, d, q_heads, kshape[1], window, sinks, scale)
    n = _sequences(starts)
    sp = _ints(starts, "starts", n + 1, device)
    cache, lp = None, None
    if lengths is not None or k_cache is not None or v_cache is not None:
        lp = _ints(lengths, "lengths", n, device)
        cache = _cache_packed(k_cache, v_cache, (n, kshape[1], window + sinks, d), dtype, device)
    out = _new(q, shape, stream, True) if out is None else out
    outr = _more_rows(out, "out", shape, dtype, device)
    wp, bytes_ = None, lib.sh_window_prefill_workspace_bytes(win, tokens, n, cache is not None)
    if bytes_:
        work = _new(q, bytes_, stream, False, torch.uint8)      # as in window_decode
        wp = work.data_ptr()
    _launch("window_prefill", lib.sh_window_prefill, device, stream, win, tokens, n, qr, kr, vr, sp, lp, cache, outr, wp, bytes_)
    return out


def window_append(k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, k_cache: torch.Tensor,
                  v_cache: torch.Tensor, *, window: int, sinks: int = 0, stream=None) -> None:
    """``sh_window_append``: store the chunks' keys and values (arguments as ``window_prefill``; ``lengths`` as before the chunk, the
    caller advances them)."""
    shape, dtype, device, kr = _head_rows(k, "k")
    tokens, kv_heads, d = shape
    vr = _more_rows(v, "v", shape, dtype, device)
    win = _window_packed(dtype, d, kv_heads, kv_heads, window, sinks, None)
    n = _sequences(starts)
    _launch("window_append", lib.sh_window_append, device, stream, win, tokens, n, kr, vr, _ints(starts, "starts", n + 1, device),
            _ints(lengths, "lengths", n, device), _cache_packed(k_cache, v_cache, (n, kv_heads, window + sinks, d), dtype, device))


def window_decode(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lengths: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                  *, window: int, sinks: int = 0, rope: Optional[Rope] = None, positions: Optional[torch.Tensor] = None,
                  scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``sh_window_decode``: one token per sequence, in one launch: its ``q`` and ``k`` are prepared by ``rope`` (if given), its key and
    value stored, and it attends over what it sees, itself included.

    ``q`` [sequences, q_heads, head_dim], ``k``/``v`` [sequences, kv_heads, head_dim], ``lengths`` int32 [sequences]: tokens held before the
    step (the caller advances them); negative: an idle slot of the batch, whose ``out`` row and cache are left as they were (a new ``out``
    is zeroed).  ``positions`` as in ``qk_norm_rope``; default: ``lengths``."""
    shape, dtype, device, qr = _head_rows(q, "q")
    n, q_heads, d = shape
    kshape, kr = _key_rows(k, "k", n, d, dtype, device)
    vr = _more_rows(v, "v", kshape, dtype, device)
    win = _window_packed(dtype, d, q_heads, kshape[1], window, sinks, scale)
    lp = _ints(lengths, "lengths", n, device)
    cache = _cache_packed(k_cache, v_cache, (n, kshape[1], window + sinks, d), dtype, device)
    ro, pos, axis_stride = None, None, 0
    if rope is not None:
        ro = rope._packed(d, dtype, device)
        if positions is not None:
            pos, axis_stride = _positions(positions, rope.axes, n, device)
        elif rope.axes != 1:
            raise ValueError("a rope of several axes needs positions")
    elif positions is not None:
        raise ValueError("positions without rope")
    out = _new(q, shape, stream, True) if out is None else out
    outr = _more_rows(out, "out", shape, dtype, device)
    wp, bytes_ = None, lib.sh_window_decode_workspace_bytes(win, n)
    if bytes_:
        work = _new(q, bytes_, stream, False, torch.uint8)      # a tensor of this call's own: it is free again in the stream's order
        wp = work.data_ptr()
    _launch("window_decode", lib.sh_window_decode, device, stream, win, n, qr, kr, vr, lp, cache, ro, pos, axis_stride, outr, wp, bytes_)
    return out


def window_status(device="cuda:0", stream=None) -> None:
    """``sh_window_status``: raise ShError(SH_EDEVICE) if a window kernel on ``device`` gave up one of its bounded waits since the last
    call (its outputs are then incomplete, though ``window_prefill`` and ``WindowCache.prefill`` returned as usual: they do not
    synchronise, and ask for nothing).  Synchronises the stream."""
    index = torch.device(device).index
    _launch("window_status", lib.sh_window_status, _current_device() if index is None else index, stream)


class WindowCache:
    """Key/value cache of a batch under the fixed policy "first ``sinks`` tokens and last ``window`` ones": the sibling of ``Handle``
    for attention with a sliding window.  Owns ``k``, ``v`` [sequences, kv_heads, sinks + window, head_dim] and ``lengths`` (int32, on the
    device; -1 marks an idle slot of the batch).  ``rope``: prepares the queries and keys of every call (positions default to the
    tokens' places in their sequences)."""

    def __init__(self, sequences: int, q_heads: int, kv_heads: int, head_dim: int, window: int, sinks: int = 0, dtype="bf16", device="cuda:0",
                 rope: Optional[Rope] = None, scale: Optional[float] = None):
        dt = INPUT_TORCH_DTYPE[DTYPE_CODE[dtype]] if isinstance(dtype, str) else dtype
        if dt not in _CODE_OF or dtype == "int4" or head_dim not in (64, 128) or sequences < 1:
            raise ValueError(f"{sequences} sequences of dtype {dtype}, head_dim {head_dim}: need one or more, f32, f16 or bf16, 64 or 128")
        _window_packed(dt, head_dim, q_heads, kv_heads, window, sinks, scale)
        self.window, self.sinks, self.rope, self.scale, self.q_heads = window, sinks, rope, scale, q_heads
        shape = (sequences, kv_heads, sinks + window, head_dim)
        self.k = torch.zeros(shape, dtype=dt, device=device)
        self.v = torch.zeros(shape, dtype=dt, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)

    def _check_heads(self, q: torch.Tensor) -> None:
        if q.dim() != 3 or q.shape[1] != self.q_heads:
            _fail("q", f"[tokens, {self.q_heads}, {self.k.shape[3]}]", q)

    def _prompt_positions(self, starts: torch.Tensor, tokens: int) -> torch.Tensor:
        """Position of each row of a chunk tensor: its sequence's length plus its place in the chunk."""
        row = torch.arange(tokens, dtype=torch.int32, device=self.k.device)
        seq = (torch.searchsorted(starts, row, right=True) - 1).clamp(0, starts.numel() - 2)
        return (self.lengths[seq] + row - starts[seq]).clamp(min=0)

    def prefill(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, positions: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Chunks of prompts (``window_prefill``), stored and counted.  On the current stream."""
        self._check_heads(q)
        if self.rope is not None:
            if positions is None:
                if self.rope.axes != 1:
                    raise ValueError("a rope of several axes needs positions")
                positions = self._prompt_positions(starts, q.shape[0])
            q, k = qk_norm_rope(q, k, positions, self.rope)
        win = dict(window=self.window, sinks=self.sinks)
        out = window_prefill(q, k, v, starts, lengths=self.lengths, k_cache=self.k, v_cache=self.v, scale=self.scale, out=out, **win)
        window_append(k, v, starts, self.lengths, self.k, self.v, **win)
        self.lengths += torch.where(self.lengths < 0, 0, starts[1:] - starts[:-1])
        return out

    def decode(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One token per sequence (``window_decode``), stored and counted.  On the current stream."""
        self._check_heads(q)
        out = window_decode(q, k, v, self.lengths, self.k, self.v, window=self.window, sinks=self.sinks, rope=self.rope, positions=positions,
                            scale=self.scale, out=out)
        self.lengths += (self.lengths >= 0).to(torch.int32)
        return out


# -- shared contexts and the cache with accumulated weights ------------------------------------------------------------
_pack_attention, _pack_records = struct.Struct("iiiiid").pack, struct.Struct("PPqq").pack


def _attention_packed(dtype, d: int, q_heads: int, kv_heads: int, slots: int, scale: Optional[float]) -> bytes:
    if kv_heads < 1 or q_heads < 1 or q_heads % kv_heads:
        raise ValueError(f"{q_heads} query heads, {kv_heads} key heads: the first must be a multiple of the second")
    if not 1 <= slots < 1 << 30:
        raise ValueError(f"{slots} rows: need 1 .. 2^30 - 1")
    if scale is not None and not (1e-30 < scale < 1e30):
        raise ValueError(f"scale {scale}: need a number between 1e-30 and 1e30")
    return _pack_attention(_CODE_OF[dtype], d, q_heads, kv_heads, slots, 0.0 if scale is None else scale)


def _slots_of(k_cache, what: str, n: Optional[int], kv_heads: Optional[int], d: Optional[int], dtype, device: int):
    """Shape of a cache [sequences, key heads, slots, head_dim] whose other sizes are given (None: free)."""
    if isinstance(k_cache, torch.Tensor) and k_cache.dim() == 4:
        s = k_cache.shape
        if (n is None or s[0] == n) and (kv_heads is None or s[1] == kv_heads) and (s[3] == d if d is not None else s[3] in (64, 128)):
            return s
    _fail(what, f"[{n or 'sequences'}, {kv_heads or 'key heads'}, slots, {d or '64 or 128'}] of {dtype} on cuda:{device}", k_cache)


def _records_packed(mass, positions, shape, device: int) -> bytes:
    if not (isinstance(mass, torch.Tensor) and mass.dtype is torch.float32 and mass.get_device() == device and mass.shape == shape):
        _fail("mass", f"[sequences, key heads, slots] = {tuple(shape)} of fp32 on cuda:{device}", mass)
    if not (isinstance(positions, torch.Tensor) and positions.dtype is torch.int32 and positions.get_device() == device and positions.shape == shape):
        _fail("positions", f"[sequences, key heads, slots] = {tuple(shape)} of int32 on cuda:{device}", positions)
    ms, ps = mass.stride(), positions.stride()
    if ms[2] != 1 and shape[2] > 1:
        _fail("mass", "contiguous slots", mass)
    if ms != ps and any(ms[i] != ps[i] for i in range(3) if shape[i] > 1):
        _fail("positions", f"the strides of mass, {ms}", positions)
    return _pack_records(mass.data_ptr(), positions.data_ptr(), ms[0], ms[1])


def _prior_packed(prior, shape, dtype, device: int):
    if prior is None:
        return None, 0, None
    if not (isinstance(prior, (tuple, list)) and len(prior) == 2 and isinstance(prior[0], torch.Tensor)):
        _fail("prior", "a pair (out, lse)", prior)
    dt = torch.float32 if prior[0].dtype is torch.float32 else dtype
    return _more_rows(prior[0], "prior", shape, dt, device), _CODE_OF[dt], _logs(prior[1], "prior's lse", shape, device)


def _logs(t, what: str, shape, device: int) -> int:
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.get_device() == device and t.shape == shape[:2] and t.is_contiguous()):
        _fail(what, f"a contiguous fp32 tensor {tuple(shape[:2])} on cuda:{device}", t)
    return t.data_ptr()


def context_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: Optional[torch.Tensor] = None,
                      lengths: Optional[torch.Tensor] = None, *, scale: Optional[float] = None, partial: bool = False,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``sh_context_attention``: attention to contexts that are complete: a prefix that a whole batch shares, or each sequence's encoder states
    (cross attention).

    ``q`` [tokens, q_heads, head_dim], ``k``/``v`` [contexts, kv_heads, rows, head_dim].  The tokens ``starts[i] .. starts[i+1] - 1`` (int32, on the
    device) see the first ``lengths[i]`` rows of context i (None: all), all of them.  ``starts`` None: one context that all tokens share, or
    one for each token.  Returns ``out`` and ``lse`` fp32 [tokens, q_heads], the logs of the rows' sums of exponentials, from which
    ``mass_decode`` and ``mass_prefill`` continue (``prior``); with ``partial`` ``out`` is fp32, so that nothing is rounded on the way.  A context of length 0 gives zeros and -inf; rows that belong to no
    context are left as they were (new tensors: zeros and -inf)."""
    shape, dtype, device, qr = _head_rows(q, "q")
    tokens, q_heads, d = shape
    kshape = _slots_of(k, "k", None, None, d, dtype, device)
    n, kv_heads, rows = kshape[0], kshape[1], kshape[2]
    at = _attention_packed(dtype, d, q_heads, kv_heads, rows, scale)
    cache = _cache_packed(k, v, kshape, dtype, device)
    sp = None
    if starts is not None:
        sp = _ints(starts, "starts", n + 1, device)
    elif n != 1 and n != tokens:
        raise ValueError(f"{n} contexts for {tokens} tokens: without starts there must be one, or one for each token")
    lp = None if lengths is None else _ints(lengths, "lengths", n, device)
    odt = torch.float32 if partial else dtype
    if (out is None) != (lse is None):
        raise ValueError("out and lse: give both or neither")
    fresh = out is None
    if fresh:
        out = torch.empty_like(q, memory_format=torch.contiguous_format) if stream is None and odt is dtype else _new(q, shape, stream, False, odt)
        lse = _new(q, shape[:2], stream, False, torch.float32)
    outr = _more_rows(out, "out", shape, odt, device)
    wp, bytes_ = None, lib.sh_context_attention_workspace_bytes(at, tokens, n, sp is not None)
    if bytes_:
        work = _new(q, bytes_, stream, False, torch.uint8)
        wp = work.data_ptr()
    _launch("context_attention", lib.sh_context_attention, device, stream, at, tokens, n, qr, cache, sp, lp, outr, _CODE_OF[odt], _logs(lse, "lse", shape, device), int(fresh), wp, bytes_)
    return out, lse


def mass_prefill(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, k_cache: torch.Tensor,
                 v_cache: torch.Tensor, mass: torch.Tensor, positions: torch.Tensor, seen: torch.Tensor, *, prior=None,
                 scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``sh_mass_prefill``: prompt chunks over a cache with accumulated weights.

    ``q`` [tokens, q_heads, head_dim], ``k``/``v`` [tokens, kv_heads, head_dim]; the tokens ``starts[i] .. starts[i+1] - 1`` are stored in the slots of
    ``k_cache``/``v_cache`` [sequences, kv_heads, slots, head_dim] from ``lengths[i]`` on, with positions from ``seen[i]`` on (the caller advances both);
    each sees the live slots and the chunk up to itself, and ``mass`` fp32 [sequences, kv_heads, slots] grows by the weights that the rows get.
    ``prior``: (out, lse) of ``context_attention(..., partial=True)`` for the same tokens; the softmax goes over both.  A sequence of negative length, or
    whose chunk has no room, takes no part; its rows of ``out``, and those of no sequence, are left as they were (a new ``out`` is
    zeroed)."""
    shape, dtype, device, qr = _head_rows(q, "q")
    tokens, q_heads, d = shape
    kshape, kr = _key_rows(k, "k", tokens, d, dtype, device)
    vr = _more_rows(v, "v", kshape, dtype, device)
    n = _sequences(starts)
    cshape = _slots_of(k_cache, "k_cache", n, kshape[1], d, dtype, device)
    at = _attention_packed(dtype, d, q_heads, kshape[1], cshape[2], scale)
    cache, rec = _cache_packed(k_cache, v_cache, cshape, dtype, device), _records_packed(mass, positions, cshape[:3], device)
    pr, pt, pl = _prior_packed(prior, shape, dtype, device)
    out = _new(q, shape, stream, True) if out is None else out
    outr = _more_rows(out, "out", shape, dtype, device)
    bytes_ = lib.sh_mass_prefill_workspace_bytes(at, tokens, n)
    work = _new(q, bytes_, stream, False, torch.uint8)
    _launch("mass_prefill", lib.sh_mass_prefill, device, stream, at, tokens, n, qr, kr, vr, _ints(starts, "starts", n + 1, device),
            _ints(lengths, "lengths", n, device), _ints(seen, "seen", n, device), cache, rec, pr, pt, pl, outr, work.data_ptr(), bytes_)
    return out


def mass_decode(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lengths: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                mass: torch.Tensor, positions: torch.Tensor, seen: torch.Tensor, *, prior=None, scale: Optional[float] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``sh_mass_decode``: one token per sequence over a cache with accumulated weights (arguments as ``mass_prefill``, ``q`` [sequences, q_heads,
    head_dim]): stored in slot ``lengths[i]``, attends over the live slots and itself, and the masses grow by its weights.  A sequence of
    negative length, or whose cache is full, takes no part."""
    shape, dtype, device, qr = _head_rows(q, "q")
    n, q_heads, d = shape
    kshape, kr = _key_rows(k, "k", n, d, dtype, device)
    vr = _more_rows(v, "v", kshape, dtype, device)
    cshape = _slots_of(k_cache, "k_cache", n, kshape[1], d, dtype, device)
    at = _attention_packed(dtype, d, q_heads, kshape[1], cshape[2], scale)
    cache, rec = _cache_packed(k_cache, v_cache, cshape, dtype, device), _records_packed(mass, positions, cshape[:3], device)
    pr, pt, pl = _prior_packed(prior, shape, dtype, device)
    out = _new(q, shape, stream, True) if out is None else out
    outr = _more_rows(out, "out", shape, dtype, device)
    bytes_ = lib.sh_mass_decode_workspace_bytes(at, n)
    work = _new(q, bytes_, stream, False, torch.uint8)
    _launch("mass_decode", lib.sh_mass_decode, device, stream, at, n, qr, kr, vr, _ints(lengths, "lengths", n, device),
            _ints(seen, "seen", n, device), cache, rec, pr, pt, pl, outr, work.data_ptr(), bytes_)
    return out


def mass_evict(k_cache: torch.Tensor, v_cache: torch.Tensor, mass: torch.Tensor, positions: torch.Tensor, lengths: torch.Tensor, *, keep: int,
               recent: int = 0, into=None, left: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """``sh_mass_evict``: every (sequence, key head) with more than ``keep`` live rows keeps that many: the ``recent`` newest positions, then the
    largest masses, among equal ones the lowest slots.

    In place, or ``into`` = (k_cache, v_cache, mass, positions) of a cache with at least ``keep`` slots, which must not overlap the first.  Returns
    the new lengths, ``min(lengths, keep)`` (``left``: where to put them; may be ``lengths``)."""
    if not (isinstance(k_cache, torch.Tensor) and k_cache.dtype in _CODE_OF and k_cache.is_cuda):
        _fail("k_cache", "a CUDA tensor [sequences, key heads, slots, 64 or 128] of f32, f16 or bf16", k_cache)
    dtype, device = k_cache.dtype, k_cache.get_device()
    shape = _slots_of(k_cache, "k_cache", None, None, None, dtype, device)
    n, heads, slots, d = shape
    room = slots
    cache, rec, to, to_rec = _cache_packed(k_cache, v_cache, shape, dtype, device), _records_packed(mass, positions, shape[:3], device), None, None
    if into is not None:
        if not (isinstance(into, (tuple, list)) and len(into) == 4):
            _fail("into", "(k_cache, v_cache, mass, positions)", into)
        tshape = _slots_of(into[0], "into", n, heads, d, dtype, device)
        room = tshape[2]
        to, to_rec = _cache_packed(into[0], into[1], tshape, dtype, device), _records_packed(into[2], into[3], tshape[:3], device)
    if not (1 <= keep <= room and 0 <= recent <= keep):
        raise ValueError(f"keep {keep}, recent {recent}: need 1 <= keep <= {room} slots and 0 <= recent <= keep")
    at = _attention_packed(dtype, d, heads, heads, slots, None)
    lp = _ints(lengths, "lengths", n, device)
    left = _new(lengths, lengths.shape, stream, False) if left is None else left
    bytes_ = lib.sh_mass_evict_workspace_bytes(at, n, keep, into is None)
    work = _new(k_cache, bytes_, stream, False, torch.uint8)
    _launch("mass_evict", lib.sh_mass_evict, device, stream, at, n, lp, cache, rec, keep, recent, to, to_rec, room, _ints(left, "left", n, device),
            work.data_ptr(), bytes_)
    return left


class MassCache:
    """Key/value cache of a batch under the policy "the ``recent`` newest tokens and those that have received most attention", at most ``budget``
    rows per (sequence, key head) after an eviction and ``spare`` more in between: the sibling of ``Handle`` and ``WindowCache`` that goes by
    accumulated attention weights.

    Owns ``k``, ``v`` [sequences, kv_heads, budget + spare, head_dim], ``mass``, ``positions`` [sequences, kv_heads, budget + spare], ``lengths`` (rows
    held; -1 marks an idle slot of the batch) and ``seen`` (tokens so far: the position of the next one), int32 on the device.  To begin a
    new sequence in slot i set ``lengths[i] = 0`` and ``seen[i]`` to ``first``.

    ``rope`` prepares the queries and keys of every call (positions default to the tokens' places).  ``prefix`` = (k, v) [1, kv_heads, rows,
    head_dim]: keys (prepared) and values that every sequence begins with; it is kept once, attended to for the whole batch at once, never
    evicted, and ``first`` is the number of its rows (else 0).

    How full the sequences are is not known on the host: it counts the tokens that have come since the last eviction, one per ``decode`` and
    ``longest`` per ``prefill``, and evicts when there may be no room.  (In a captured graph, and after its tensors have been given other
    contents, call ``evict`` where it belongs.)"""

    def __init__(self, sequences: int, q_heads: int, kv_heads: int, head_dim: int, budget: int, recent: int, spare: int = 64, dtype="bf16",
                 device="cuda:0", rope: Optional[Rope] = None, scale: Optional[float] = None, prefix=None):
        dt = INPUT_TORCH_DTYPE[DTYPE_CODE[dtype]] if isinstance(dtype, str) else dtype
        if dt not in _CODE_OF or dtype == "int4" or head_dim not in (64, 128) or sequences < 1:
            raise ValueError(f"{sequences} sequences of dtype {dtype}, head_dim {head_dim}: need one or more, f32, f16 or bf16, 64 or 128")
        if not (1 <= budget and 0 <= recent <= budget and 1 <= spare):
            raise ValueError(f"budget {budget}, recent {recent}, spare {spare}: need 1 <= budget, 0 <= recent <= budget, 1 <= spare")
        _attention_packed(dt, head_dim, q_heads, kv_heads, budget + spare, scale)
        self.q_heads, self.budget, self.recent, self.spare, self.rope, self.scale, self.prefix = q_heads, budget, recent, spare, rope, scale, prefix
        self.k, self.v, self.mass, self.positions = self._rows(sequences, kv_heads, budget + spare, head_dim, dt, device)
        self.first = 0
        if prefix is not None:
            if not (isinstance(prefix, (tuple, list)) and len(prefix) == 2):
                _fail("prefix", "a pair (k, v)", prefix)
            s = _slots_of(prefix[0], "prefix", 1, kv_heads, head_dim, dt, self.k.get_device())
            _cache_packed(*prefix, s, dt, self.k.get_device())
            self.first = s[2]
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.seen = torch.full((sequences,), self.first, dtype=torch.int32, device=device)
        self._room = budget + spare

    @staticmethod
    def _rows(sequences, kv_heads, slots, head_dim, dt, device, new=torch.zeros):
        shape = (sequences, kv_heads, slots)
        return (new((*shape, head_dim), dtype=dt, device=device), new((*shape, head_dim), dtype=dt, device=device),
                new(shape, dtype=torch.float32, device=device), new(shape, dtype=torch.int32, device=device))

    @staticmethod
    def _stored(starts, tokens: int, lengths, slots: int) -> torch.Tensor:
        """Rows of each sequence that ``mass_prefill`` stores in caches of that many slots: none where it is idle or has no room."""
        at = starts.clamp(0, tokens)
        count = (at[1:] - at[:-1]).clamp(min=0)
        return torch.where((lengths >= 0) & (count <= slots - lengths), count, 0)

    def _prepare(self, q, k, positions, default):
        if q.dim() != 3 or q.shape[1] != self.q_heads:
            _fail("q", f"[tokens, {self.q_heads}, {self.k.shape[3]}]", q)
        if self.rope is not None:
            if positions is None:
                if self.rope.axes != 1:
                    raise ValueError("a rope of several axes needs positions")
                positions = default()
            q, k = qk_norm_rope(q, k, positions, self.rope)
        elif positions is not None:
            raise ValueError("positions without rope")
        prior = None if self.prefix is None else context_attention(q, *self.prefix, scale=self.scale, partial=True)
        return q, k, prior

    def prefill(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, starts: torch.Tensor, positions: Optional[torch.Tensor] = None,
                longest: Optional[int] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Chunks of prompts (``mass_prefill``), stored and counted.  ``longest``: the most tokens that a sequence has here, or more.  Default: what
        ``starts`` says, for which the call waits for the stream (one sequence, and under capture: all tokens).  A chunk that the spare
        slots do not hold is read in full in a cache of its own size and then evicted into this one.
        (If a sequence has more than ``longest`` tokens and there is no room for them, it takes no part: its ``lengths`` and ``seen`` stay.)"""
        tokens, n = q.shape[0], self.k.shape[0]
        if longest is not None and not 0 <= int(longest) <= tokens:
            raise ValueError(f"longest {longest}: need 0 .. {tokens}")
        if tokens > 0:
            _ints(starts, "starts", n + 1, self.k.get_device())
        if longest is None:
            bound = tokens == 0 or n == 1 or (starts.is_cuda and torch.cuda.is_current_stream_capturing())
            longest = tokens if bound else self._stored(starts, tokens, self.lengths, 1 << 30).max()
        longest = int(longest)
        if longest == 0:
            return _new(q, q.shape, None, True) if out is None else out

        def places():
            row = torch.arange(tokens, dtype=torch.int32, device=self.k.device)
            seq = (torch.searchsorted(starts, row, right=True) - 1).clamp(0, starts.numel() - 2)
            return self.seen[seq] + (row - starts[seq]).clamp(min=0)

        q, k, prior = self._prepare(q, k, positions, places)
        if longest > self._room and longest <= self.spare:
            self.evict()
        if longest <= self._room:
            count = self._stored(starts, tokens, self.lengths, self.k.shape[2])
            out = mass_prefill(q, k, v, starts, self.lengths, self.k, self.v, self.mass, self.positions, self.seen, prior=prior, scale=self.scale, out=out)
            self.lengths += count
            self._room -= longest
        else:
            hk, d = self.k.shape[1], self.k.shape[3]
            # (every row of it that anybody looks at is written by the eviction into it or stored with the chunk)
            whole = self._rows(n, hk, self.budget + longest, d, self.k.dtype, self.k.device, new=torch.empty)
            held = mass_evict(self.k, self.v, self.mass, self.positions, self.lengths, keep=self.budget, recent=self.recent, into=whole)
            count = self._stored(starts, tokens, held, self.budget + longest)
            out = mass_prefill(q, k, v, starts, held, *whole, self.seen, prior=prior, scale=self.scale, out=out)
            mass_evict(*whole, held + count, keep=self.budget, recent=self.recent, into=(self.k, self.v, self.mass, self.positions), left=self.lengths)
            self._room = self.spare
        self.seen += count
        return out

    def decode(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One token per sequence (``mass_decode``), stored and counted; before it the eviction, if some sequence may be full.  (One that is full
        all the same, after replays of a captured step, takes no part: its ``lengths`` and ``seen`` stay.)  On the current stream."""
        q, k, prior = self._prepare(q, k, positions, lambda: self.seen)
        if self._room == 0:
            self.evict()
        out = mass_decode(q, k, v, self.lengths, self.k, self.v, self.mass, self.positions, self.seen, prior=prior, scale=self.scale, out=out)
        active = self.lengths == self.lengths.clamp(0, self.k.shape[2] - 1)      # (neither idle nor full, as the kernel has it)
        self.lengths += active
        self.seen += active
        self._room -= 1
        return out

    def evict(self) -> None:
        """Bring every sequence down to ``budget`` rows (``mass_evict``, in place).  On the current stream."""
        mass_evict(self.k, self.v, self.mass, self.positions, self.lengths, keep=self.budget, recent=self.recent, left=self.lengths)
        self._room = self.spare
