"""Python binding of libpdec.so (include/pdec.h): argument marshalling only.

Device memory and streams come from PyTorch (ROCm); every step of encoding
and decoding runs in the library's HIP kernels.  There is no fallback: if the
library is missing or fails, calls raise.
"""
from __future__ import annotations

import ctypes
import os
from typing import NamedTuple, Optional, Sequence

import numpy as np

from . import configs as C

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpdec.so")

PD_AR, PD_JACOBI, PD_GS_JACOBI, PD_HYBRID = 0, 1, 2, 3
MODE_IDS = {"ar": PD_AR, "jacobi": PD_JACOBI, "gs_jacobi": PD_GS_JACOBI, "hybrid": PD_HYBRID}
PD_STOP_PREFIX = 0x100                  # or-ed into the mode: the prefix stopping condition
STOP_FLAGS = {"block": 0, "prefix": PD_STOP_PREFIX}


def mode_word(mode, stop="block") -> int:
    """The mode argument of pd_decode: the mode id, or-ed with the stopping-condition flag."""
    return (MODE_IDS[mode] if isinstance(mode, str) else int(mode)) | STOP_FLAGS[stop]
FLAG_CONVERGED, FLAG_EOS, FLAG_MAX_ITERS, FLAG_NONFINITE = 1, 2, 4, 8
STATUS = {0: "PD_OK", 1: "PD_E_ARG", 2: "PD_E_SHAPE", 3: "PD_E_WORKSPACE", 4: "PD_E_DEVICE",
          5: "PD_E_UNSUPPORTED", 6: "PD_E_STATE"}


class PdError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class pd_config(ctypes.Structure):
    _fields_ = [("n_enc", ctypes.c_int32), ("n_dec", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("pre_ln", ctypes.c_int32), ("act_gelu", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("pad_id", ctypes.c_int32), ("bos_id", ctypes.c_int32), ("eos_id", ctypes.c_int32),
                ("ln_eps", ctypes.c_float), ("logit_scale", ctypes.c_float),
                ("enc_emb_scale", ctypes.c_float), ("dec_emb_scale", ctypes.c_float)]


EXPORTS = ("pd_weight_count", "pd_weight_shape", "pd_model_create", "pd_model_destroy",
           "pd_ctx_workspace_bytes", "pd_ctx_create", "pd_ctx_destroy", "pd_encode", "pd_decode", "pd_decode_init",
           "pd_debug_logits", "pd_ctx_set_timing", "pd_ctx_vocab_timing", "pd_ctx_rows_processed",
           "pd_trace_scratch_bytes", "pd_ctx_set_trace", "pd_ctx_trace_count", "pd_ctx_product_timing",
           "pd_ctx_iteration_kernels", "pd_decode_traced_static", "pd_beam_select_bytes", "pd_beam_select",
           "pd_cache_bytes", "pd_cache_attend_bytes", "pd_cache_attend", "pd_cache_read", "pd_pages_bytes",
           "pd_pages_fork", "pd_pages_compact", "pd_decode_beam_bytes", "pd_decode_beam", "pd_last_error")
TRACE_STATIC_BYTES = 8 << 20      # PD_TRACE_STATIC_BYTES

CACHE_TYPES = {"f32": 0, "bf16": 1, "int4": 2}      # PD_F32, PD_BF16, PD_INT4


class pd_cache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("layers", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libpdec.so and declare its signatures (raises if it is not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise OSError(f"{path} is not built: run `python -m paper_2305_10427_amd.build`")
    L = ctypes.CDLL(path)
    P, I32, I64, SZ, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p
    L.pd_weight_count.argtypes = [P(pd_config)]
    L.pd_weight_count.restype = I32
    L.pd_weight_shape.argtypes = [P(pd_config), I32, P(I64), P(I64)]
    L.pd_weight_shape.restype = I32
    L.pd_model_create.argtypes = [P(pd_config), P(VP), I32, P(VP)]
    L.pd_model_create.restype = I32
    L.pd_model_destroy.argtypes = [VP]
    L.pd_model_destroy.restype = None
    L.pd_ctx_workspace_bytes.argtypes = [VP, I32, I32, I32, P(SZ)]
    L.pd_ctx_workspace_bytes.restype = I32
    L.pd_ctx_create.argtypes = [VP, I32, I32, I32, VP, SZ, P(VP)]
    L.pd_ctx_create.restype = I32
    L.pd_ctx_destroy.argtypes = [VP]
    L.pd_ctx_destroy.restype = None
    L.pd_encode.argtypes = [VP, VP, P(I32), I32, I32, VP]
    L.pd_encode.restype = I32
    L.pd_decode.argtypes = [VP, I32, I32, I32, I32, P(I32), VP, I32, VP, VP, VP, VP]
    L.pd_decode.restype = I32
    L.pd_decode_init.argtypes = [VP, I32, I32, I32, I32, P(I32), VP, I32, VP, I32, VP, VP, VP, VP]
    L.pd_decode_init.restype = I32
    L.pd_debug_logits.argtypes = [VP, VP, I32, VP, VP]
    L.pd_debug_logits.restype = I32
    L.pd_ctx_set_timing.argtypes = [VP, I32]
    L.pd_ctx_set_timing.restype = I32
    L.pd_ctx_vocab_timing.argtypes = [VP, P(I64), P(ctypes.c_double)]
    L.pd_ctx_vocab_timing.restype = I32
    L.pd_ctx_rows_processed.argtypes = [VP, P(I64)]
    L.pd_ctx_rows_processed.restype = I32
    L.pd_trace_scratch_bytes.argtypes = [VP, I32, P(SZ)]
    L.pd_trace_scratch_bytes.restype = I32
    L.pd_ctx_set_trace.argtypes = [VP, VP, I64, VP, SZ]
    L.pd_ctx_set_trace.restype = I32
    L.pd_ctx_trace_count.argtypes = [VP, P(I64)]
    L.pd_ctx_trace_count.restype = I32
    L.pd_ctx_product_timing.argtypes = [VP, P(I64), P(ctypes.c_double), P(ctypes.c_double)]
    L.pd_ctx_product_timing.restype = I32
    L.pd_ctx_iteration_kernels.argtypes = [VP, P(I64)]
    L.pd_ctx_iteration_kernels.restype = I32
    L.pd_decode_traced_static.argtypes = [VP, I32, I32, I32, I32, P(I32), VP, I32, VP, VP, VP, VP, I64, VP]
    L.pd_decode_traced_static.restype = I32
    F32, PC = ctypes.c_float, P(pd_cache)
    L.pd_beam_select_bytes.argtypes = [I32, I32, I32, I32, P(SZ)]
    L.pd_beam_select_bytes.restype = I32
    L.pd_beam_select.argtypes = [VP, I32, I64, I32, I32, I32, VP, VP, VP, VP, I32, I32, F32, VP, VP, VP, VP, VP, VP,
                                 VP, VP, SZ, VP]
    L.pd_beam_select.restype = I32
    L.pd_cache_bytes.argtypes = [PC, P(SZ), P(SZ)]
    L.pd_cache_bytes.restype = I32
    L.pd_cache_attend_bytes.argtypes = [PC, I32, I32, I32, I32, P(SZ)]
    L.pd_cache_attend_bytes.restype = I32
    L.pd_cache_attend.argtypes = [PC, I32, VP, I32, I64, I32, VP, VP, I32, I64, VP, I32, VP, I32, I32, I32, F32, VP,
                                  I32, I64, VP, SZ, VP]
    L.pd_cache_attend.restype = I32
    L.pd_cache_read.argtypes = [PC, I32, VP, I32, VP, I32, VP, I32, VP, VP, VP]
    L.pd_cache_read.restype = I32
    L.pd_pages_bytes.argtypes = [PC, I32, P(SZ)]
    L.pd_pages_bytes.restype = I32
    L.pd_pages_fork.argtypes = [PC, VP, I32, VP, I32, VP, I32, I32, VP, VP, VP, VP, VP, SZ, VP]
    L.pd_pages_fork.restype = I32
    L.pd_pages_compact.argtypes = [PC, VP, I32, VP, I32, VP, VP, VP, VP, SZ, VP]
    L.pd_pages_compact.restype = I32
    L.pd_decode_beam_bytes.argtypes = [VP, I32, I32, P(SZ)]
    L.pd_decode_beam_bytes.restype = I32
    L.pd_decode_beam.argtypes = [VP, I32, F32, I32, P(I32), VP, I32, VP, VP, VP, VP, VP, SZ, VP]
    L.pd_decode_beam.restype = I32
    L.pd_last_error.argtypes = []
    L.pd_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


def _check(status: int):
    if status != 0:
        raise PdError(status, load_library().pd_last_error().decode())


def make_config(cfg: C.ModelConfig) -> pd_config:
    return pd_config(cfg.n_enc, cfg.n_dec, cfg.d_model, cfg.n_heads, cfg.d_ff, cfg.vocab,
                     int(cfg.pre_ln), int(cfg.act_gelu), 1 if cfg.dtype == C.BF16 else 0,
                     C.PAD_ID, C.BOS_ID, C.EOS_ID, cfg.ln_eps, cfg.logit_scale, -1.0,
                     -1.0 if cfg.dec_emb_scale is None else float(cfg.dec_emb_scale))


def _stream_handle(stream) -> int:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return int(s.cuda_stream)


def _host_i32(a) -> ctypes.Array:
    a = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    return (ctypes.c_int32 * len(a))(*a.tolist())


class Model:
    """Weights uploaded to the GPU plus the library's pd_model handle."""

    def __init__(self, cfg: C.ModelConfig, weights, device: str = "cuda"):
        import torch
        L = load_library()
        self.cfg = cfg
        self.c_cfg = make_config(cfg)
        n = L.pd_weight_count(ctypes.byref(self.c_cfg))
        names = [nm for nm, _ in C.param_shapes(cfg)]
        if n != len(names):
            raise PdError(1, f"library expects {n} weights, configuration has {len(names)}")
        self.tensors = []
        for i, nm in enumerate(names):
            rows, cols = ctypes.c_int64(), ctypes.c_int64()
            _check(L.pd_weight_shape(ctypes.byref(self.c_cfg), i, ctypes.byref(rows), ctypes.byref(cols)))
            want = (rows.value, cols.value) if cols.value > 1 else (rows.value,)
            if tuple(weights.values[nm].shape) != want:
                raise PdError(2, f"weight {nm}: shape {weights.values[nm].shape} != {want}")
            if cfg.dtype == C.BF16:
                host = torch.from_numpy(weights.bf16_bits[nm].view(np.int16).copy()).view(torch.bfloat16)
            else:
                host = torch.from_numpy(np.ascontiguousarray(weights.values[nm], np.float32))
            self.tensors.append(host.to(device).contiguous())
        ptrs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in self.tensors])
        h = ctypes.c_void_p()
        _check(L.pd_model_create(ctypes.byref(self.c_cfg), ptrs, n, ctypes.byref(h)))
        self.handle = h

    def weight_bytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self.tensors)

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.pd_model_destroy(self.handle)
            self.handle = None


class Context:
    """A decoding context: caller-owned workspace + the library's pd_ctx."""

    def __init__(self, model: Model, max_batch: int, max_src: int, max_tgt: int, device: str = "cuda"):
        import torch
        L = load_library()
        self.model = model
        self.max_batch, self.max_src, self.max_tgt = max_batch, max_src, max_tgt
        nbytes = ctypes.c_size_t()
        _check(L.pd_ctx_workspace_bytes(model.handle, max_batch, max_src, max_tgt, ctypes.byref(nbytes)))
        self.workspace = torch.empty(nbytes.value + 256, dtype=torch.uint8, device=device)
        base = self.workspace.data_ptr()
        self.ws_ptr = (base + 255) // 256 * 256
        h = ctypes.c_void_p()
        _check(L.pd_ctx_create(model.handle, max_batch, max_src, max_tgt, ctypes.c_void_p(self.ws_ptr),
                               nbytes.value, ctypes.byref(h)))
        self.handle = h
        self.B = 0
        self.device = device
        self._beam_ws = None

    def encode(self, src, src_len: Sequence[int], stream=None):
        """src: int32 device tensor [B, n_max]; src_len: host ints."""
        import torch
        src = src.to(device=self.device, dtype=torch.int32).contiguous()
        B, n_max = src.shape
        self._src = src                      # keep alive until the kernels have read it
        _check(load_library().pd_encode(self.handle, ctypes.c_void_p(src.data_ptr()), _host_i32(src_len),
                                        B, n_max, ctypes.c_void_p(_stream_handle(stream))))
        self.B = B

    def decode(self, mode, tgt_m: Sequence[int], block: int = 1, max_iters: int = 0, horizon: int = 0,
               stream=None, out=None, init=None, stop: str = "block"):
        """Returns (ids [B, m_max], lengths [B], k [B], flags [B]) as device int32 tensors.
        init: optional int32 tensor [B, >= max(tgt_m)], the initial draft (default all [PAD]).
        stop: "block" (Eq. (3)) or "prefix" (PD_STOP_PREFIX)."""
        import torch
        mode_id = mode_word(mode, stop)
        tgt_m = [int(x) for x in tgt_m]
        if len(tgt_m) != self.B:
            raise PdError(1, f"tgt_m has {len(tgt_m)} entries, the encoded batch has {self.B}")
        m_max = max(tgt_m)
        B = len(tgt_m)
        if out is None:   # at least one column, so that the library itself reports a bad tgt_m
            out = (torch.empty((B, max(m_max, 1)), dtype=torch.int32, device=self.device),
                   torch.empty(B, dtype=torch.int32, device=self.device),
                   torch.empty(B, dtype=torch.int32, device=self.device),
                   torch.empty(B, dtype=torch.int32, device=self.device))
        ids, ln, k, fl = out
        if init is None:
            _check(load_library().pd_decode(self.handle, mode_id, int(block), int(horizon), int(max_iters),
                                            _host_i32(tgt_m), ctypes.c_void_p(ids.data_ptr()), ids.shape[1],
                                            ctypes.c_void_p(ln.data_ptr()), ctypes.c_void_p(k.data_ptr()),
                                            ctypes.c_void_p(fl.data_ptr()), ctypes.c_void_p(_stream_handle(stream))))
        else:
            init = init.to(device=self.device, dtype=torch.int32).contiguous()
            if init.dim() != 2 or init.shape[0] != B:
                raise PdError(1, f"init must be [B, >= m_max], got {tuple(init.shape)}")
            self._init = init                # keep alive until the kernels have read it
            _check(load_library().pd_decode_init(self.handle, mode_id, int(block), int(horizon), int(max_iters),
                                                 _host_i32(tgt_m), ctypes.c_void_p(init.data_ptr()), init.shape[1],
                                                 ctypes.c_void_p(ids.data_ptr()), ids.shape[1],
                                                 ctypes.c_void_p(ln.data_ptr()), ctypes.c_void_p(k.data_ptr()),
                                                 ctypes.c_void_p(fl.data_ptr()),
                                                 ctypes.c_void_p(_stream_handle(stream))))
        return ids, ln, k, fl

    def decode_beam(self, tgt_m: Sequence[int], beam: int = 5, alpha: float = 1.0, cache: str = "native", stream=None):
        """Beam search (pd_decode_beam): (ids [B, beam, m_max], lengths [B, beam], scores [B, beam] float32, k [B],
        flags [B]) as device tensors, hypotheses best first.  cache: "native" (the model's type) or "int4".  One
        workspace, of the most that a call has needed, is kept with the context."""
        import torch
        tgt_m = [int(x) for x in tgt_m]
        if len(tgt_m) != self.B:
            raise PdError(1, f"tgt_m has {len(tgt_m)} entries, the encoded batch has {self.B}")
        if cache not in ("native", "int4"):
            raise PdError(1, f"unknown cache type {cache!r}")
        L = load_library()
        dt = CACHE_TYPES[self.model.cfg.dtype if cache == "native" else cache]
        n = ctypes.c_size_t()
        _check(L.pd_decode_beam_bytes(self.handle, int(beam), dt, ctypes.byref(n)))
        need = n.value
        dev = self.workspace.device
        B, m_max = len(tgt_m), max(tgt_m, default=0)
        rows = max(B, 1)                     # nothing encoded: the library itself reports it

        def launch(handle):
            if self._beam_ws is None or self._beam_ws.numel() < need + 256:
                self._beam_ws = None         # here, so that the new one is allocated on the stream that uses it
                self._beam_ws = torch.empty(need + 256, dtype=torch.uint8, device=dev)
            ws = self._beam_ws
            ws.record_stream(torch.cuda.current_stream(dev))
            ids = torch.empty((rows, beam, max(m_max, 1)), dtype=torch.int32, device=dev)
            ln = torch.empty((rows, beam), dtype=torch.int32, device=dev)
            scores = torch.empty((rows, beam), dtype=torch.float32, device=dev)
            k, fl = (torch.empty(rows, dtype=torch.int32, device=dev) for _ in range(2))
            _check(L.pd_decode_beam(self.handle, int(beam), float(alpha), dt, _host_i32(tgt_m), ids.data_ptr(),
                                    ids.shape[2], ln.data_ptr(), scores.data_ptr(), k.data_ptr(), fl.data_ptr(),
                                    (ws.data_ptr() + 255) // 256 * 256, need, handle))
            return ids, ln, scores, k, fl

        return _on(dev, stream, launch)

    def decode_traced_static(self, mode, tgt_m: Sequence[int], capacity: int, block: int = 1, max_iters: int = 0,
                             horizon: int = 0, stream=None, stop: str = "block"):
        """pd_decode_traced_static: decode with the trace on, the trace scratch
        in the library's static array.  Returns (ids, lengths, k, flags,
        records, count); records is a numpy structured array (TRACE_DTYPE) of
        the first min(count, capacity) records."""
        import torch
        mode_id = mode_word(mode, stop)
        tgt_m = [int(x) for x in tgt_m]
        if len(tgt_m) != self.B:
            raise PdError(1, f"tgt_m has {len(tgt_m)} entries, the encoded batch has {self.B}")
        B = len(tgt_m)
        ids = torch.empty((B, max(max(tgt_m), 1)), dtype=torch.int32, device=self.device)
        ln, k, fl = (torch.empty(B, dtype=torch.int32, device=self.device) for _ in range(3))
        rec = torch.empty(max(int(capacity), 1) * 6, dtype=torch.int32, device=self.device)
        _check(load_library().pd_decode_traced_static(
            self.handle, mode_id, int(block), int(horizon), int(max_iters), _host_i32(tgt_m),
            ctypes.c_void_p(ids.data_ptr()), ids.shape[1], ctypes.c_void_p(ln.data_ptr()),
            ctypes.c_void_p(k.data_ptr()), ctypes.c_void_p(fl.data_ptr()), ctypes.c_void_p(rec.data_ptr()),
            int(capacity), ctypes.c_void_p(_stream_handle(stream))))
        torch.cuda.current_stream().synchronize() if stream is None else stream.synchronize()
        n = ctypes.c_int64()
        _check(load_library().pd_ctx_trace_count(self.handle, ctypes.byref(n)))
        kept = min(n.value, int(capacity))
        raw = rec[: kept * 6].cpu().numpy()
        return ids, ln, k, fl, raw.view(np.dtype(self.TRACE_DTYPE)), n.value

    def debug_logits(self, tgt_in, stream=None):
        """Teacher-forced logits [B, T, V] for decoder inputs tgt_in [B, T] (BOS first)."""
        import torch
        tgt_in = tgt_in.to(device=self.device, dtype=torch.int32).contiguous()
        B, T = tgt_in.shape
        logits = torch.empty((B, T, self.model.cfg.vocab), dtype=torch.float32, device=self.device)
        _check(load_library().pd_debug_logits(self.handle, ctypes.c_void_p(tgt_in.data_ptr()), T,
                                              ctypes.c_void_p(logits.data_ptr()),
                                              ctypes.c_void_p(_stream_handle(stream))))
        return logits

    def set_timing(self, enable: bool):
        _check(load_library().pd_ctx_set_timing(self.handle, int(enable)))

    def vocab_timing(self):
        """(launches, total_ms) of the fused vocabulary kernel since set_timing(True)."""
        n, ms = ctypes.c_int64(), ctypes.c_double()
        _check(load_library().pd_ctx_vocab_timing(self.handle, ctypes.byref(n), ctypes.byref(ms)))
        return n.value, ms.value

    def product_timing(self):
        """(launches, total_ms, bytes) of the decoder's timed product launches since set_timing(True)."""
        n, ms, b = ctypes.c_int64(), ctypes.c_double(), ctypes.c_double()
        _check(load_library().pd_ctx_product_timing(self.handle, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(b)))
        return n.value, ms.value, b.value

    def iteration_kernels(self) -> int:
        """Kernels in the iteration graph replayed last."""
        n = ctypes.c_int64()
        _check(load_library().pd_ctx_iteration_kernels(self.handle, ctypes.byref(n)))
        return n.value

    def rows_processed(self) -> int:
        """Rows evaluated by all iterations since set_timing (synchronous)."""
        n = ctypes.c_int64()
        _check(load_library().pd_ctx_rows_processed(self.handle, ctypes.byref(n)))
        return n.value

    TRACE_DTYPE = [("iteration", "<i4"), ("sentence", "<i4"), ("position", "<i4"), ("token", "<i4"),
                   ("top1", "<f4"), ("lse", "<f4")]

    def set_trace(self, capacity: int, max_rows: int):
        """Turn the decoding trace on (capacity records, iterations of up to
        max_rows rows; both buffers allocated here) or off (capacity 0)."""
        import torch
        L = load_library()
        if capacity <= 0:
            _check(L.pd_ctx_set_trace(self.handle, None, 0, None, 0))
            self._trace = None
            return
        nbytes = ctypes.c_size_t()
        _check(L.pd_trace_scratch_bytes(self.model.handle, int(max_rows), ctypes.byref(nbytes)))
        rec = torch.empty(capacity * 6, dtype=torch.int32, device=self.device)
        scratch = torch.empty(nbytes.value // 8, dtype=torch.float64, device=self.device)
        _check(L.pd_ctx_set_trace(self.handle, ctypes.c_void_p(rec.data_ptr()), int(capacity),
                                  ctypes.c_void_p(scratch.data_ptr()), nbytes.value))
        self._trace = (rec, scratch)

    def trace(self):
        """Records appended since set_trace, as a numpy structured array
        (fields of TRACE_DTYPE), and the full count (may exceed capacity)."""
        if getattr(self, "_trace", None) is None:
            raise PdError(6, "tracing is off: call set_trace first")
        n = ctypes.c_int64()
        _check(load_library().pd_ctx_trace_count(self.handle, ctypes.byref(n)))
        rec = self._trace[0]
        kept = min(n.value, rec.numel() // 6)
        raw = rec[: kept * 6].cpu().numpy()
        return raw.view(np.dtype(self.TRACE_DTYPE)), n.value

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.pd_ctx_destroy(self.handle)
            self.handle = None


# --- beam search's operators ---------------------------------------------------
# They are for decoding: tensors that require a gradient are refused unless gradients are off.


class BeamStep(NamedTuple):
    """Survivors of a step, [B, beam] each, best first (flags [B]): see pd_beam_select."""
    scores: object
    parents: object
    tokens: object
    lens: object
    done: object
    src: object
    flags: object


class PageFork(NamedTuple):
    """New table, lengths, references per page, and (sequences without a slot, pages in use)."""
    table: object
    lens: object
    refs: object
    status: object


class PageMoves(NamedTuple):
    """Table with the new ids, new id of each page (-1: free), and (pages moved, pages in use)."""
    table: object
    remap: object
    status: object


def _on(dev, stream, launch, *used):
    """launch(stream handle) with `stream` (default: the current stream of `dev`) made current, so that outputs and
    scratch belong to it.  The tensors `used` (None: not there) are kept from reuse until a given stream has read them."""
    import torch
    if stream is not None:
        if stream.device != dev:
            raise PdError(1, f"the stream is on {stream.device}, the tensors are on {dev}")
        with torch.cuda.stream(stream):
            out = launch(stream.cuda_stream)
        for t in used:
            if t is not None:
                t.record_stream(stream)
        return out
    if dev.index != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            return launch(torch._C._cuda_getCurrentRawStream(dev.index))
    return launch(torch._C._cuda_getCurrentRawStream(dev.index))


def _tensor(name, t, dtypes, shape, dev, contiguous=True):
    """Refuses anything but a tensor of one of the dtypes, of the shape (None: any size) on the device."""
    import torch
    try:                                     # the usual case, quickly
        if t.dtype in dtypes and t.shape == shape and t.device == dev and t.is_cuda and (not contiguous or t.is_contiguous()):
            return t
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise PdError(1, f"{name} must be a tensor of {' or '.join(str(d) for d in dtypes)}")
    if t.dim() != len(shape) or any(w is not None and n != w for n, w in zip(t.shape, shape)):
        raise PdError(2, f"{name} has shape {tuple(t.shape)}, expected {tuple('any' if w is None else w for w in shape)}")
    if t.device != dev or dev.type != "cuda":
        raise PdError(1, f"{name} is on {t.device}: every tensor of a call belongs on one GPU")
    if contiguous and not t.is_contiguous():
        raise PdError(1, f"{name} must be contiguous")
    return t


def _shape(t, dims):
    """A tensor's own shape, or that of any tensor of `dims` dimensions where it is not one (_tensor then refuses it)."""
    shape = getattr(t, "shape", ())
    return shape if len(shape) == dims else (None,) * dims


def _no_gradient(**tensors):
    """Refuses tensors that would lose a gradient: the operators have no backward pass."""
    import torch
    for name, t in tensors.items():
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise PdError(5, f"{name} requires a gradient, which this operator does not give: detach it, or call under "
                             "torch.no_grad()")


def _rows(name, t):
    """Elements from one row of a 3-D tensor to the next: the last two dimensions packed, rows of any distance."""
    if t.is_contiguous():
        return t.shape[1] * t.shape[2]
    n = t.shape[2]
    if (t.shape[2] > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != n):
        raise PdError(1, f"the rows of {name} must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * n


def beam_select(logits, scores, lens, done, *, eos_id: int = C.EOS_ID, pad_id: int = C.PAD_ID, alpha: float = 1.0,
                max_len=None, stream=None) -> BeamStep:
    """One step of beam search (pd_beam_select): logits [B, beam, V] float32 or bfloat16 (rows of any distance,
    the beams of a sentence evenly spaced), scores float32, lens and done int32 [B, beam], max_len int32 [B] or None."""
    import torch
    L = load_library()
    if not isinstance(scores, torch.Tensor):
        raise PdError(1, "scores must be a tensor")
    dev = scores.device
    f32, i32 = (torch.float32,), (torch.int32,)
    shape = _shape(logits, 3)
    _tensor("logits", logits, (torch.float32, torch.bfloat16), shape, dev, contiguous=False)
    B, K, V = shape
    ld = logits.stride(1) if K > 1 else logits.stride(0) if B > 1 else V
    if (V > 1 and logits.stride(2) != 1) or (B > 1 and logits.stride(0) != K * ld):
        raise PdError(1, "the rows of logits must be contiguous and evenly spaced")
    _tensor("scores", scores, f32, (B, K), dev)
    _tensor("lens", lens, i32, (B, K), dev)
    _tensor("done", done, i32, (B, K), dev)
    if max_len is not None:
        _tensor("max_len", max_len, i32, (B,), dev)
    _no_gradient(logits=logits, scores=scores)
    dt = 1 if logits.dtype == torch.bfloat16 else 0
    n = ctypes.c_size_t()
    _check(L.pd_beam_select_bytes(dt, B, K, V, ctypes.byref(n)))

    def launch(handle):
        out = torch.empty_like(scores)
        ints = lens.new_empty(5, B, K)
        flags = lens.new_empty(B)
        ws = lens.new_empty(-(-n.value // 4))
        at, step = ints.data_ptr(), 4 * B * K
        _check(L.pd_beam_select(logits.data_ptr(), dt, ld, B, K, V, scores.data_ptr(), lens.data_ptr(),
                                done.data_ptr(), None if max_len is None else max_len.data_ptr(), eos_id, pad_id,
                                alpha, out.data_ptr(), at, at + step, at + 2 * step, at + 3 * step, at + 4 * step,
                                flags.data_ptr(), ws.data_ptr(), n.value, handle))
        return BeamStep(out, *ints.unbind(0), flags)

    return _on(dev, stream, launch, logits, scores, lens, done, max_len)


class PagedCache:
    """A pool of pages of keys and values (pd_cache): dtype "f32", "bf16" or "int4", layouts as pdec.h states.

    The tensors are allocated here (zeroed) unless given.  Page tables are int32 [sequences, pages], lengths int32."""

    def __init__(self, dtype: str, layers: int, pages: int, page_size: int, kv_heads: int, head_dim: int, *, k=None,
                 v=None, k_scale=None, v_scale=None, device="cuda"):
        import torch
        if dtype not in CACHE_TYPES:
            raise PdError(1, f"unknown cache dtype {dtype!r}")
        c = pd_cache(CACHE_TYPES[dtype], layers, pages, page_size, kv_heads, head_dim)
        kv, sc = ctypes.c_size_t(), ctypes.c_size_t()
        _check(load_library().pd_cache_bytes(ctypes.byref(c), ctypes.byref(kv), ctypes.byref(sc)))
        t = {"f32": torch.float32, "bf16": torch.bfloat16, "int4": torch.uint8}[dtype]
        pack = 2 if dtype == "int4" else 1
        head = (layers, pages, kv_heads)
        shapes = {"k": (t, head + (page_size, head_dim // pack)), "v": (t, head + (head_dim, page_size // pack))}
        if dtype == "int4":
            shapes["k_scale"] = shapes["v_scale"] = (torch.bfloat16, head + (page_size, max(1, head_dim // 32), 2))
        given = {"k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale}
        dev = k.device if k is not None else torch.empty(0, device=device).device
        for name, x in given.items():
            if name not in shapes:
                if x is not None:
                    raise PdError(1, f"{name} is for a cache in 4 bits")
                setattr(self, name, None)
                continue
            dt, shape = shapes[name]
            if x is None:
                x = torch.zeros(shape, dtype=dt, device=dev)
            setattr(self, name, _tensor(name, x, (dt,), shape, dev))
            setattr(c, name, x.data_ptr())
        _no_gradient(k=k, v=v, k_scale=k_scale, v_scale=v_scale)
        self.dtype, self.layers, self.pages, self.page_size = dtype, layers, pages, page_size
        self.kv_heads, self.head_dim, self.device = kv_heads, head_dim, dev
        self._c = c
        self._p = ctypes.byref(c)
        self._buffers = self.k, self.v, self.k_scale, self.v_scale

    def _table(self, table, lens):
        import torch
        i32 = (torch.int32,)
        shape = _shape(table, 2)
        _tensor("table", table, i32, shape, self.device)
        _tensor("lens", lens, i32, shape[:1], self.device)
        return shape

    def _bytes(self, fn, *sizes):
        n = ctypes.c_size_t()
        _check(getattr(load_library(), fn)(self._p, *sizes, ctypes.byref(n)))
        return n.value

    def attend(self, q, table, lens, *, layer: int = 0, group: int = 1, max_len: Optional[int] = None, new_k=None,
               new_v=None, out_dtype=None, scale: Optional[float] = None, stream=None):
        """out [S, heads, head_dim] of q [S, heads, head_dim] over each sequence's keys (pd_cache_attend); new_k and
        new_v [S, kv_heads, head_dim] are appended at position lens - 1 first.  max_len: a bound on the lengths
        (default: what the table can name); out_dtype: float32 or bfloat16 (default: q's)."""
        import torch
        L = load_library()
        S, ld = self._table(table, lens)
        dev, dh = self.device, self.head_dim
        types = (torch.float32, torch.bfloat16)
        H = _shape(q, 3)[1]
        _tensor("q", q, types, (S, H, dh), dev, contiguous=False)
        _no_gradient(q=q)
        odt = q.dtype if out_dtype is None else out_dtype
        if odt not in types:
            raise PdError(1, "out_dtype must be torch.float32 or torch.bfloat16")
        if (new_k is None) != (new_v is None):
            raise PdError(1, "new_k and new_v go together")
        kp = vp = None
        ndt = nld = 0
        if new_k is not None:
            shape = (S, self.kv_heads, dh)
            _tensor("new_k", new_k, types, shape, dev, contiguous=False)
            _tensor("new_v", new_v, types, shape, dev, contiguous=False)
            nld = _rows("new_k", new_k)
            if new_v.dtype != new_k.dtype or _rows("new_v", new_v) != nld:
                raise PdError(1, "new_k and new_v must have the same type and row distance")
            _no_gradient(new_k=new_k, new_v=new_v)
            kp, vp, ndt = new_k.data_ptr(), new_v.data_ptr(), int(new_k.dtype == torch.bfloat16)
        top = ld * self.page_size if max_len is None else max_len
        n = self._bytes("pd_cache_attend_bytes", H, S, group, top)

        def launch(handle):
            out = torch.empty((S, H, dh), dtype=odt, device=dev) if odt != q.dtype else q.new_empty(S, H, dh)
            ws = lens.new_empty(-(-n // 4)) if n else None
            _check(L.pd_cache_attend(self._p, layer, q.data_ptr(), int(q.dtype == torch.bfloat16), _rows("q", q), H, kp,
                                     vp, ndt, nld, table.data_ptr(), ld, lens.data_ptr(), S, group, top,
                                     dh ** -0.5 if scale is None else scale, out.data_ptr(),
                                     int(odt == torch.bfloat16), H * dh, None if ws is None else ws.data_ptr(), n, handle))
            return out

        return _on(dev, stream, launch, *self._buffers, q, new_k, new_v, table, lens)

    def read(self, table, lens, first, *, layer: int = 0, count: int = 1, stream=None):
        """Values held at positions first .. first + count - 1 of each sequence, float32
        ([S, count, kv_heads, head_dim] of keys, of values); zero outside the sequence."""
        import torch
        S, ld = self._table(table, lens)
        dev = self.device
        _tensor("first", first, (torch.int32,), (S,), dev)

        def launch(handle):
            shape = (S, max(count, 1), self.kv_heads, self.head_dim)
            k = torch.empty(shape, dtype=torch.float32, device=dev)
            v = torch.empty_like(k)
            _check(load_library().pd_cache_read(self._p, layer, table.data_ptr(), ld, lens.data_ptr(), S,
                                                first.data_ptr(), count, k.data_ptr(), v.data_ptr(), handle))
            return k, v

        return _on(dev, stream, launch, *self._buffers, table, lens, first)

    def fork(self, table, lens, parents, *, grow: bool = True, stream=None) -> PageFork:
        """The table of the sequences whose parents are given (-1: empty), with a slot for the next token if grow
        (pd_pages_fork)."""
        import torch
        S, ld = self._table(table, lens)
        dev = self.device
        _tensor("parents", parents, (torch.int32,), _shape(parents, 1), dev)
        n_out = parents.shape[0]
        n = self._bytes("pd_pages_bytes", n_out)

        def launch(handle):
            new = lens.new_empty(n_out, ld)
            rest = lens.new_empty(n_out + self.pages + 2)
            ws = lens.new_empty(-(-n // 4))
            at = rest.data_ptr()
            _check(load_library().pd_pages_fork(self._p, table.data_ptr(), ld, lens.data_ptr(), S, parents.data_ptr(),
                                                n_out, int(grow), new.data_ptr(), at, at + 4 * n_out,
                                                at + 4 * (n_out + self.pages), ws.data_ptr(), n, handle))
            return PageFork(new, *rest.split_with_sizes((n_out, self.pages, 2)))

        return _on(dev, stream, launch, *self._buffers, table, lens, parents)

    def compact(self, table, lens, *, stream=None) -> PageMoves:
        """Moves the pages in use to the front of the pool (pd_pages_compact)."""
        import torch
        S, ld = self._table(table, lens)
        dev = self.device
        n = self._bytes("pd_pages_bytes", S)

        def launch(handle):
            new = lens.new_empty(S, ld)
            rest = lens.new_empty(self.pages + 2)
            ws = lens.new_empty(-(-n // 4))
            at = rest.data_ptr()
            _check(load_library().pd_pages_compact(self._p, table.data_ptr(), ld, lens.data_ptr(), S, new.data_ptr(), at,
                                                   at + 4 * self.pages, ws.data_ptr(), n, handle))
            return PageMoves(new, *rest.split_with_sizes((self.pages, 2)))

        return _on(dev, stream, launch, *self._buffers, table, lens)
