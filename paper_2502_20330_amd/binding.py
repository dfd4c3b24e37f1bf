"""ctypes binding of librapid.so: argument marshalling only.

Every step of the verification path runs in the library's gfx950 kernels; torch
supplies device memory and the stream.  There is no CPU fallback: if the library
has not been built, importing works but the first call raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "librapid.so")

RAPID_OK = 0
RAPID_EINVAL, RAPID_EALIGN, RAPID_EUNSUPPORTED, RAPID_EWORKSPACE, RAPID_EHIP, RAPID_ETOOLARGE = -1, -2, -3, -4, -5, -6
STATIC_SCRATCH_BYTES = 32 << 20
OPT_ACCEPT_WAIT_US, OPT_ACCEPT_SLICE, OPT_PROBE_SKEW, OPT_ATTN_WAIT_US = 1, 2, 3, 4
EXPORTS = ["rapid_create", "rapid_destroy", "rapid_strerror", "rapid_last_hip_error", "rapid_set_option",
           "rapid_verify_attn_chunk", "rapid_verify_attn_workspace_bytes", "rapid_verify_attn",
           "rapid_verify_attn_exchange_bytes", "rapid_verify_attn_exchange", "rapid_verify_attn_static",
           "rapid_accept_workspace_bytes", "rapid_accept", "rapid_accept_prestats", "rapid_accept_filled",
           "rapid_lm_head_chunk", "rapid_lm_head_stat_chunks", "rapid_lm_head", "rapid_kv_append", "rapid_kv_commit",
           "rapid_kv_commit_pages",
           "rapid_kv_append_quant", "rapid_kv_read_quant", "rapid_verify_attn_quant", "rapid_verify_attn_quant_workspace_bytes",
           "rapid_verify_attn_prefix", "rapid_verify_attn_prefix_workspace_bytes",
           "rapid_verify_attn_window", "rapid_verify_attn_window_workspace_bytes", "rapid_verify_attn_window_plan",
           "rapid_kv_append_rope", "rapid_kv_append_rope_quant", "rapid_quant_rows", "rapid_lm_head_quant",
           "rapid_lm_head_quant_workspace_bytes",
           "rapid_retrieve", "rapid_hbm_read_probe"]


class RapidError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"librapid: {message} (status {status})")
        self.status = status


class AttnShape(ctypes.Structure):
    """Mirror of ``rapid_attn_shape`` in include/rapid.h."""
    _fields_ = [("batch", ctypes.c_int32), ("q_max", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("max_ctx", ctypes.c_int32),
                ("gamma", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("kv_batch_stride", ctypes.c_int64), ("kv_token_stride", ctypes.c_int64),
                ("kv_head_stride", ctypes.c_int64), ("kv_page_stride", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("chunk_tokens", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("ctx_sum_hint", ctypes.c_int64)]


class QuantLayout(ctypes.Structure):
    """Mirror of ``rapid_quant_layout`` in include/rapid.h."""
    _fields_ = [("scale_batch_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64),
                ("scale_page_stride", ctypes.c_int64)]


class PrefixLayout(ctypes.Structure):
    """Mirror of ``rapid_prefix_layout`` in include/rapid.h."""
    _fields_ = [("max_prefix", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class Rope(ctypes.Structure):
    """Mirror of ``rapid_rope`` in include/rapid.h."""
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("amplitude", ctypes.c_float),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64)]


_lib = None


def load_library() -> ctypes.CDLL:
    """Load librapid.so and declare the C signatures.  Raises if it is not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RapidError(-100, f"{LIB_PATH} not found: build it with "
                               "`python -m paper_2502_20330_amd.build` (there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    lib.rapid_create.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    lib.rapid_create.restype = ctypes.c_int
    lib.rapid_destroy.argtypes = [ctypes.c_void_p]
    lib.rapid_destroy.restype = None
    lib.rapid_strerror.argtypes = [ctypes.c_int]
    lib.rapid_strerror.restype = ctypes.c_char_p
    lib.rapid_last_hip_error.argtypes = [ctypes.c_void_p]
    lib.rapid_last_hip_error.restype = ctypes.c_int
    lib.rapid_set_option.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64]
    lib.rapid_set_option.restype = ctypes.c_int
    lib.rapid_verify_attn_chunk.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape)]
    lib.rapid_verify_attn_chunk.restype = ctypes.c_int
    lib.rapid_verify_attn_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape)]
    lib.rapid_verify_attn_workspace_bytes.restype = ctypes.c_size_t
    lib.rapid_verify_attn.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape), vp, vp, vp, i32p, i32p, i32p,
                                      vp, f32p, vp, ctypes.c_size_t, vp]
    lib.rapid_verify_attn.restype = ctypes.c_int
    lib.rapid_verify_attn_exchange_bytes.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape)]
    lib.rapid_verify_attn_exchange_bytes.restype = ctypes.c_size_t
    lib.rapid_verify_attn_exchange.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape), vp, vp, vp, i32p, i32p, i32p,
                                               vp, f32p, vp, ctypes.c_size_t, vp, ctypes.c_size_t, vp]
    lib.rapid_verify_attn_exchange.restype = ctypes.c_int
    lib.rapid_verify_attn_static.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape), vp, vp, vp, i32p, i32p, i32p,
                                             vp, f32p, vp]
    lib.rapid_verify_attn_static.restype = ctypes.c_int
    lib.rapid_accept_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    lib.rapid_accept_workspace_bytes.restype = ctypes.c_size_t
    lib.rapid_accept.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, f32p, f32p, i32p, i32p,
                                 ctypes.c_float, ctypes.c_float, ctypes.c_float, f32p, i32p, i32p, f32p,
                                 vp, ctypes.c_size_t, vp]
    lib.rapid_accept.restype = ctypes.c_int
    lib.rapid_accept_prestats.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, f32p, f32p, i32p, i32p,
                                          ctypes.c_float, ctypes.c_float, ctypes.c_float, f32p,
                                          f32p, ctypes.c_int, f32p, ctypes.c_int, i32p, i32p, f32p,
                                          vp, ctypes.c_size_t, vp]
    lib.rapid_accept_prestats.restype = ctypes.c_int
    lib.rapid_accept_filled.argtypes = lib.rapid_accept_prestats.argtypes
    lib.rapid_accept_filled.restype = ctypes.c_int
    lib.rapid_lm_head_chunk.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    lib.rapid_lm_head_chunk.restype = ctypes.c_int
    lib.rapid_lm_head_stat_chunks.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    lib.rapid_lm_head_stat_chunks.restype = ctypes.c_int
    lib.rapid_lm_head.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp, ctypes.c_float,
                                  f32p, ctypes.c_int64, f32p, vp]
    lib.rapid_lm_head.restype = ctypes.c_int
    lib.rapid_kv_append.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape), vp, vp, i32p, i32p, i32p, vp, vp, vp]
    lib.rapid_kv_append.restype = ctypes.c_int
    lib.rapid_kv_commit.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, i32p, i32p, i32p, vp]
    lib.rapid_kv_commit.restype = ctypes.c_int
    lib.rapid_kv_commit_pages.argtypes = [ctypes.c_void_p, ctypes.POINTER(AttnShape), i32p, i32p, i32p, i32p, i32p,
                                          ctypes.c_int, i32p, vp]
    lib.rapid_kv_commit_pages.restype = ctypes.c_int
    shape_p, quant_p, prefix_p = ctypes.POINTER(AttnShape), ctypes.POINTER(QuantLayout), ctypes.POINTER(PrefixLayout)
    lib.rapid_kv_append_quant.argtypes = [vp, shape_p, quant_p, vp, vp, i32p, i32p, i32p, vp, vp, vp, vp, vp]
    lib.rapid_kv_append_quant.restype = ctypes.c_int
    lib.rapid_kv_read_quant.argtypes = [vp, shape_p, quant_p, vp, vp, vp, vp, i32p, i32p, i32p, vp, vp, vp]
    lib.rapid_kv_read_quant.restype = ctypes.c_int
    lib.rapid_verify_attn_quant_workspace_bytes.argtypes = [vp, shape_p]
    lib.rapid_verify_attn_quant_workspace_bytes.restype = ctypes.c_size_t
    lib.rapid_verify_attn_quant.argtypes = [vp, shape_p, quant_p, vp, vp, vp, vp, vp, i32p, i32p, i32p, vp, f32p,
                                            vp, ctypes.c_size_t, vp]
    lib.rapid_verify_attn_quant.restype = ctypes.c_int
    lib.rapid_verify_attn_prefix_workspace_bytes.argtypes = [vp, shape_p, prefix_p]
    lib.rapid_verify_attn_prefix_workspace_bytes.restype = ctypes.c_size_t
    lib.rapid_verify_attn_prefix.argtypes = [vp, shape_p, prefix_p, vp, vp, vp, i32p, i32p, vp, vp, i32p, i32p, i32p, vp, f32p,
                                             vp, ctypes.c_size_t, vp]
    lib.rapid_verify_attn_prefix.restype = ctypes.c_int
    lib.rapid_verify_attn_window_workspace_bytes.argtypes = [vp, shape_p, ctypes.c_int, ctypes.c_int]
    lib.rapid_verify_attn_window_workspace_bytes.restype = ctypes.c_size_t
    lib.rapid_verify_attn_window_plan.argtypes = [vp, shape_p, ctypes.c_int, ctypes.c_int, i32p]
    lib.rapid_verify_attn_window_plan.restype = ctypes.c_int
    lib.rapid_verify_attn_window.argtypes = [vp, shape_p, ctypes.c_int, ctypes.c_int, vp, vp, vp, i32p, i32p, i32p, vp, f32p,
                                             vp, ctypes.c_size_t, vp]
    lib.rapid_verify_attn_window.restype = ctypes.c_int
    rope_p = ctypes.POINTER(Rope)
    lib.rapid_kv_append_rope.argtypes = [vp, shape_p, rope_p, vp, vp, vp, f32p, i32p, i32p, i32p, i32p, vp, vp, vp, vp]
    lib.rapid_kv_append_rope.restype = ctypes.c_int
    lib.rapid_kv_append_rope_quant.argtypes = [vp, shape_p, quant_p, rope_p, vp, vp, vp, f32p, i32p, i32p, i32p, i32p, vp, vp, vp, vp, vp,
                                               vp]
    lib.rapid_kv_append_rope_quant.restype = ctypes.c_int
    lib.rapid_quant_rows.argtypes = [vp, ctypes.c_int64, ctypes.c_int, vp, ctypes.c_int64, vp, f32p, vp]
    lib.rapid_quant_rows.restype = ctypes.c_int
    lib.rapid_lm_head_quant_workspace_bytes.argtypes = [vp, ctypes.c_int, ctypes.c_int]
    lib.rapid_lm_head_quant_workspace_bytes.restype = ctypes.c_size_t
    lib.rapid_lm_head_quant.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp, f32p, ctypes.c_float, f32p, ctypes.c_int64,
                                        f32p, vp, ctypes.c_size_t, vp]
    lib.rapid_lm_head_quant.restype = ctypes.c_int
    lib.rapid_retrieve.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, f32p, f32p, ctypes.c_int, ctypes.c_float,
                                   f32p, i32p, i32p, vp]
    lib.rapid_retrieve.restype = ctypes.c_int
    lib.rapid_hbm_read_probe.argtypes = [ctypes.c_void_p, vp, ctypes.c_size_t, vp, vp]
    lib.rapid_hbm_read_probe.restype = ctypes.c_int
    _lib = lib
    return lib


def _check(lib, status: int, ctx=None):
    if status != RAPID_OK:
        msg = lib.rapid_strerror(status).decode()
        if ctx is not None and status == -5:
            msg += f" (hip error {lib.rapid_last_hip_error(ctx)})"
        raise RapidError(status, msg)


# A call of a few microseconds of device time must not wait for its marshalling: plain integers go where the prototypes
# say c_void_p (ctypes converts them), the raw stream comes from torch without a Stream object.
def _dptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _strides(t: torch.Tensor):
    """Strides of [rows, .., d] without what torch keeps for axes of length 1, which nothing steps along."""
    d = t.shape[-1]
    return tuple(s if n > 1 or i == t.dim() - 1 else (d if t.dim() == 4 and i == 1 else 0)
                 for i, (n, s) in enumerate(zip(t.shape, t.stride())))


def _sizes(*tensors) -> bytes:
    """What a call's checks go by, for a key: each tensor's type, device, sizes and strides."""
    global _sizes
    try:
        from ._signature import sizes
    except ImportError as e:
        raise RapidError(-100, f"{_PKG}/_signature.so: {e}; build it with `python -m paper_2502_20330_amd.build`") from e
    _sizes = sizes
    return sizes(*tensors)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(device: torch.device) -> int:
    if _raw_stream is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


class Rapid:
    """One library context on one GPU plus a grow-only workspace tensor."""

    def __init__(self, device: int = 0):
        if not torch.cuda.is_available():
            raise RapidError(-101, "no GPU visible: the verification path has no CPU implementation")
        self.lib = load_library()
        self.device = torch.device("cuda", device)
        self._ctx = ctypes.c_void_p()
        torch.cuda.set_device(self.device)
        _check(self.lib, self.lib.rapid_create(ctypes.byref(self._ctx), device))
        self._ws: Optional[torch.Tensor] = None
        self._ws_exchange: Optional[torch.Tensor] = None
        self._ws_args = (None, 0, None, 0)             # address and size of the exchange memory and of the workspace, as a call takes them
        self._ws_accept: Optional[torch.Tensor] = None
        self._ws_streams: dict = {}                    # address and size of the quantised and the prefix attention's workspace, by stream
        self._ws_kept: dict = {}                       # and the tensors
        self._plans: dict = {}                         # shapes and layouts of calls by their sizes (_planned)
        self._sink: Optional[torch.Tensor] = None

    def close(self):
        if self._ctx:
            self.lib.rapid_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_option(self, option: int, value: int):
        _check(self.lib, self.lib.rapid_set_option(self._ctx, int(option), int(value)))

    def accept_status(self):
        """(rejected out-of-range draft ids, exchange waits that gave up) of the last rapid_accept call that
        used this object's workspace; synchronises."""
        torch.cuda.synchronize(self.device)
        w = self._ws_accept[:8].view(torch.int32).cpu()
        return int(w[0]), int(w[1])

    def _workspace(self, nbytes: int) -> torch.Tensor:
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
            self._ws_args = (*self._ws_args[:2], self._ws.data_ptr(), self._ws.numel())
        return self._ws

    def _exchange_workspace(self, nbytes: int) -> torch.Tensor:
        # its own buffer, zero at first: the attention call keeps the number of the call in it.  At once large enough for every
        # shape (128 workgroups of 32 rows of 64)
        if self._ws_exchange is None or self._ws_exchange.numel() < nbytes:
            self._ws_exchange = torch.zeros(max(nbytes, 3 << 20), dtype=torch.uint8, device=self.device)
            self._ws_args = (self._ws_exchange.data_ptr(), self._ws_exchange.numel(), *self._ws_args[2:])
        return self._ws_exchange

    def clear_exchange(self):
        """Attention calls of this object that overlapped in time (on two streams, or a graph's replay beside an eager call) can spoil
        later ones too, until the memory that they exchange their partial results through is cleared: by this method, on the current
        stream, after they have ended."""
        if self._ws_exchange is not None:
            self._ws_exchange.zero_()

    def _accept_workspace(self, nbytes: int) -> torch.Tensor:
        # its own buffer: the accept pass keeps a call counter in it from one call to the next
        if self._ws_accept is None or self._ws_accept.numel() < nbytes:
            self._ws_accept = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        return self._ws_accept

    # ------------------------------------------------------------------ attention
    def attn_shape(self, q, k_cache, ctx_max: int, *, gamma: Optional[int] = None, page_table=None,
                   softmax_scale: Optional[float] = None, chunk_tokens: int = 0,
                   ctx_sum_hint: int = 0) -> AttnShape:
        B, Qmax, Hq, d = q.shape
        rows, tokens, Hkv, _ = k_cache.shape
        st0, st1, st2, st3 = k_cache.stride()
        if st3 != 1:
            raise RapidError(-1, "head_dim must be the contiguous dimension of the KV cache")
        scale = float(softmax_scale) if softmax_scale is not None else d ** -0.5
        gamma = Qmax - 1 if gamma is None else int(gamma)
        if page_table is None:
            return AttnShape(B, Qmax, Hq, Hkv, d, int(ctx_max), gamma, scale, st0, st1, st2, 0, 0, 0,
                             int(chunk_tokens), 0, int(ctx_sum_hint))
        return AttnShape(B, Qmax, Hq, Hkv, d, int(ctx_max), gamma, scale, 0, st1, st2, st0, tokens,
                         page_table.shape[1], int(chunk_tokens), rows, int(ctx_sum_hint))

    def verify_attn_chunk(self, shape: AttnShape) -> int:
        c = self.lib.rapid_verify_attn_chunk(self._ctx, ctypes.byref(shape))
        if c < 0:
            _check(self.lib, c)
        return c

    def rapid_verify_attn(self, q, k_cache, v_cache, ctx_lens, gamma: Optional[int] = None, *, gammas=None,
                          page_table=None, max_ctx: Optional[int] = None, softmax_scale: Optional[float] = None,
                          chunk_tokens: int = 0, out=None, lse_out=None, shape: Optional[AttnShape] = None,
                          ctx_sum_hint: int = 0):
        """q bf16 [B,Qmax,Hq,d]; k_cache/v_cache bf16 [B,Lmax,Hkv,d] (any batch/token/head strides)
        or paged [n_pages,page,Hkv,d] with page_table int32 [B,max_pages]; ctx_lens int32 [B]
        (device).  ``max_ctx`` is a host upper bound of ctx_lens (default: the cache capacity).
        Returns out bf16 [B,Qmax,Hq,d]; fills lse_out fp32 [B,Hq,Qmax] if given."""
        assert q.dtype == torch.bfloat16 and k_cache.dtype == torch.bfloat16 and v_cache.dtype == torch.bfloat16
        assert q.is_contiguous() and ctx_lens.dtype == torch.int32
        assert k_cache.stride() == v_cache.stride() and k_cache.shape == v_cache.shape
        if shape is None:
            if max_ctx is None:
                max_ctx = k_cache.shape[1] if page_table is None else page_table.shape[1] * k_cache.shape[1]
            shape = self.attn_shape(q, k_cache, max_ctx, gamma=gamma, page_table=page_table,
                                    softmax_scale=softmax_scale, chunk_tokens=chunk_tokens,
                                    ctx_sum_hint=ctx_sum_hint)
        if out is None:
            out = torch.empty_like(q)
        args = (self._ctx, shape, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), ctx_lens.data_ptr(), _dptr(gammas),
                _dptr(page_table), out.data_ptr(), _dptr(lse_out))
        call, stream = self.lib.rapid_verify_attn_exchange, _stream_ptr(self.device)
        if self._ws_exchange is None and not torch.cuda.is_current_stream_capturing():   # (a fill that is only recorded does not clear it)
            self._exchange_workspace(0)
        rc = call(*args, *self._ws_args, stream)
        if rc == RAPID_EWORKSPACE:                             # the last check of the call: nothing has been launched
            need = 0 if self._ws_exchange is None else self.lib.rapid_verify_attn_exchange_bytes(self._ctx, shape)
            if need:
                self._exchange_workspace(need)
            else:
                self._workspace(self.lib.rapid_verify_attn_workspace_bytes(self._ctx, shape))
            rc = call(*args, *self._ws_args, stream)
        if rc:
            _check(self.lib, rc, self._ctx)
        return out

    def rapid_verify_attn_static(self, q, k_cache, v_cache, ctx_lens, gamma: Optional[int] = None, *, gammas=None,
                                 page_table=None, max_ctx: Optional[int] = None,
                                 softmax_scale: Optional[float] = None, chunk_tokens: int = 0, out, lse_out=None,
                                 ctx_sum_hint: int = 0):
        """The allocation-free form of :meth:`rapid_verify_attn`: the caller passes `out`, the split partials go
        to the library's static device array, and neither this method nor the library allocates anything."""
        if max_ctx is None:
            max_ctx = k_cache.shape[1] if page_table is None else page_table.shape[1] * k_cache.shape[1]
        shape = self.attn_shape(q, k_cache, max_ctx, gamma=gamma, page_table=page_table, softmax_scale=softmax_scale,
                                chunk_tokens=chunk_tokens, ctx_sum_hint=ctx_sum_hint)
        rc = self.lib.rapid_verify_attn_static(self._ctx, ctypes.byref(shape), _dptr(q), _dptr(k_cache),
                                               _dptr(v_cache), _dptr(ctx_lens), _dptr(gammas), _dptr(page_table),
                                               _dptr(out), _dptr(lse_out), _stream_ptr(self.device))
        _check(self.lib, rc, self._ctx)
        return out

    # ------------------------------------------------------------------ accept
    def rapid_accept(self, target_logits, draft_logits, draft_tokens, eta: float, uniforms, *, gammas=None,
                     temperature: float = 1.0, tail_alpha: float = 0.1, want_ratio: bool = True, outs=None,
                     target_stats=None, draft_stats=None):
        """target_logits fp32 [B,g+1,V], draft_logits fp32 [B,g,V], draft_tokens int32 [B,g],
        uniforms fp32 [B,g+1].  Returns (n_accepted int32 [B], out_tokens int32 [B,g+1], ratio fp32 [B,g] or None).
        target_stats / draft_stats: optional fp32 [rows, chunks, 2] row statistics (see rapid_lm_head); with
        either one the call goes to rapid_accept_prestats.  Ratios past a sequence's drafts are 0, in a buffer passed in
        `outs` untouched."""
        B, g1, V = target_logits.shape
        g = g1 - 1
        assert target_logits.dtype == torch.float32 and target_logits.is_contiguous()
        assert draft_logits.dtype == torch.float32 and draft_logits.is_contiguous() and draft_logits.shape == (B, g, V)
        assert draft_tokens.dtype == torch.int32 and draft_tokens.shape == (B, g) and draft_tokens.is_contiguous()
        assert uniforms.dtype == torch.float32 and uniforms.shape == (B, g + 1) and uniforms.is_contiguous()
        if outs is None:
            n_acc = torch.empty(B, dtype=torch.int32, device=self.device)
            toks = torch.empty(B, g + 1, dtype=torch.int32, device=self.device)
            ratio = torch.empty((B, g), dtype=torch.float32, device=self.device) if want_ratio else None
        else:
            n_acc, toks, ratio = outs
        # a ratio buffer made here is written in full (a fill of its own was a sixth of a small call's time); the caller's keeps what
        # it holds past a sequence's drafts
        fill = outs is None and want_ratio and gammas is not None
        prestats = fill or target_stats is not None or draft_stats is not None
        args = (self._ctx, B, g, V, target_logits.data_ptr(), draft_logits.data_ptr(), draft_tokens.data_ptr(), _dptr(gammas),
                float(eta), float(temperature), float(tail_alpha), uniforms.data_ptr())
        results = (_dptr(n_acc), _dptr(toks), _dptr(ratio))
        if prestats:
            for st, rows in ((target_stats, B * (g + 1)), (draft_stats, B * g)):
                assert st is None or (st.dtype == torch.float32 and st.is_contiguous() and st.dim() == 3
                                      and st.shape[0] == rows and st.shape[2] == 2)
            args += (_dptr(target_stats), 0 if target_stats is None else target_stats.shape[1],
                     _dptr(draft_stats), 0 if draft_stats is None else draft_stats.shape[1])
        call = self.lib.rapid_accept_filled if fill else self.lib.rapid_accept_prestats if prestats else self.lib.rapid_accept
        ws, stream = self._ws_accept, _stream_ptr(self.device)
        rc = call(*args, *results, _dptr(ws), 0 if ws is None else ws.numel(), stream)
        if rc == RAPID_EWORKSPACE:                             # the last check of the call: nothing has been launched
            ws = self._accept_workspace(self.lib.rapid_accept_workspace_bytes(self._ctx, B, g, V))
            rc = call(*args, *results, ws.data_ptr(), ws.numel(), stream)
        if rc:
            _check(self.lib, rc, self._ctx)
        return n_acc, toks, ratio

    # ------------------------------------------------------------------ cache bookkeeping
    def rapid_kv_append(self, k_cache, v_cache, k_new, v_new, ctx_lens, gamma: Optional[int] = None, *, gammas=None,
                        page_table=None, max_ctx: Optional[int] = None):
        """Writes rows 0..gamma_b of k_new/v_new (bf16 [B,Qmax,Hkv,d]) into the caches in place as the last
        gamma_b+1 tokens of every sequence (ctx_lens counts them).  Cache layout as for rapid_verify_attn."""
        B, Qmax, Hkv, d = k_new.shape
        assert k_new.is_contiguous() and v_new.is_contiguous() and v_new.shape == k_new.shape
        assert k_new.dtype == torch.bfloat16 and k_cache.dtype == torch.bfloat16
        q_like = k_new                                         # only sizes are read from it
        ctx_max = max_ctx if max_ctx is not None else (k_cache.shape[1] if page_table is None else
                                                       page_table.shape[1] * k_cache.shape[1])
        shape = self.attn_shape(q_like, k_cache, ctx_max, gamma=gamma if gamma is not None else Qmax - 1,
                                page_table=page_table)
        rc = self.lib.rapid_kv_append(self._ctx, ctypes.byref(shape), _dptr(k_new), _dptr(v_new), _dptr(ctx_lens),
                                      _dptr(gammas), _dptr(page_table), _dptr(k_cache), _dptr(v_cache),
                                      _stream_ptr(self.device))
        _check(self.lib, rc, self._ctx)

    def rapid_kv_commit(self, ctx_lens, n_accepted, gamma: int = 0, *, gammas=None):
        """ctx_lens[b] <- ctx_lens[b] - (gamma_b+1) + 1 + n_accepted[b], in place on the device."""
        assert ctx_lens.dtype == torch.int32 and n_accepted.dtype == torch.int32
        rc = self.lib.rapid_kv_commit(self._ctx, ctx_lens.numel(), int(gamma), _dptr(gammas), _dptr(n_accepted),
                                      _dptr(ctx_lens), _stream_ptr(self.device))
        _check(self.lib, rc, self._ctx)
        return ctx_lens

    def rapid_kv_commit_pages(self, ctx_lens, n_accepted, page_table, *, page_size: int, q_max: int, max_ctx: int,
                              gamma: Optional[int] = None, gammas=None, n_pages: int = 0):
        """The length update of :meth:`rapid_kv_commit` for a paged cache plus the page ids that can be handed
        back to the allocator.  Returns (released int32 [B, cap] (page ids, then -1), n_released int32 [B])."""
        B = ctx_lens.numel()
        s = AttnShape()
        s.batch, s.q_max, s.n_q_heads, s.n_kv_heads, s.head_dim = B, q_max, 1, 1, 128
        s.max_ctx, s.gamma, s.softmax_scale = int(max_ctx), (q_max - 1 if gamma is None else int(gamma)), 1.0
        s.kv_token_stride, s.kv_head_stride, s.kv_page_stride = 128, 128, 128 * page_size
        s.page_size, s.max_pages, s.n_pages = int(page_size), page_table.shape[1], int(n_pages)
        cap = (q_max + page_size - 2) // page_size + 1
        rel = torch.empty((B, cap), dtype=torch.int32, device=self.device)
        cnt = torch.empty(B, dtype=torch.int32, device=self.device)
        rc = self.lib.rapid_kv_commit_pages(self._ctx, ctypes.byref(s), _dptr(gammas), _dptr(n_accepted),
                                            _dptr(page_table), _dptr(ctx_lens), _dptr(rel), cap, _dptr(cnt),
                                            _stream_ptr(self.device))
        _check(self.lib, rc, self._ctx)
        return rel, cnt

    # ------------------------------------------------------------------ cache in 8 bits, shared prefix
    def _planned(self, key, plan, *args):
        """What a call of these sizes, strides, types and devices needs besides addresses: plan(*args) checks them and answers, once for
        each key, which holds them all (the checks took three times as long as the rest of a small call).  Numbers are the host's: a tensor in a
        key would stand for itself and not for its value."""
        self._need(not any(isinstance(x, torch.Tensor) for x in key), "sizes and the scale are numbers, not tensors")
        for t in args:
            self._need(not isinstance(t, torch.Tensor) or t.device == self.device, f"a tensor is not on {self.device}")
        got = plan(*args)
        if len(self._plans) >= 1024:                           # sizes that change all the time
            self._plans.clear()
        self._plans[key] = got
        return got

    @staticmethod
    def _need(ok, what: str):
        if not ok:
            raise RapidError(RAPID_EINVAL, what)

    def _check_lengths(self, batch: int, ctx_lens, gammas, page_table):
        """The index arrays that the calls on a batch share."""
        self._need(ctx_lens.dtype == torch.int32 and ctx_lens.shape == (batch,) and ctx_lens.is_contiguous(),
                   "ctx_lens: int32 [B], contiguous")
        self._need(gammas is None or (gammas.dtype == torch.int32 and gammas.shape == (batch,) and gammas.is_contiguous()),
                   "gammas: int32 [B], contiguous")
        self._need(page_table is None or (page_table.dtype == torch.int32 and page_table.dim() == 2 and
                                          page_table.shape[0] == batch and page_table.is_contiguous()),
                   "page_table: int32 [B, max_pages], contiguous")

    def _check_attn(self, q, out, lse_out):
        """q and the outputs of an attention call."""
        self._need(q.dtype == torch.bfloat16 and q.dim() == 4 and q.is_contiguous(), "q: bf16 [B, Qmax, Hq, d], contiguous")
        self._need(out.dtype == torch.bfloat16 and out.shape == q.shape and out.is_contiguous(), "out: bf16 like q, contiguous")
        self._need(lse_out is None or (lse_out.dtype == torch.float32 and lse_out.is_contiguous() and
                                       lse_out.shape == (q.shape[0], q.shape[2], q.shape[1])),
                   "lse_out: fp32 [B, Hq, Qmax], contiguous")

    def _check_cache(self, k_cache, v_cache):
        """A bf16 cache."""
        self._need(k_cache.dtype == torch.bfloat16 and v_cache.dtype == torch.bfloat16 and k_cache.dim() == 4
                   and k_cache.shape == v_cache.shape and _strides(k_cache) == _strides(v_cache) and k_cache.stride(3) == 1,
                   "k_cache and v_cache: bf16 [B or pages, tokens, Hkv, d], d contiguous, the same sizes and strides")

    def _quant_shape(self, batch, q_max, hq, gamma, k_codes, v_codes, k_scales, v_scales, page_table, max_ctx, softmax_scale):
        """References to the AttnShape and QuantLayout of a cache in 8 bits: codes [B or pages, tokens, Hkv, d] with any outer strides, scales
        [B or pages, Hkv, tokens], tokens contiguous and the rows a multiple of 16 long (views of memory that goes on are fine)."""
        one_byte = (torch.float8_e4m3fn, torch.uint8)
        scale_byte = (torch.float8_e8m0fnu, torch.uint8)
        self._need(k_codes.dtype in one_byte and v_codes.dtype in one_byte, "codes: float8_e4m3fn or uint8")
        self._need(k_scales.dtype in scale_byte and v_scales.dtype in scale_byte, "scales: float8_e8m0fnu or uint8")
        self._need(k_codes.dim() == 4 and k_codes.shape == v_codes.shape and _strides(k_codes) == _strides(v_codes),
                   "k_codes and v_codes: [B or pages, tokens, Hkv, d], the same sizes and strides")
        rows, tokens, hkv, d = k_codes.shape
        st, ss = _strides(k_codes), _strides(k_scales)
        self._need(st[3] == 1, "head_dim must be the contiguous dimension of the codes")
        self._need(k_scales.dim() == 3 and k_scales.shape == v_scales.shape and ss == _strides(v_scales) and ss[2] == 1
                   and k_scales.shape[:2] == (rows, hkv) and k_scales.shape[2] >= tokens,
                   "k_scales and v_scales: [B or pages, Hkv, tokens], tokens contiguous, the same sizes and strides")
        gamma = q_max - 1 if gamma is None else int(gamma)
        scale = d ** -0.5 if softmax_scale is None else float(softmax_scale)
        if page_table is None:
            ctx_max = tokens if max_ctx is None else int(max_ctx)
            self._need(rows == batch and ctx_max <= tokens, "the cache holds fewer sequences or tokens than the call names")
            self._need(k_scales.shape[2] >= -(-ctx_max // 16) * 16, "rows of scales: max_ctx rounded up to a multiple of 16")
            shape = AttnShape(batch, q_max, hq, hkv, d, ctx_max, gamma, scale, st[0], st[1], st[2], 0, 0, 0, 0, 0, 0)
            return ctypes.byref(shape), ctypes.byref(QuantLayout(ss[0], ss[1], 0))
        ctx_max = page_table.shape[1] * tokens if max_ctx is None else int(max_ctx)
        shape = AttnShape(batch, q_max, hq, hkv, d, ctx_max, gamma, scale, 0, st[1], st[2], st[0], tokens, page_table.shape[1], 0, rows, 0)
        return ctypes.byref(shape), ctypes.byref(QuantLayout(0, ss[1], ss[0]))

    _NO_WORKSPACE = (None, 0)

    def _capturing(self) -> bool:
        if torch.cuda.current_device() == self.device.index:
            return torch.cuda.is_current_stream_capturing()
        with torch.cuda.device(self.device):
            return torch.cuda.is_current_stream_capturing()

    def _stream_workspace(self, stream: int):
        # Address and size.  Eager calls of a stream share a workspace, so that calls on two may overlap; a captured call begins with none.
        # (The default stream is never captured.)
        return self._NO_WORKSPACE if stream and self._capturing() else self._ws_streams.get(stream, self._NO_WORKSPACE)

    def _new_workspace(self, stream: int, nbytes: int) -> torch.Tensor:
        # a captured call takes memory of its graph's, like any temporary tensor of a capture; a stream's own grows only
        if stream and self._capturing():
            return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        ws = torch.empty(max(nbytes, 2 * self._ws_streams.get(stream, self._NO_WORKSPACE)[1], 256), dtype=torch.uint8, device=self.device)
        self._ws_kept[stream], self._ws_streams[stream] = ws, (ws.data_ptr(), ws.numel())
        return ws

    def rapid_kv_append_quant(self, k_codes, v_codes, k_scales, v_scales, k_new, v_new, ctx_lens, gamma: Optional[int] = None, *,
                              gammas=None, page_table=None, max_ctx: Optional[int] = None):
        """Quantises rows 0..gamma_b of k_new/v_new (bf16 [B,Qmax,Hkv,d]) into the caches in place as the last gamma_b+1 tokens of
        every sequence (ctx_lens counts them).  k_codes/v_codes: float8_e4m3fn or uint8 [B,Lmax,Hkv,d] (any batch/token/head
        strides) or, with page_table, [n_pages,page,Hkv,d]; k_scales/v_scales: float8_e8m0fnu or uint8 [B,Hkv,Lmax] or
        [n_pages,Hkv,page], rows of a multiple of 16."""
        key = ("append", gamma, max_ctx, _sizes(k_codes, v_codes, k_scales, v_scales, k_new, v_new, ctx_lens, gammas, page_table))
        shape, layout = self._plans.get(key) or self._planned(
            key, self._plan_append, k_codes, v_codes, k_scales, v_scales, k_new, v_new, ctx_lens, gammas, page_table, gamma, max_ctx)
        rc = self.lib.rapid_kv_append_quant(self._ctx, shape, layout, k_new.data_ptr(), v_new.data_ptr(), ctx_lens.data_ptr(),
                                            _dptr(gammas), _dptr(page_table), k_codes.data_ptr(), v_codes.data_ptr(),
                                            k_scales.data_ptr(), v_scales.data_ptr(), _stream_ptr(self.device))
        if rc:
            _check(self.lib, rc, self._ctx)

    def _plan_append(self, k_codes, v_codes, k_scales, v_scales, k_new, v_new, ctx_lens, gammas, page_table, gamma, max_ctx):
        self._need(k_new.dim() == 4 and k_new.shape == v_new.shape and k_new.is_contiguous() and v_new.is_contiguous()
                   and k_new.dtype == torch.bfloat16 and v_new.dtype == torch.bfloat16,
                   "k_new and v_new: bf16 [B, Qmax, Hkv, d], contiguous")
        self._need(k_new.shape[2:] == k_codes.shape[2:], "k_new and the cache differ in heads or head_dim")
        self._check_lengths(k_new.shape[0], ctx_lens, gammas, page_table)
        return self._quant_shape(*k_new.shape[:3], gamma, k_codes, v_codes, k_scales, v_scales, page_table, max_ctx, 1.0)

    def rapid_kv_read_quant(self, k_codes, v_codes, k_scales, v_scales, ctx_lens, rows: int, gamma: Optional[int] = None, *,
                            gammas=None, page_table=None, max_ctx: Optional[int] = None, outs=None):
        """The last gamma_b+1 tokens of every sequence (gamma_b < rows) as bf16: (k, v) [B,rows,Hkv,d], zeros past a sequence's
        rows.  Cache as for :meth:`rapid_kv_append_quant`; `outs`: two tensors to write to."""
        if outs is None:
            shape = (ctx_lens.numel(), int(rows), *k_codes.shape[2:])
            outs = tuple(torch.empty(shape, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        k_out, v_out = outs
        key = ("read", rows, gamma, max_ctx, _sizes(k_codes, v_codes, k_scales, v_scales, k_out, v_out, ctx_lens, gammas, page_table))
        shape, layout = self._plans.get(key) or self._planned(
            key, self._plan_read, k_codes, v_codes, k_scales, v_scales, k_out, v_out, ctx_lens, gammas, page_table, rows, gamma, max_ctx)
        rc = self.lib.rapid_kv_read_quant(self._ctx, shape, layout, k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(),
                                          v_scales.data_ptr(), ctx_lens.data_ptr(), _dptr(gammas), _dptr(page_table),
                                          k_out.data_ptr(), v_out.data_ptr(), _stream_ptr(self.device))
        if rc:
            _check(self.lib, rc, self._ctx)
        return outs

    def _plan_read(self, k_codes, v_codes, k_scales, v_scales, k_out, v_out, ctx_lens, gammas, page_table, rows, gamma, max_ctx):
        batch, (hkv, d) = ctx_lens.numel(), k_codes.shape[2:]
        self._need(all(t.dtype == torch.bfloat16 and t.shape == (batch, rows, hkv, d) and t.is_contiguous() for t in (k_out, v_out)),
                   "outs: two of bf16 [B, rows, Hkv, d], contiguous")
        self._check_lengths(batch, ctx_lens, gammas, page_table)
        return self._quant_shape(batch, int(rows), hkv, gamma, k_codes, v_codes, k_scales, v_scales, page_table, max_ctx, 1.0)

    def rapid_verify_attn_quant(self, q, k_codes, v_codes, k_scales, v_scales, ctx_lens, gamma: Optional[int] = None, *, gammas=None,
                                page_table=None, max_ctx: Optional[int] = None, softmax_scale: Optional[float] = None,
                                out=None, lse_out=None):
        """:meth:`rapid_verify_attn` on a cache in 8 bits (layout: :meth:`rapid_kv_append_quant`): q bf16 [B,Qmax,Hq,d]; returns
        out bf16 [B,Qmax,Hq,d] and fills lse_out fp32 [B,Hq,Qmax] if given.  One position (Qmax = 1) is a decode step.
        Calls on different streams may overlap, and graphs (captured by torch.cuda.graph) may overlap with them and one another."""
        if out is None:
            out = torch.empty_like(q)

        key = ("attn", gamma, max_ctx, softmax_scale,
               _sizes(q, k_codes, v_codes, k_scales, v_scales, ctx_lens, gammas, page_table, out, lse_out))
        shape, layout = self._plans.get(key) or self._planned(key, self._plan_attn, q, k_codes, v_codes, k_scales, v_scales, ctx_lens, gammas,
                                                              page_table, out, lse_out, gamma, max_ctx, softmax_scale)
        args = (self._ctx, shape, layout, q.data_ptr(), k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(),
                v_scales.data_ptr(), ctx_lens.data_ptr(), _dptr(gammas), _dptr(page_table), out.data_ptr(), _dptr(lse_out))
        call, stream = self.lib.rapid_verify_attn_quant, _stream_ptr(self.device)
        rc = call(*args, *self._stream_workspace(stream), stream)
        if rc == RAPID_EWORKSPACE:                             # the last check of the call: nothing has been launched
            ws = self._new_workspace(stream, self.lib.rapid_verify_attn_quant_workspace_bytes(self._ctx, shape))
            rc = call(*args, ws.data_ptr(), ws.numel(), stream)
        if rc:
            _check(self.lib, rc, self._ctx)
        return out

    def _plan_attn(self, q, k_codes, v_codes, k_scales, v_scales, ctx_lens, gammas, page_table, out, lse_out, gamma, max_ctx, softmax_scale):
        self._check_attn(q, out, lse_out)
        self._need(q.shape[3] == k_codes.shape[3], "q and the cache differ in head_dim")
        self._check_lengths(q.shape[0], ctx_lens, gammas, page_table)
        return self._quant_shape(*q.shape[:3], gamma, k_codes, v_codes, k_scales, v_scales, page_table, max_ctx, softmax_scale)

    def rapid_verify_attn_prefix(self, q, k_cache, v_cache, ctx_lens, prefix_len, gamma: Optional[int] = None, *, k_prefix=None,
                                 v_prefix=None, prefix_table=None, max_prefix: Optional[int] = None, gammas=None, page_table=None,
                                 max_ctx: Optional[int] = None, softmax_scale: Optional[float] = None, out=None, lse_out=None):
        """:meth:`rapid_verify_attn` for a batch whose sequences follow one shared prefix, which is read once.  prefix_len int32
        [1] (device); the prefix is k_prefix/v_prefix bf16 [P,Hkv,d] (any token/head strides) or, with page_table, pages of
        k_cache/v_cache that prefix_table int32 [max_pages] names; max_prefix bounds prefix_len on the host (default: what is
        given).  ctx_lens counts a sequence's own tokens, which k_cache/v_cache hold as for rapid_verify_attn.  Streams
        and graphs as for :meth:`rapid_verify_attn_quant`."""
        if out is None:
            out = torch.empty_like(q)
        key = ("prefix", gamma, max_prefix, max_ctx, softmax_scale,
               _sizes(q, k_cache, v_cache, ctx_lens, prefix_len, k_prefix, v_prefix, prefix_table, gammas, page_table, out, lse_out))
        shape, prefix = self._plans.get(key) or self._planned(
            key, self._plan_prefix, q, k_cache, v_cache, ctx_lens, prefix_len, k_prefix, v_prefix, prefix_table, gammas, page_table, out,
            lse_out, gamma, max_prefix, max_ctx, softmax_scale)
        args = (self._ctx, shape, prefix, q.data_ptr(), _dptr(k_prefix), _dptr(v_prefix), prefix_len.data_ptr(), _dptr(prefix_table),
                k_cache.data_ptr(), v_cache.data_ptr(), ctx_lens.data_ptr(), _dptr(gammas), _dptr(page_table), out.data_ptr(),
                _dptr(lse_out))
        call, stream = self.lib.rapid_verify_attn_prefix, _stream_ptr(self.device)
        rc = call(*args, *self._stream_workspace(stream), stream)
        if rc == RAPID_EWORKSPACE:                             # the last check of the call: nothing has been launched
            ws = self._new_workspace(stream, self.lib.rapid_verify_attn_prefix_workspace_bytes(self._ctx, shape, prefix))
            rc = call(*args, ws.data_ptr(), ws.numel(), stream)
        if rc:
            _check(self.lib, rc, self._ctx)
        return out

    def _plan_prefix(self, q, k_cache, v_cache, ctx_lens, prefix_len, k_prefix, v_prefix, prefix_table, gammas, page_table, out, lse_out,
                     gamma, max_prefix, max_ctx, softmax_scale):
        self._check_attn(q, out, lse_out)
        self._check_lengths(q.shape[0], ctx_lens, gammas, page_table)
        self._check_cache(k_cache, v_cache)
        self._need(k_cache.shape[3] == q.shape[3], "q and the cache differ in head_dim")
        self._need(prefix_len.dtype == torch.int32 and prefix_len.numel() == 1, "prefix_len: int32 [1]")
        tokens, hkv, d = k_cache.shape[1:]
        scale = d ** -0.5 if softmax_scale is None else float(softmax_scale)
        shape = self._cache_shape(*q.shape[:3], k_cache, gamma, page_table, max_ctx, scale)
        if prefix_table is not None:
            self._need(page_table is not None and k_prefix is None and v_prefix is None,
                       "prefix_table names pages of a paged cache, in the place of k_prefix and v_prefix")
            self._need(prefix_table.dtype == torch.int32 and prefix_table.dim() == 1 and prefix_table.is_contiguous(),
                       "prefix_table: int32 [max_pages], contiguous")
            n = prefix_table.numel()
            return ctypes.byref(shape), ctypes.byref(PrefixLayout(n * tokens if max_prefix is None else int(max_prefix), n, 0, 0))
        self._need(k_prefix is not None and v_prefix is not None and k_prefix.dtype == torch.bfloat16
                   and v_prefix.dtype == torch.bfloat16 and k_prefix.dim() == 3 and k_prefix.shape == v_prefix.shape
                   and k_prefix.shape[1:] == (hkv, d), "k_prefix and v_prefix: bf16 [P, Hkv, d] as the cache's, the same sizes and strides")
        sp = _strides(k_prefix[None])
        self._need(sp == _strides(v_prefix[None]) and sp[3] == 1, "k_prefix and v_prefix: d contiguous, the same strides")
        n = k_prefix.shape[0]
        self._need(max_prefix is None or max_prefix <= n, "the prefix holds fewer tokens than max_prefix")
        return ctypes.byref(shape), ctypes.byref(PrefixLayout(n if max_prefix is None else int(max_prefix), 0, sp[1], sp[2]))

    # ------------------------------------------------------------------ a window
    def rapid_verify_attn_window(self, q, k_cache, v_cache, ctx_lens, window: int, gamma: Optional[int] = None, *, sinks: int = 0,
                                 gammas=None, page_table=None, max_ctx: Optional[int] = None, softmax_scale: Optional[float] = None,
                                 out=None, lse_out=None):
        """:meth:`rapid_verify_attn` where a row attends the last `window` keys up to its own, and the first `sinks`.  q bf16 [B,Qmax,Hq,d]
        of any Qmax: one position, a round's, a whole prompt or a piece of one.  Streams and graphs as for
        :meth:`rapid_verify_attn_quant`."""
        if out is None:
            out = torch.empty_like(q)
        key = ("window", gamma, window, sinks, max_ctx, softmax_scale,
               _sizes(q, k_cache, v_cache, ctx_lens, gammas, page_table, out, lse_out))
        shape, window, sinks = self._plans.get(key) or self._planned(
            key, self._plan_window, q, k_cache, v_cache, ctx_lens, gammas, page_table, out, lse_out, gamma, window, sinks, max_ctx, softmax_scale)
        args = (self._ctx, shape, window, sinks, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), ctx_lens.data_ptr(), _dptr(gammas),
                _dptr(page_table), out.data_ptr(), _dptr(lse_out))
        call, stream = self.lib.rapid_verify_attn_window, _stream_ptr(self.device)
        rc = call(*args, *self._stream_workspace(stream), stream)
        if rc == RAPID_EWORKSPACE:                             # the last check of the call: nothing has been launched
            ws = self._new_workspace(stream, self.lib.rapid_verify_attn_window_workspace_bytes(self._ctx, shape, window, sinks))
            rc = call(*args, ws.data_ptr(), ws.numel(), stream)
        if rc:
            _check(self.lib, rc, self._ctx)
        return out

    def _plan_window(self, q, k_cache, v_cache, ctx_lens, gammas, page_table, out, lse_out, gamma, window, sinks, max_ctx, softmax_scale):
        self._check_attn(q, out, lse_out)
        self._check_lengths(q.shape[0], ctx_lens, gammas, page_table)
        self._check_cache(k_cache, v_cache)
        self._need(k_cache.shape[3] == q.shape[3], "q and the cache differ in head_dim")
        self._need(int(window) == window and int(sinks) == sinks, "window and sinks are whole numbers")
        scale = q.shape[3] ** -0.5 if softmax_scale is None else float(softmax_scale)
        most = (1 << 31) - 1                                   # of a C int; more is all there is
        return ctypes.byref(self._cache_shape(*q.shape[:3], k_cache, gamma, page_table, max_ctx, scale)), min(int(window), most), min(int(sinks), most)

    # ------------------------------------------------------------------ append with rotary positions
    def rapid_kv_append_rope(self, k_cache, v_cache, k_new, v_new, inv_freq, ctx_lens, gamma: Optional[int] = None, *, q_new=None,
                             q_out=None, positions=None, interleaved: bool = False, amplitude: float = 1.0, gammas=None, page_table=None,
                             max_ctx: Optional[int] = None):
        """:meth:`rapid_kv_append` with the rotary positions on the way: rows 0..gamma_b of k_new (rotated) and v_new become the last
        gamma_b+1 tokens of every sequence; the same rows of q_new, rotated, are written to q_out, which is returned (bf16
        [B,Qmax,Hq,d]; made here where q_new is given and q_out is not; may be q_new).  q_new/k_new/v_new: bf16 [B,Qmax,heads,d],
        heads side by side, rows any distance apart, so that they may be slices of one projection's output.  inv_freq: fp32
        [rotary_dim/2]; positions: int32 [B,Qmax], by default a row's token.  Cache layout as for rapid_verify_attn."""
        if q_out is None and q_new is not None:
            q_out = torch.empty(q_new.shape, dtype=torch.bfloat16, device=self.device)
        key = ("rope", gamma, max_ctx, interleaved, amplitude,
               _sizes(k_cache, v_cache, k_new, v_new, inv_freq, ctx_lens, q_new, q_out, positions, gammas, page_table))
        shape, rope = self._plans.get(key) or self._planned(
            key, self._plan_rope, k_cache, v_cache, None, None, k_new, v_new, inv_freq, ctx_lens, q_new, q_out, positions, gammas, page_table,
            gamma, max_ctx, interleaved, amplitude)
        rc = self.lib.rapid_kv_append_rope(self._ctx, shape, rope, _dptr(q_new), k_new.data_ptr(), v_new.data_ptr(), inv_freq.data_ptr(),
                                           _dptr(positions), ctx_lens.data_ptr(), _dptr(gammas), _dptr(page_table), _dptr(q_out),
                                           k_cache.data_ptr(), v_cache.data_ptr(), _stream_ptr(self.device))
        if rc:
            _check(self.lib, rc, self._ctx)
        return q_out

    def rapid_kv_append_rope_quant(self, k_codes, v_codes, k_scales, v_scales, k_new, v_new, inv_freq, ctx_lens,
                                   gamma: Optional[int] = None, *, q_new=None, q_out=None, positions=None, interleaved: bool = False,
                                   amplitude: float = 1.0, gammas=None, page_table=None, max_ctx: Optional[int] = None):
        """:meth:`rapid_kv_append_rope` into a cache in 8 bits (layout: :meth:`rapid_kv_append_quant`)."""
        if q_out is None and q_new is not None:
            q_out = torch.empty(q_new.shape, dtype=torch.bfloat16, device=self.device)
        key = ("rope_quant", gamma, max_ctx, interleaved, amplitude,
               _sizes(k_codes, v_codes, k_scales, v_scales, k_new, v_new, inv_freq, ctx_lens, q_new, q_out, positions, gammas, page_table))
        shape, layout, rope = self._plans.get(key) or self._planned(
            key, self._plan_rope, k_codes, v_codes, k_scales, v_scales, k_new, v_new, inv_freq, ctx_lens, q_new, q_out, positions, gammas,
            page_table, gamma, max_ctx, interleaved, amplitude)
        rc = self.lib.rapid_kv_append_rope_quant(self._ctx, shape, layout, rope, _dptr(q_new), k_new.data_ptr(), v_new.data_ptr(),
                                                 inv_freq.data_ptr(), _dptr(positions), ctx_lens.data_ptr(), _dptr(gammas), _dptr(page_table),
                                                 _dptr(q_out), k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(),
                                                 v_scales.data_ptr(), _stream_ptr(self.device))
        if rc:
            _check(self.lib, rc, self._ctx)
        return q_out

    def _row_stride(self, t, name: str) -> int:
        """Elements from one row (sequence, position) of t [B, Qmax, heads, d] to the next."""
        B, Q, heads, d = t.shape
        s0, s1, s2, s3 = t.stride()
        row = s1 if Q > 1 else s0 if B > 1 else heads * d
        self._need((s3 == 1 or d == 1) and (s2 == d or heads == 1) and (Q == 1 or B == 1 or s0 == Q * s1),
                   f"{name}: heads side by side, rows the same distance apart")
        return row

    def _plan_rope(self, k_cache, v_cache, k_scales, v_scales, k_new, v_new, inv_freq, ctx_lens, q_new, q_out, positions, gammas, page_table,
                   gamma, max_ctx, interleaved, amplitude):
        news = [(t, name) for t, name in ((q_new, "q_new"), (k_new, "k_new"), (v_new, "v_new")) if t is not None]
        self._need(all(t.dtype == torch.bfloat16 and t.dim() == 4 for t, _ in news), "q_new, k_new and v_new: bf16 [B, Qmax, heads, d]")
        B, Q, hkv, d = k_new.shape
        self._need(v_new.shape == k_new.shape and k_cache.dim() == 4 and k_cache.shape[2:] == k_new.shape[2:],
                   "k_new, v_new and the cache differ in heads or head_dim")
        self._need(inv_freq.dtype == torch.float32 and inv_freq.dim() == 1 and inv_freq.is_contiguous(), "inv_freq: fp32 [rotary_dim / 2]")
        self._need(positions is None or (positions.dtype == torch.int32 and positions.shape == (B, Q) and positions.is_contiguous()),
                   "positions: int32 [B, Qmax], contiguous")
        self._need((q_new is None) == (q_out is None), "q_out goes with q_new")
        hq = hkv
        if q_new is not None:
            hq = q_new.shape[2]
            self._need(q_new.shape == (B, Q, hq, d), "q_new: as many sequences, positions and elements a head as k_new")
            self._need(q_out.dtype == torch.bfloat16 and q_out.shape == q_new.shape and q_out.is_contiguous(), "q_out: bf16 like q_new, contiguous")
        self._check_lengths(B, ctx_lens, gammas, page_table)
        strides = [self._row_stride(t, name) for t, name in news]
        rope = Rope(2 * inv_freq.numel(), int(bool(interleaved)), float(amplitude), *([0] if q_new is None else []), *strides)
        if k_scales is not None:
            return (*self._quant_shape(B, Q, hq, gamma, k_cache, v_cache, k_scales, v_scales, page_table, max_ctx, 1.0), ctypes.byref(rope))
        self._check_cache(k_cache, v_cache)
        return ctypes.byref(self._cache_shape(B, Q, hq, k_cache, gamma, page_table, max_ctx, 1.0)), ctypes.byref(rope)

    def _cache_shape(self, batch, q_max, hq, k_cache, gamma, page_table, max_ctx, scale) -> AttnShape:
        """Of a bf16 cache [B or pages, tokens, Hkv, d]."""
        (rows, tokens, hkv, d), st = k_cache.shape, _strides(k_cache)
        gamma = q_max - 1 if gamma is None else int(gamma)
        if page_table is None:
            ctx_max = tokens if max_ctx is None else int(max_ctx)
            self._need(rows == batch and ctx_max <= tokens, "the cache holds fewer sequences or tokens than the call names")
            return AttnShape(batch, q_max, hq, hkv, d, ctx_max, gamma, scale, st[0], st[1], st[2], 0, 0, 0, 0, 0, 0)
        ctx_max = page_table.shape[1] * tokens if max_ctx is None else int(max_ctx)
        return AttnShape(batch, q_max, hq, hkv, d, ctx_max, gamma, scale, 0, st[1], st[2], st[0], tokens, page_table.shape[1], 0, rows, 0)

    # ------------------------------------------------------------------ retrieval
    def rapid_retrieve(self, chunk_emb, query_emb, top_k: int, threshold: float = 0.3):
        """chunk_emb fp32 [n, dim], query_emb fp32 [dim] -> (similarity fp32 [n], selected int32 [top_k]
        (document order, then -1), n_selected int32 [1]); all on the device."""
        n, dim = chunk_emb.shape
        assert chunk_emb.dtype == torch.float32 and chunk_emb.is_contiguous()
        assert query_emb.dtype == torch.float32 and query_emb.is_contiguous() and query_emb.shape == (dim,)
        sim = torch.empty(n, dtype=torch.float32, device=self.device)
        sel = torch.empty(max(int(top_k), 1), dtype=torch.int32, device=self.device)
        cnt = torch.empty(1, dtype=torch.int32, device=self.device)
        rc = self.lib.rapid_retrieve(self._ctx, n, dim, _dptr(chunk_emb), _dptr(query_emb), int(top_k),
                                     float(threshold), _dptr(sim), _dptr(sel), _dptr(cnt), _stream_ptr(self.device))
        _check(self.lib, rc, self._ctx)
        return sim, sel, cnt

    # ------------------------------------------------------------------ output head
    def lm_head_chunk(self, vocab: int, n_rows: int = 1) -> int:
        """Vocabulary entries per statistics chunk that rapid_lm_head uses for this vocabulary and row count."""
        return self.lib.rapid_lm_head_chunk(self._ctx, int(vocab), int(n_rows))

    def rapid_lm_head(self, h, w, *, temperature: float = 1.0, want_stats: bool = True, logits=None, stats=None):
        """h bf16 [rows, hidden], w bf16 [vocab, hidden] -> (logits fp32 [rows, vocab],
        stats fp32 [rows, chunks, 2] or None); chunk size: :meth:`lm_head_chunk`."""
        rows, hidden = h.shape
        vocab = w.shape[0]
        assert h.dtype == torch.bfloat16 and w.dtype == torch.bfloat16 and h.is_contiguous() and w.is_contiguous()
        assert w.shape[1] == hidden
        if logits is None:
            logits = torch.empty(rows, vocab, dtype=torch.float32, device=self.device)
        assert logits.dtype == torch.float32 and logits.stride(-1) == 1 and logits.shape == (rows, vocab)
        if want_stats and stats is None:
            stats = torch.empty(rows, self.lib.rapid_lm_head_stat_chunks(self._ctx, vocab, rows), 2, dtype=torch.float32,
                                device=self.device)
        rc = self.lib.rapid_lm_head(self._ctx, rows, hidden, vocab, _dptr(h), _dptr(w), float(temperature),
                                    _dptr(logits), logits.stride(0) if rows > 1 else vocab,
                                    _dptr(stats) if want_stats else None, _stream_ptr(self.device))
        _check(self.lib, rc, self._ctx)
        return logits, (stats if want_stats else None)

    def rapid_quant_rows(self, x, codes=None, scales=None):
        """Rows of x (bf16 [rows, cols], any row stride) as 8-bit integers: (codes int8 [rows, pitch], scales fp32 [rows]), pitch = cols
        rounded up to a multiple of 256 (zeros behind the row): what :meth:`rapid_lm_head_quant` takes for an output embedding."""
        if codes is None or scales is None:
            self._need(x.dim() == 2, "x: bf16 [rows, cols], cols contiguous")
            codes = torch.empty((x.shape[0], -(-x.shape[1] // 256) * 256), dtype=torch.int8, device=self.device) if codes is None else codes
            scales = torch.empty(x.shape[0], dtype=torch.float32, device=self.device) if scales is None else scales
        key = ("rows", _sizes(x, codes, scales))
        rows, cols, stride = self._plans.get(key) or self._planned(key, self._plan_rows, x, codes, scales)
        rc = self.lib.rapid_quant_rows(self._ctx, rows, cols, x.data_ptr(), stride, codes.data_ptr(), scales.data_ptr(),
                                       _stream_ptr(self.device))
        if rc:
            _check(self.lib, rc, self._ctx)
        return codes, scales

    def _plan_rows(self, x, codes, scales):
        self._need(x.dim() == 2 and x.dtype == torch.bfloat16 and (x.stride(1) == 1 or x.shape[1] == 1), "x: bf16 [rows, cols], cols contiguous")
        rows, cols = x.shape
        self._need(codes.dtype == torch.int8 and codes.shape == (rows, -(-cols // 256) * 256) and codes.is_contiguous(),
                   "codes: int8 [rows, cols rounded up to a multiple of 256], contiguous")
        self._need(scales.dtype == torch.float32 and scales.shape == (rows,) and scales.is_contiguous(), "scales: fp32 [rows], contiguous")
        return rows, cols, x.stride(0) if rows > 1 else cols

    def rapid_lm_head_quant(self, h, w_codes, w_scales, *, temperature: float = 1.0, want_stats: bool = True, logits=None, stats=None):
        """:meth:`rapid_lm_head` on an output embedding in 8-bit integers (:meth:`rapid_quant_rows` of it): h bf16 [rows, hidden], w_codes
        int8 [vocab, pitch], w_scales fp32 [vocab] -> (logits fp32 [rows, vocab], stats fp32 [rows, chunks, 2] or None).  Streams and
        graphs as for :meth:`rapid_verify_attn_quant`."""
        self._need(h.dim() == 2 and w_codes.dim() == 2, "h [rows, hidden], w_codes [vocab, pitch]")
        (rows, hidden), (vocab, pitch) = h.shape, w_codes.shape
        if logits is None:
            logits = torch.empty((rows, vocab), dtype=torch.float32, device=self.device)
        if not want_stats:
            stats = None
        elif stats is None:
            stats = torch.empty((rows, self.lib.rapid_lm_head_stat_chunks(self._ctx, vocab, rows), 2), dtype=torch.float32,
                                device=self.device)
        key = ("head", _sizes(h, w_codes, w_scales, logits, stats))
        ldz = self._plans.get(key) or self._planned(key, self._plan_head, h, w_codes, w_scales, logits, stats)
        args = (self._ctx, rows, hidden, vocab, h.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(), float(temperature), logits.data_ptr(),
                ldz, _dptr(stats))
        call, stream = self.lib.rapid_lm_head_quant, _stream_ptr(self.device)
        rc = call(*args, *self._stream_workspace(stream), stream)
        if rc == RAPID_EWORKSPACE:                             # the last check of the call: nothing has been launched
            ws = self._new_workspace(stream, self.lib.rapid_lm_head_quant_workspace_bytes(self._ctx, rows, hidden))
            rc = call(*args, ws.data_ptr(), ws.numel(), stream)
        if rc:
            _check(self.lib, rc, self._ctx)
        return logits, stats

    def _plan_head(self, h, w_codes, w_scales, logits, stats):
        """The distance of the logits' rows."""
        (rows, hidden), (vocab, pitch) = h.shape, w_codes.shape
        self._need(h.dtype == torch.bfloat16 and h.is_contiguous(), "h: bf16 [rows, hidden], contiguous")
        self._need(w_codes.dtype == torch.int8 and w_codes.is_contiguous() and pitch == -(-hidden // 256) * 256,
                   "w_codes: int8 [vocab, hidden rounded up to a multiple of 256], contiguous")
        self._need(w_scales.dtype == torch.float32 and w_scales.shape == (vocab,) and w_scales.is_contiguous(), "w_scales: fp32 [vocab], contiguous")
        self._need(logits.dtype == torch.float32 and logits.shape == (rows, vocab) and (logits.stride(1) == 1 or vocab == 1),
                   "logits: fp32 [rows, vocab], vocab contiguous")
        self._need(stats is None or (stats.dtype == torch.float32 and stats.is_contiguous() and
                                     stats.shape == (rows, self.lib.rapid_lm_head_stat_chunks(self._ctx, vocab, rows), 2)),
                   "stats: fp32 [rows, chunks, 2], contiguous")
        return logits.stride(0) if rows > 1 else vocab

    # ------------------------------------------------------------------ measurement aid
    def rapid_hbm_read_probe(self, buf: torch.Tensor, nbytes: Optional[int] = None):
        """Streams the first `nbytes` bytes (default: all, rounded down to 16 KiB) of a dense tensor's
        memory through the attention kernel's load path; for timing only."""
        total = buf.numel() * buf.element_size()
        nbytes = (total if nbytes is None else nbytes) // 16384 * 16384
        if self._sink is None:
            self._sink = torch.zeros(1, dtype=torch.int32, device=self.device)
        _check(self.lib, self.lib.rapid_hbm_read_probe(self._ctx, _dptr(buf), nbytes, _dptr(self._sink),
                                                       _stream_ptr(self.device)), self._ctx)
        return nbytes


_default: dict = {}

def _get(device: int = 0) -> Rapid:
    if device not in _default:
        _default[device] = Rapid(device)
    return _default[device]


def rapid_verify_attn(q, k_cache, v_cache, ctx_lens, gamma=None, **kw):
    """Module-level form of :meth:`Rapid.rapid_verify_attn` on the tensors' device."""
    return _get(q.device.index or 0).rapid_verify_attn(q, k_cache, v_cache, ctx_lens, gamma, **kw)


def rapid_lm_head(h, w, **kw):
    """Module-level form of :meth:`Rapid.rapid_lm_head` on the tensors' device."""
    return _get(h.device.index or 0).rapid_lm_head(h, w, **kw)


def rapid_accept(target_logits, draft_logits, draft_tokens, eta, uniforms, **kw):
    """Module-level form of :meth:`Rapid.rapid_accept` on the tensors' device."""
    return _get(target_logits.device.index or 0).rapid_accept(target_logits, draft_logits, draft_tokens, eta,
                                                              uniforms, **kw)


def rapid_verify_attn_quant(q, k_codes, v_codes, k_scales, v_scales, ctx_lens, gamma=None, **kw):
    """Module-level form of :meth:`Rapid.rapid_verify_attn_quant` on the tensors' device."""
    return _get(q.device.index or 0).rapid_verify_attn_quant(q, k_codes, v_codes, k_scales, v_scales, ctx_lens, gamma, **kw)


def rapid_verify_attn_prefix(q, k_cache, v_cache, ctx_lens, prefix_len, gamma=None, **kw):
    """Module-level form of :meth:`Rapid.rapid_verify_attn_prefix` on the tensors' device."""
    return _get(q.device.index or 0).rapid_verify_attn_prefix(q, k_cache, v_cache, ctx_lens, prefix_len, gamma, **kw)


def rapid_lm_head_quant(h, w_codes, w_scales, **kw):
    """Module-level form of :meth:`Rapid.rapid_lm_head_quant` on the tensors' device."""
    return _get(h.device.index or 0).rapid_lm_head_quant(h, w_codes, w_scales, **kw)


def rapid_verify_attn_window(q, k_cache, v_cache, ctx_lens, window, gamma=None, **kw):
    """Module-level form of :meth:`Rapid.rapid_verify_attn_window` on the tensors' device."""
    return _get(q.device.index or 0).rapid_verify_attn_window(q, k_cache, v_cache, ctx_lens, window, gamma, **kw)
