"""The quantised KV cache: e4m3 values in blocks of 32 with a power-of-two scale each, half the bytes of
the bf16 cache (include/unstep.h has the number format)."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import HEAD_DIM, Cache, _calls_mx8, _check, _need, _ptr, _stream, _used_on, _vp, lib
from .rotary import layout_code, norm_weights, table_rot

E4M3 = torch.float8_e4m3fn
SCALES = HEAD_DIM // 32


class CacheMX8:
    """KV cache of one attention layer: device buffers k8, v8 (e4m3 [B, H, (S+R)*T, 128]) and k_scale,
    v_scale (uint8 [B, H, (S+R)*T, 4], the power of two 2^(byte - 127) of each block of 32) owned by this
    object, host-held positions owned by the library handle.  The index calls are those of Cache."""

    def __init__(self, batch: int, n_heads: int, grid_h: int, grid_w: int, sink_frames: int, ring_frames: int,
                 device="cuda", k8: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None,
                 v8: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, head_dim: int = HEAD_DIM):
        self.B, self.H, self.grid_h, self.grid_w = batch, n_heads, grid_h, grid_w
        self.S, self.R = sink_frames, ring_frames
        self.T = grid_h * grid_w
        self.slots = (sink_frames + ring_frames) * self.T
        shape, scales = (batch, n_heads, self.slots, head_dim), (batch, n_heads, self.slots, SCALES)
        given = next((t for t in (k8, k_scale, v8, v_scale) if t is not None), None)
        where = given.device if given is not None else device
        make = lambda t, s, dt: torch.zeros(s, dtype=torch.uint8, device=where).view(dt) if t is None else t  # noqa: E731
        self.k8, self.v8 = make(k8, shape, E4M3), make(v8, shape, E4M3)
        self.k_scale, self.v_scale = (make(t, scales, torch.uint8) for t in (k_scale, v_scale))
        self.device = self.k8.device
        for t, name, s, dt in ((self.k8, "k8", shape, E4M3), (self.v8, "v8", shape, E4M3),
                               (self.k_scale, "k_scale", scales, torch.uint8),
                               (self.v_scale, "v_scale", scales, torch.uint8)):
            _need(t, name, s, dt, self.device)
        h = _vp()
        _check(lib.unstep_cache_create_mx8(ctypes.byref(h), batch, n_heads, head_dim, grid_h, grid_w, sink_frames,
                                           ring_frames, self.k8.data_ptr(), self.k_scale.data_ptr(),
                                           self.v8.data_ptr(), self.v_scale.data_ptr()))
        self.handle = h
        self._ws: Optional[torch.Tensor] = None
        # the native calls' view of this cache; None: not on a GPU, or a subclass with its own checks or outputs
        self._native = None
        if all(getattr(type(self), f.__name__) is f for f in _CHECK_METHODS):
            self._native = _calls_mx8.cache(h.value, self.B, self.H, self.T, self.k8, _SCRATCH_METHODS)

    def __del__(self, _destroy=lib.unstep_cache_destroy):
        self._native = None                # it holds the handle's address
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            _destroy(h)
            self.handle = None

    # -- host index state and checks: those of Cache ----------------------------------
    frame_map = Cache.frame_map
    advance = Cache.advance
    segments = Cache.segments
    workspace_bytes = Cache.workspace_bytes
    _strides = Cache._strides
    _qkv_strides = Cache._qkv_strides
    _chunk_out = Cache._chunk_out
    _lse = Cache._lse
    _workspace_bytes = Cache._workspace_bytes

    def workspace(self, start_frame: int, n_frames: int, window_frames: int) -> Optional[torch.Tensor]:
        """Device scratch for split-key attention, grown on demand and kept; while a graph is captured a new one, which
        the graph's memory pool holds: the kept one may be replaced, or in use elsewhere, when the graph is replayed.
        Calls that may overlap otherwise (two streams) need a workspace argument each."""
        need = self.workspace_bytes(start_frame, n_frames, window_frames)
        if need == 0:
            return None
        if self.device.type == "cuda" and torch.cuda.is_current_stream_capturing():
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws

    def _queries(self, q8, q_scale, n_frames: int, make: bool) -> Tuple[torch.Tensor, torch.Tensor]:
        """Quantised queries [B, N, H, 128] and their scales [B, N, H, 4], checked, or (make) new ones."""
        head = (self.B, n_frames * self.T, self.H)
        if make and q8 is None:
            q8 = torch.empty(head + (HEAD_DIM,), dtype=E4M3, device=self.device)
        if make and q_scale is None:
            q_scale = torch.empty(head + (SCALES,), dtype=torch.uint8, device=self.device)
        _need(q8, "q8", head + (HEAD_DIM,), E4M3, self.device)
        _need(q_scale, "q_scale", head + (SCALES,), torch.uint8, self.device)
        return q8, q_scale

    # -- step path ----------------------------------------------------------------------
    def unstep_kv_append_mx8(self, start_frame: int, n_frames: int, q: Optional[torch.Tensor], k: torch.Tensor,
                             v: torch.Tensor, cos_t: torch.Tensor, sin_t: torch.Tensor, layout: str = "interleaved",
                             q_norm_weight: Optional[torch.Tensor] = None, k_norm_weight: Optional[torch.Tensor] = None,
                             norm_eps: float = 1e-6, softmax_scale: float = 0.0, q8: Optional[torch.Tensor] = None,
                             q_scale: Optional[torch.Tensor] = None,
                             stream=None) -> Optional[Tuple[torch.Tensor, torch.Tensor]]:
        """Rotate and quantise the chunk's keys and values into the cache; returns the quantised queries
        (q8, q_scale), which hold the softmax scale, or None without q."""
        if stream is None and self._native is not None:
            r = _calls_mx8.append_mx8(self._native, start_frame, n_frames, q, k, v, cos_t, sin_t, layout, q_norm_weight,
                                      k_norm_weight, norm_eps, softmax_scale, q8, q_scale)
            if r is not None:
                return r[0]
        ts, hs = self._qkv_strides(q, k, v, n_frames)
        rot, code = table_rot(self, cos_t, sin_t, n_frames), layout_code(layout)
        norm_weights(self, q, q_norm_weight, k_norm_weight)
        if q is not None:
            q8, q_scale = self._queries(q8, q_scale, n_frames, True)
        with torch.cuda.device(self.device):
            _check(lib.unstep_kv_append_mx8(self.handle, start_frame, n_frames, _ptr(q), k.data_ptr(), v.data_ptr(), ts,
                                            hs, cos_t.data_ptr(), sin_t.data_ptr(), code, rot, _ptr(q_norm_weight),
                                            _ptr(k_norm_weight), norm_eps, softmax_scale, _ptr(q8), _ptr(q_scale),
                                            _stream(stream)))
            _used_on(stream, q8, q_scale)
        return None if q is None else (q8, q_scale)

    def unstep_window_attn_mx8(self, start_frame: int, n_frames: int, window_frames: int, q8: torch.Tensor,
                               q_scale: torch.Tensor, out: Optional[torch.Tensor] = None,
                               lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                               use_split: bool = True, stream=None) -> torch.Tensor:
        if stream is None and self._native is not None:
            r = _calls_mx8.window_attn_mx8(self._native, start_frame, n_frames, window_frames, q8, q_scale, out, lse,
                                           workspace, use_split, self)
            if r is not None:
                return r
        q8, q_scale = self._queries(q8, q_scale, n_frames, False)
        out = self._chunk_out(out, "out", n_frames)
        self._lse(lse, n_frames)
        if workspace is None and use_split:
            workspace = self.workspace(start_frame, n_frames, window_frames)
        with torch.cuda.device(self.device):
            _check(lib.unstep_window_attn_mx8(self.handle, start_frame, n_frames, window_frames, q8.data_ptr(),
                                              q_scale.data_ptr(), out.data_ptr(), _ptr(lse), _ptr(workspace),
                                              self._workspace_bytes(workspace), _stream(stream)))
            _used_on(stream, out, workspace)
        return out

    def unstep_step_mx8(self, start_frame: int, n_frames: int, window_frames: int, q: torch.Tensor, k: torch.Tensor,
                        v: torch.Tensor, cos_t: torch.Tensor, sin_t: torch.Tensor, layout: str = "interleaved",
                        q_norm_weight: Optional[torch.Tensor] = None, k_norm_weight: Optional[torch.Tensor] = None,
                        norm_eps: float = 1e-6, softmax_scale: float = 0.0, q8: Optional[torch.Tensor] = None,
                        q_scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        use_split: bool = True, stream=None) -> torch.Tensor:
        """unstep_kv_append_mx8 and unstep_window_attn_mx8 in one call."""
        if stream is None and self._native is not None:
            r = _calls_mx8.step_mx8(self._native, start_frame, n_frames, q, k, v, cos_t, sin_t, window_frames, layout,
                                    q_norm_weight, k_norm_weight, norm_eps, softmax_scale, q8, q_scale, out, lse, workspace,
                                    use_split, self)
            if r is not None:
                return r
        if q is None:
            raise ValueError("unstep_step_mx8 needs q")
        ts, hs = self._qkv_strides(q, k, v, n_frames)
        rot, code = table_rot(self, cos_t, sin_t, n_frames), layout_code(layout)
        norm_weights(self, q, q_norm_weight, k_norm_weight)
        q8, q_scale = self._queries(q8, q_scale, n_frames, True)
        out = self._chunk_out(out, "out", n_frames)
        self._lse(lse, n_frames)
        if workspace is None and use_split:
            workspace = self.workspace(start_frame, n_frames, window_frames)
        with torch.cuda.device(self.device):
            _check(lib.unstep_step_mx8(self.handle, start_frame, n_frames, window_frames, q.data_ptr(), k.data_ptr(),
                                       v.data_ptr(), ts, hs, cos_t.data_ptr(), sin_t.data_ptr(), code, rot,
                                       _ptr(q_norm_weight), _ptr(k_norm_weight), norm_eps, softmax_scale, q8.data_ptr(),
                                       q_scale.data_ptr(), out.data_ptr(), _ptr(lse), _ptr(workspace),
                                       self._workspace_bytes(workspace), _stream(stream)))
            _used_on(stream, q8, q_scale, out, workspace)
        return out

    def unstep_kv_read_mx8(self, start_frame: int, n_frames: int, k_out: Optional[torch.Tensor] = None,
                           v_out: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The frames' rotated keys and values as bf16 [B, N, H, 128], exact."""
        if stream is None and self._native is not None:
            r = _calls_mx8.read_mx8(self._native, start_frame, n_frames, k_out, v_out)
            if r is not None:
                return r
        n = max(0, n_frames)
        k_out, v_out = self._chunk_out(k_out, "k_out", n), self._chunk_out(v_out, "v_out", n)
        with torch.cuda.device(self.device):
            _check(lib.unstep_kv_read_mx8(self.handle, start_frame, n_frames, k_out.data_ptr(), v_out.data_ptr(),
                                          _stream(stream)))
            _used_on(stream, k_out, v_out)
        return k_out, v_out


_CHECK_METHODS = (CacheMX8._strides, CacheMX8._qkv_strides, CacheMX8._chunk_out, CacheMX8._lse, CacheMX8._workspace_bytes,
                  CacheMX8._queries)
_SCRATCH_METHODS = (CacheMX8.workspace, CacheMX8.workspace_bytes, CacheMX8.workspace)


def unstep_mx8_dequantize(x8: torch.Tensor, scale: torch.Tensor, out: Optional[torch.Tensor] = None,
                          stream=None) -> torch.Tensor:
    """bf16 values of quantised rows x8 [..., 128] (e4m3) with scale bytes [..., 4], exact for what the
    quantising append writes."""
    if stream is None:
        r = _calls_mx8.dequantize(x8, scale, out)
        if r is not None:
            return r
    if x8.dim() < 1 or x8.shape[-1] != HEAD_DIM:
        raise ValueError("x8 must have shape [..., 128]")
    _need(x8, "x8", tuple(x8.shape), E4M3, x8.device)
    _need(scale, "scale", tuple(x8.shape[:-1]) + (SCALES,), torch.uint8, x8.device)
    if out is None:
        out = torch.empty(x8.shape, dtype=torch.bfloat16, device=x8.device)
    _need(out, "out", tuple(x8.shape), torch.bfloat16, x8.device)
    if x8.numel() == 0:
        return out
    with torch.cuda.device(x8.device):
        _check(lib.unstep_mx8_dequantize(x8.data_ptr(), scale.data_ptr(), out.data_ptr(), x8.numel() // HEAD_DIM,
                                         _stream(stream)))
        _used_on(stream, out)
    return out
