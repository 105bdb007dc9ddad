"""Rotary options: tables with the caller's split of the pairs over (frame, row, column) and a scaled
frame axis, and the append that rotates in either layout over a part of the head."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import HEAD_DIM, _calls_mx8, _check, _need, _ptr, _stream, _used_on, lib

ROTARY_LAYOUTS = {"interleaved": 0, "half": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}


class _Rotary(ctypes.Structure):
    _fields_ = [("dim_t", ctypes.c_int32), ("dim_h", ctypes.c_int32), ("dim_w", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("theta", ctypes.c_double), ("factor", ctypes.c_double),
                ("trained_frames", ctypes.c_double), ("turns_fast", ctypes.c_double), ("turns_slow", ctypes.c_double),
                ("amplitude", ctypes.c_double)]


def unstep_rotary_tables(start_frame: int, n_frames: int, grid_h: int, grid_w: int,
                         dims: Tuple[int, int, int] = (44, 42, 42), theta: float = 10000.0, scaling: str = "none",
                         factor: float = 1.0, trained_frames: float = 0.0, turns: Tuple[float, float] = (32.0, 1.0),
                         amplitude: float = 0.0, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None,
                         device="cuda", stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Device cos/sin tables [N, sum(dims) / 2] float32, computed on the stream (nothing is uploaded or
    waited for).  dims: the dimensions of a head turned by the frame, the row and the column; scaling: none,
    linear, base or parts (unstep_rotary_scaling in include/unstep.h); turns: the parts' (fast, slow) bounds;
    out: tables to fill."""
    if scaling not in ROTARY_SCALINGS:
        raise ValueError(f"unknown scaling {scaling!r}")
    d_t, d_h, d_w = dims
    if out is None and stream is None and device == "cuda" and torch.cuda.is_initialized():
        r = _calls_mx8.tables(start_frame, n_frames, grid_h, grid_w, d_t, d_h, d_w, theta, ROTARY_SCALINGS[scaling], factor,
                              trained_frames, *turns, amplitude)
        if r is not None:
            return r
    opt = _Rotary(d_t, d_h, d_w, ROTARY_SCALINGS[scaling], theta, factor, trained_frames, turns[0], turns[1], amplitude)
    shape = (max(0, n_frames) * max(0, grid_h) * max(0, grid_w), max(0, sum(dims)) // 2)
    if out is None:
        both = torch.empty((2,) + shape, dtype=torch.float32, device=device)
        c, s = both.unbind(0)
    else:
        c, s = out
        for t, name in ((c, "cos"), (s, "sin")):
            _need(t, name, shape, torch.float32, c.device)
    with torch.cuda.device(c.device):
        _check(lib.unstep_rotary_tables(start_frame, n_frames, grid_h, grid_w, ctypes.addressof(opt), c.data_ptr(),
                                        s.data_ptr(), _stream(stream)))
        _used_on(stream, c, s)
    return c, s


def layout_code(layout: str) -> int:
    if layout not in ROTARY_LAYOUTS:
        raise ValueError(f"unknown layout {layout!r}")
    return ROTARY_LAYOUTS[layout]


def table_rot(cache, cos_t: torch.Tensor, sin_t: torch.Tensor, n_frames: int) -> int:
    """The rotated dimensions of tables [N, rot_dim / 2], checked."""
    if cos_t is None or cos_t.dim() != 2:
        raise ValueError("cos_t must have shape [tokens, rotated dimensions / 2]")
    pairs = cos_t.shape[1]
    for t, name in ((cos_t, "cos_t"), (sin_t, "sin_t")):
        _need(t, name, (n_frames * cache.T, pairs), torch.float32, cache.device)
    return 2 * pairs


def norm_weights(cache, q, wq, wk) -> None:
    if wk is None and wq is None:
        return
    _need(wk, "k_norm_weight", (cache.H * HEAD_DIM,), torch.bfloat16, cache.device)
    if q is not None:
        _need(wq, "q_norm_weight", (cache.H * HEAD_DIM,), torch.bfloat16, cache.device)


def append_rotary(cache, start_frame, n_frames, q, k, v, cos_t, sin_t, layout, wq, wk, eps, q_rot, stream):
    if stream is None and cache._native is not None:
        r = _calls_mx8.append_rotary(cache._native, start_frame, n_frames, q, k, v, cos_t, sin_t, layout, wq, wk, eps, q_rot)
        if r is not None:
            return r[0]
    ts, hs = cache._qkv_strides(q, k, v, n_frames)
    rot, code = table_rot(cache, cos_t, sin_t, n_frames), layout_code(layout)
    norm_weights(cache, q, wq, wk)
    if q is not None:
        q_rot = cache._chunk_out(q_rot, "q_rot", n_frames)
    with torch.cuda.device(cache.device):
        _check(lib.unstep_kv_append_rotary(cache.handle, start_frame, n_frames, _ptr(q), k.data_ptr(), v.data_ptr(), ts,
                                           hs, cos_t.data_ptr(), sin_t.data_ptr(), code, rot, _ptr(wq), _ptr(wk), eps,
                                           _ptr(q_rot), _stream(stream)))
        _used_on(stream, q_rot)
    return q_rot
