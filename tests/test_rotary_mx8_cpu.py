"""Refusals and host state of the rotary options and the quantised cache: every bad call is refused before
anything is enqueued and leaves the positions as they were.  No kernel runs here (addresses are fake and
never read)."""
import ctypes
import math

import pytest
import torch

u = pytest.importorskip("paper_2609_32518_amd")
from paper_2609_32518_amd.rotary import _Rotary  # noqa: E402

A = [0x10000 * (i + 1) for i in range(16)]         # fake device addresses


def opts(**kw):
    d = dict(dim_t=44, dim_h=42, dim_w=42, scaling=0, theta=1e4, factor=1.0, trained_frames=0.0, turns_fast=32.0,
             turns_slow=1.0, amplitude=0.0)
    d.update(kw)
    return _Rotary(**d)


def tables(o, f0=0, C=1, gh=2, gw=2, c=A[0], s=A[1]):
    return u.lib.unstep_rotary_tables(f0, C, gh, gw, ctypes.addressof(o) if o is not None else None, c, s, None)


@pytest.mark.parametrize("rc,kw,call", [
    ("E_NULL", {}, dict(c=None)), ("E_NULL", {}, dict(s=None)), ("E_NULL", None, {}),
    ("E_SHAPE", dict(dim_t=43), {}), ("E_SHAPE", dict(dim_t=46), {}), ("E_SHAPE", dict(dim_t=-2), {}),
    ("E_SHAPE", dict(dim_t=0, dim_h=0, dim_w=0), {}), ("E_SHAPE", dict(dim_t=60), {}),
    ("E_SHAPE", dict(dim_t=2147483646, dim_h=2147483646, dim_w=20), {}),
    ("E_SHAPE", {}, dict(C=0)), ("E_SHAPE", {}, dict(gh=0)), ("E_SHAPE", {}, dict(gw=-1)),
    ("E_SHAPE", {}, dict(C=2 ** 31 - 1, gh=2 ** 31 - 1, gw=2 ** 31 - 1)), ("E_SHAPE", {}, dict(C=1, gh=4096, gw=2049)),
    ("E_RANGE", {}, dict(f0=-1)), ("E_RANGE", {}, dict(f0=2 ** 31 - 1, C=1)),
    ("E_RANGE", dict(theta=1.0), {}), ("E_RANGE", dict(theta=math.nan), {}), ("E_RANGE", dict(scaling=4), {}),
    ("E_RANGE", dict(scaling=-1), {}), ("E_RANGE", dict(scaling=1, factor=0.5), {}), ("E_RANGE", dict(scaling=2, factor=math.inf), {}),
    ("E_RANGE", dict(scaling=3, factor=2.0), {}), ("E_RANGE", dict(scaling=3, factor=2.0, trained_frames=10.0, turns_fast=1.0), {}),
    ("E_RANGE", dict(scaling=3, factor=2.0, trained_frames=10.0, turns_slow=-1.0), {}),
    ("E_RANGE", dict(amplitude=-1.0), {}), ("E_RANGE", dict(amplitude=math.nan), {}),
    ("E_ALIGN", {}, dict(c=A[0] + 4)), ("E_ALIGN", {}, dict(s=A[1] + 8))])
def test_table_refusals(rc, kw, call):
    assert tables(None if kw is None else opts(**kw), **call) == getattr(u, rc)


def handle(mx8, B=1, H=2, gh=2, gw=3, S=1, R=4, D=128, k=A[0], ks=A[1], v=A[2], vs=A[3]):
    h = u._vp()
    if mx8:
        rc = u.lib.unstep_cache_create_mx8(ctypes.byref(h), B, H, D, gh, gw, S, R, k, ks, v, vs)
    else:
        rc = u.lib.unstep_cache_create(ctypes.byref(h), B, H, D, gh, gw, S, R, k, v)
    return rc, h


@pytest.mark.parametrize("rc,kw", [("E_NULL", dict(k=None)), ("E_NULL", dict(ks=None)), ("E_NULL", dict(v=None)),
                                   ("E_NULL", dict(vs=None)), ("E_ALIGN", dict(ks=A[1] + 4)), ("E_ALIGN", dict(v=A[2] + 8)),
                                   ("E_SHAPE", dict(D=64)), ("E_SHAPE", dict(R=0)), ("E_SHAPE", dict(gh=4096, gw=2048))])
def test_create_refusals(rc, kw):
    assert handle(True, **kw)[0] == getattr(u, rc)


def append(h, kind, f0=0, C=1, q=A[4], k=A[5], v=A[6], ts=256, hs=128, cos=A[7], sin=A[8], layout=0, rot=128, wq=None, wk=None,
           eps=1e-6, scale=0.0, q8=A[9], qs=A[10]):
    if kind == "rotary":
        return u.lib.unstep_kv_append_rotary(h, f0, C, q, k, v, ts, hs, cos, sin, layout, rot, wq, wk, eps, q8, None)
    if kind == "mx8":
        return u.lib.unstep_kv_append_mx8(h, f0, C, q, k, v, ts, hs, cos, sin, layout, rot, wq, wk, eps, scale, q8, qs, None)
    return u.lib.unstep_step_mx8(h, f0, C, 0, q, k, v, ts, hs, cos, sin, layout, rot, wq, wk, eps, scale, q8, qs, A[11], None,
                                 None, 0, None)


BAD_APPENDS = [
    ("E_NULL", dict(k=None)), ("E_NULL", dict(cos=None)), ("E_NULL", dict(q8=None)), ("E_NULL", dict(wq=A[12])),
    ("E_NULL", dict(wk=A[12])), ("E_SHAPE", dict(C=0)), ("E_SHAPE", dict(rot=0)), ("E_SHAPE", dict(rot=8)),
    ("E_SHAPE", dict(rot=120)), ("E_SHAPE", dict(rot=144)), ("E_SHAPE", dict(hs=64)), ("E_SHAPE", dict(ts=128)),
    ("E_RANGE", dict(layout=2)), ("E_RANGE", dict(layout=-1)), ("E_RANGE", dict(f0=-1)), ("E_RANGE", dict(C=6)),
    ("E_RANGE", dict(wq=A[12], wk=A[13], eps=-1.0)), ("E_RANGE", dict(wq=A[12], wk=A[13], eps=math.nan)),
    ("E_STATE", dict(f0=1)), ("E_ALIGN", dict(q=A[4] + 2)), ("E_ALIGN", dict(ts=260)), ("E_ALIGN", dict(q8=A[9] + 8)),
    ("E_ALIGN", dict(wq=A[12] + 2, wk=A[13])), ("E_ALIGN", dict(sin=A[8] + 4))]


@pytest.mark.parametrize("kind", ["rotary", "mx8", "step"])
@pytest.mark.parametrize("rc,kw", BAD_APPENDS)
def test_append_refusals(kind, rc, kw):
    ok, h = handle(kind != "rotary")
    assert ok == u.OK
    try:
        assert append(h, kind, **kw) == getattr(u, rc)
        assert u.lib.unstep_last_error()
        newest = ctypes.c_int32()
        u.lib.unstep_cache_frame_map(h, (ctypes.c_int32 * 5)(), ctypes.byref(newest))
        assert newest.value == -1
        if kind != "rotary":
            assert append(h, kind, qs=None) == u.E_NULL
            assert append(h, kind, qs=A[10] + 2) == u.E_ALIGN
            assert append(h, kind, scale=math.nan) == u.E_RANGE and append(h, kind, scale=math.inf) == u.E_RANGE
        if kind == "step":
            assert append(h, kind, q=None) == u.E_NULL
    finally:
        u.lib.unstep_cache_destroy(h)


def test_size_refusals():
    _, h = handle(True, H=33)
    _, big = handle(True, H=31, gh=2048, gw=1024, S=0, R=3)     # a frame of 2^21 tokens x 31 heads is allowed
    try:
        strides = dict(ts=33 * 128, hs=128)
        assert append(h, "mx8", wq=A[12], wk=A[13], **strides) == u.E_SHAPE            # more heads than a token's waves hold
        assert append(h, "mx8", ts=2 ** 32 + 8, hs=128) == u.E_SHAPE
        assert append(big, "mx8", C=3, ts=31 * 128, hs=128) == u.E_SHAPE               # 3 of them are not, in one chunk
        assert u.lib.unstep_cache_advance(big, 0, 3) == u.OK
        assert u.lib.unstep_kv_read_mx8(big, 0, 3, A[4], A[5], None) == u.E_SHAPE      # 3 x 2^21 x 31 rows
    finally:
        u.lib.unstep_cache_destroy(h)
        u.lib.unstep_cache_destroy(big)


def test_one_kind_of_cache_refuses_the_others_calls():
    _, hb = handle(False)
    _, hq = handle(True)
    try:
        assert u.lib.unstep_cache_advance(hb, 0, 1) == u.OK and u.lib.unstep_cache_advance(hq, 0, 1) == u.OK
        for kind in ("mx8", "step"):
            assert append(hb, kind) == u.E_STATE
        assert append(hq, "rotary") == u.E_STATE
        assert u.lib.unstep_kv_append(hq, 0, 1, None, A[5], A[6], 256, 128, A[7], A[8], None, None) == u.E_STATE
        assert u.lib.unstep_kv_append_qknorm(hq, 0, 1, None, A[5], A[6], 256, 128, A[7], A[8], None, A[9], 1e-6, None, None) == u.E_STATE
        assert u.lib.unstep_window_attn(hq, 0, 1, 0, A[5], A[6], None, 0.0, None, 0, None) == u.E_STATE
        assert u.lib.unstep_window_attn_noalloc(hq, 0, 1, 0, A[5], A[6], None, 0.0, None) == u.E_STATE
        assert u.lib.unstep_step(hq, 0, 1, 0, A[4], A[5], A[6], 256, 128, A[7], A[8], A[9], A[10], None, 0.0, None, 0, None) == u.E_STATE
        assert u.lib.unstep_window_attn_mx8(hb, 0, 1, 0, A[5], A[6], A[7], None, None, 0, None) == u.E_STATE
        assert u.lib.unstep_kv_read_mx8(hb, 0, 1, A[5], A[6], None) == u.E_STATE
        for call in (append(None, "mx8"), append(None, "step"), append(None, "rotary"),
                     u.lib.unstep_window_attn_mx8(None, 0, 1, 0, A[5], A[6], A[7], None, None, 0, None),
                     u.lib.unstep_kv_read_mx8(None, 0, 1, A[5], A[6], None)):
            assert call == u.E_NULL
    finally:
        u.lib.unstep_cache_destroy(hb)
        u.lib.unstep_cache_destroy(hq)


def test_attention_and_read_refusals():
    _, h = handle(True)
    attn = lambda f0=3, C=1, W=1, q8=A[4], qs=A[5], out=A[6], lse=None, ws=None: u.lib.unstep_window_attn_mx8(  # noqa: E731
        h, f0, C, W, q8, qs, out, lse, ws, 0, None)
    read = lambda f0=3, C=1, k=A[4], v=A[5]: u.lib.unstep_kv_read_mx8(h, f0, C, k, v, None)  # noqa: E731
    try:
        for f in range(8):                                   # frames 0 and 4..7 are stored (one sink, a ring of four)
            assert u.lib.unstep_cache_advance(h, f, 1) == u.OK
        assert attn(q8=None) == attn(qs=None) == attn(out=None) == u.E_NULL
        assert attn(C=0) == u.E_SHAPE and attn(f0=-1) == attn(W=-1) == attn(f0=7, W=10) == u.E_RANGE
        assert attn(f0=8) == attn(f0=3) == u.E_STATE
        assert attn(f0=7, q8=A[4] + 8) == attn(f0=7, qs=A[5] + 1) == attn(f0=7, lse=A[7] + 2) == attn(f0=7, ws=A[8] + 4) == u.E_ALIGN
        assert read(f0=7, k=None) == read(f0=7, v=None) == u.E_NULL and read(C=0) == u.E_SHAPE and read(f0=-1) == u.E_RANGE
        assert read(f0=3) == read(f0=7, C=2) == read(f0=0, C=2) == read(f0=4, C=2 ** 31 - 5) == u.E_STATE
        assert read(f0=7, k=A[4] + 2) == u.E_ALIGN
    finally:
        u.lib.unstep_cache_destroy(h)
    deq = u.lib.unstep_mx8_dequantize
    assert deq(None, A[0], A[1], 4, None) == deq(A[0], None, A[1], 4, None) == deq(A[0], A[1], None, 4, None) == u.E_NULL
    assert deq(A[0], A[1], A[2], -1, None) == deq(A[0], A[1], A[2], 2 ** 27 + 1, None) == u.E_SHAPE
    assert deq(A[0] + 8, A[1], A[2], 4, None) == deq(A[0], A[1], A[2] + 8, 4, None) == u.E_ALIGN
    assert deq(A[0], A[1], A[2], 0, None) == u.OK


def test_binding_checks_tensors():
    c = u.CacheMX8(1, 2, 2, 3, 1, 4, device="cpu")
    assert c.k8.dtype == torch.float8_e4m3fn and c.k8.shape == (1, 2, 30, 128) and c.k_scale.shape == (1, 2, 30, 4)
    x = torch.zeros(1, 6, 2, 128, dtype=torch.bfloat16)
    t = torch.zeros(6, 64)
    good = dict(q=x, k=x, v=x, cos_t=t, sin_t=t)
    for bad in (dict(k=x.float()), dict(v=x[:, :5]), dict(cos_t=t[:5]), dict(sin_t=t[:, :32]), dict(cos_t=t.double()),
                dict(q=x.transpose(1, 2).contiguous()), dict(cos_t=t[0])):
        with pytest.raises(ValueError):
            c.unstep_kv_append_mx8(0, 1, **{**good, **bad})
        with pytest.raises(ValueError):
            c.unstep_step_mx8(0, 1, 0, **{**good, **bad})
    with pytest.raises(ValueError, match="layout"):
        c.unstep_kv_append_mx8(0, 1, layout="both", **good)
    with pytest.raises(ValueError, match="k_norm_weight"):
        c.unstep_kv_append_mx8(0, 1, q_norm_weight=torch.zeros(256, dtype=torch.bfloat16), **good)
    with pytest.raises(ValueError, match="q_scale"):
        c.unstep_kv_append_mx8(0, 1, q_scale=torch.zeros(1, 6, 2, 4), **good)
    with pytest.raises(ValueError, match="q8"):
        c.unstep_window_attn_mx8(0, 1, 0, None, torch.zeros(1, 6, 2, 4, dtype=torch.uint8))
    with pytest.raises(ValueError):
        c.unstep_step_mx8(0, 1, 0, None, x, x, t, t)
    with pytest.raises(ValueError):
        u.CacheMX8(1, 2, 2, 3, 1, 4, device="cpu", k_scale=torch.zeros(1, 2, 30, 8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        u.unstep_mx8_dequantize(torch.zeros(3, 64, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(3, 4, dtype=torch.uint8))
    with pytest.raises(ValueError):
        u.unstep_rotary_tables(0, 1, 2, 2, scaling="cubic", device="cpu")
    assert c.frame_map() == ([-1] * 5, -1)
