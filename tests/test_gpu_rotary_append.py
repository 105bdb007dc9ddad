"""Rotary tables and the rotating appends on the GPU: tables within a float rounding of float64, every
output of the appends equal bit for bit to the oracle's (bf16 rows, or e4m3 codes and scale bytes), rows
outside the chunk untouched, quantised rows read back exactly.  Inputs are seeded; expected values come
from oracle only."""
import numpy as np
import pytest
import torch

import synth
from oracle import mx8, rmsnorm
from oracle.numerics import bf16_to_f64, f32_to_bf16_bits
from tests.gpu_helpers import dev, host

pytestmark = pytest.mark.gpu

u = pytest.importorskip("paper_2609_32518_amd")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

DIMS = {128: (44, 42, 42), 96: (32, 32, 32), 64: (64, 0, 0), 48: (0, 24, 24), 16: (4, 6, 6)}


@pytest.mark.parametrize("start,C,gh,gw,dims,kw", [
    (0, 1, 1, 1, (128, 0, 0), {}), (123, 5, 1, 1, (16, 0, 0), {}), (9, 3, 30, 52, (44, 42, 42), {}),
    (60000, 2, 7, 9, (44, 42, 42), dict(scaling="parts", factor=4.0, trained_frames=1024.0)),
    (2 ** 31 - 9, 4, 3, 8, (64, 32, 32), dict(scaling="linear", factor=3.5)),
    (1000, 1, 1, 17, (2, 62, 64), dict(scaling="base", factor=8.0)), (1000, 1, 5, 1, (64, 32, 16), dict(scaling="base", factor=8.0)),
    (7, 1, 2, 3, (0, 8, 8), dict(theta=500000.0, amplitude=0.75)), (0, 600, 1, 1, (32, 16, 16), {}), (3, 1, 2, 1000, (0, 0, 128), {})])
def test_tables(start, C, gh, gw, dims, kw):
    c, s = u.unstep_rotary_tables(start, C, gh, gw, dims=dims, **kw)
    ref = {k: v for k, v in kw.items() if k not in ("trained_frames", "amplitude")}
    amp = kw.get("amplitude") or (0.1 * np.log(kw["factor"]) + 1 if kw.get("scaling") == "parts" else 1.0)
    wc, ws = mx8.tables(start, C, gh, gw, dims, amp, trained=kw.get("trained_frames", 0.0), **ref)
    for got, want in ((c, wc), (s, ws)):
        assert tuple(got.shape) == want.shape
        # half a float step of a value below 2, and the angle's float64 rounding (2^-52 of an angle below 2^31)
        assert np.abs(got.cpu().numpy() - want).max() <= 2.0 ** -24 * amp + 2.0 ** -20 * (start > 2 ** 30)
    again = (torch.empty_like(c), torch.empty_like(s))
    assert u.unstep_rotary_tables(start, C, gh, gw, dims=dims, out=again, **kw)[0] is again[0]
    assert torch.equal(again[0], c) and torch.equal(again[1], s)


def chunk(B, N, H, seed, layout):
    g = np.random.default_rng(seed)
    bits = [f32_to_bf16_bits(g.standard_normal((B, N, H, 128)) * np.exp2(g.integers(-8, 8, (1, 1, H, 128)))) for _ in range(3)]
    if layout == "fused":
        q, k, v = torch.stack([dev(b) for b in bits], dim=2).unbind(2)
    elif layout == "padded":                                    # rows of a wider tensor
        wide = torch.full((B, N, H + 1, 160), 7.0, dtype=torch.bfloat16, device="cuda")
        q, k, v = (wide.clone()[:, :, :H, :128] for _ in range(3))
        for t, b in zip((q, k, v), bits):
            t.copy_(dev(b))
    else:
        q, k, v = (dev(b) for b in bits)
    return bits, (q, k, v)


def weights(H, seed):
    w = [f32_to_bf16_bits(1 + 0.2 * np.random.default_rng(seed + i).standard_normal(H * 128)) for i in range(2)]
    return w, [dev(x) for x in w]


def expected(bits, c, s, half, w):
    """binary32 (in float64) q and k after normalisation and rotation."""
    out = []
    for i in range(2):
        x = bits[i]
        if w is not None:
            x = rmsnorm.rms_norm_bf16(x.reshape(x.shape[:2] + (-1,)), w[i]).reshape(x.shape)
        out.append(mx8.rotate(x, c, s, half))
    return out


CASES = [  # B, H, gh, gw, S, R, f0, C, rot, layout, norm, strides
    (1, 1, 1, 1, 0, 4, 2, 1, 128, "interleaved", False, "plain"), (1, 12, 1, 1, 1, 6, 9, 1, 128, "half", True, "plain"),
    (2, 3, 3, 5, 1, 4, 5, 2, 96, "half", False, "fused"), (2, 5, 3, 5, 2, 3, 0, 3, 64, "interleaved", True, "fused"),
    (1, 13, 4, 4, 0, 5, 3, 2, 48, "half", True, "padded"), (1, 32, 1, 3, 0, 2, 1, 1, 16, "half", True, "plain"),
    (3, 2, 2, 3, 1, 3, 4, 1, 16, "interleaved", False, "padded"), (1, 2, 7, 11, 0, 9, 8, 3, 128, "half", False, "fused")]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("with_q", [True, False])
def test_append_is_the_oracles(case, with_q):
    B, H, gh, gw, S, R, f0, C, rot, layout, norm, strides = case
    T, N, slots = gh * gw, C * gh * gw, (S + R) * gh * gw
    bits, (q, k, v) = chunk(B, N, H, 17, strides)
    c, s = (np.ascontiguousarray(t, np.float32) for t in mx8.tables(f0, C, gh, gw, DIMS[rot]))
    ct, st = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
    w, wd = weights(H, 5) if norm else (None, (None, None))
    want_q, want_k = expected(bits, c, s, layout == "half", w)
    kw = dict(layout=layout, q_norm_weight=wd[0] if with_q else None, k_norm_weight=wd[1])
    rows = np.concatenate([((f if f < S else S + (f - S) % R) * T) + np.arange(T) for f in range(f0, f0 + C)])
    others = np.setdiff1d(np.arange(slots), rows)

    # bf16 cache
    fill = torch.full((B, H, slots, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    cache = u.Cache(B, H, gh, gw, S, R, k_cache=fill.clone(), v_cache=fill.clone())
    for f in range(f0):
        cache.advance(f, 1)
    got = cache.unstep_kv_append_rotary(f0, C, q if with_q else None, k, v, ct, st, **kw)
    assert (got is None) == (not with_q)
    if with_q:
        assert np.array_equal(host(got), f32_to_bf16_bits(want_q))
    for buf, want in ((cache.k, f32_to_bf16_bits(want_k)), (cache.v, bits[2])):
        b = host(buf)
        assert np.array_equal(b[:, :, rows], want.transpose(0, 2, 1, 3))
        assert np.all(b[:, :, others] == 0x4040)
    assert cache.frame_map()[1] == f0 + C - 1

    # quantised cache
    m = u.CacheMX8(B, H, gh, gw, S, R)
    for t in (m.k8, m.v8, m.k_scale, m.v_scale):
        t.view(torch.uint8).fill_(77)
    for f in range(f0):
        m.advance(f, 1)
    got = m.unstep_kv_append_mx8(f0, C, q if with_q else None, k, v, ct, st, **kw)
    assert (got is None) == (not with_q)
    raw = lambda t: t.view(torch.uint8).cpu().numpy()  # noqa: E731
    if with_q:
        mul = np.float64(np.float32(128 ** -0.5 * 1.4426950408889634))
        codes, scale = mx8.quantise((want_q * mul).astype(np.float32).astype(np.float64))
        assert np.array_equal(raw(got[1]), scale) and np.array_equal(raw(got[0]), codes)
        assert np.array_equal(bf16_to_f64(host(u.unstep_mx8_dequantize(*got))), mx8.values(codes, scale))
    back = m.unstep_kv_read_mx8(f0, C)
    for data, sc, y, r in ((m.k8, m.k_scale, want_k, back[0]), (m.v8, m.v_scale, bf16_to_f64(bits[2]), back[1])):
        codes, scale = mx8.quantise(y)
        assert np.array_equal(raw(sc)[:, :, rows], scale.transpose(0, 2, 1, 3))
        assert np.array_equal(raw(data)[:, :, rows], codes.transpose(0, 2, 1, 3))
        assert np.all(raw(data)[:, :, others] == 77) and np.all(raw(sc)[:, :, others] == 77)
        assert np.array_equal(bf16_to_f64(host(r)), mx8.values(codes, scale))


@pytest.mark.parametrize("norm", [False, True])
def test_interleaved_whole_head_is_the_plain_append(norm):
    B, H, gh, gw, C = 2, 3, 5, 6, 2
    _, (q, k, v) = chunk(B, C * gh * gw, H, 3, "fused")
    ct, st = u.unstep_rope_tables(0, C, gh, gw)
    _, wd = weights(H, 8)
    a, b = u.Cache(B, H, gh, gw, 0, 3), u.Cache(B, H, gh, gw, 0, 3)
    if norm:
        qa = a.unstep_kv_append_qknorm(0, C, q, k, v, ct, st, *wd)
        qb = b.unstep_kv_append_rotary(0, C, q, k, v, ct, st, q_norm_weight=wd[0], k_norm_weight=wd[1])
    else:
        qa = a.unstep_kv_append(0, C, q, k, v, ct, st)
        qb = b.unstep_kv_append_rotary(0, C, q, k, v, ct, st)
    for x, y in ((qa, qb), (a.k, b.k), (a.v, b.v)):
        assert np.array_equal(host(x), host(y))


def test_quantising_extremes():
    """Blocks of zeros, of the smallest and the largest numbers, ties, and values that are not finite."""
    H = 2
    x = np.zeros((1, 8, H, 128), np.float64)
    x[0, 1, 0, :32] = 2.0 ** -130
    x[0, 1, 0, 32:64] = 2.0 ** -95
    x[0, 1, 0, 64:96] = 3.0e38
    x[0, 1, 1, :16] = np.arange(16) * 2.0 ** -107
    x[0, 2, 0, :16] = [448, 17, 19, 21, 25, 27, -17, -19, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, -(2.0 ** -10), 464, 240, 232]
    x[0, 2, 1, :8] = [450, 1.0625, 1.1875, 1.3125, 448, -449, 2.0 ** -8, 2.0 ** -9]
    x[0, 3, 0, 5], x[0, 3, 0, 40], x[0, 3, 1, 127] = np.inf, -np.inf, np.nan
    x[0, 3, :, :] += np.where(np.isfinite(x[0, 3]), 1.5, 0.0)
    x[0, 4, 0, :32] = np.nan
    bits = np.where(np.isnan(x), 0x7FC0, 0).astype(np.uint16)
    fin = ~np.isnan(x)
    with np.errstate(over="ignore"):
        f = x.astype(np.float32).view(np.uint32)
    bits[fin] = (f[fin] >> 16).astype(np.uint16)
    y = bf16_to_f64(bits)
    m = u.CacheMX8(1, H, 2, 4, 0, 1)
    zero = torch.zeros(8, 8, device="cuda")
    d = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    q8, qs = m.unstep_kv_append_mx8(0, 1, d, d, d, torch.ones_like(zero), zero, softmax_scale=1.0 / 1.4426950408889634)
    codes, scale = mx8.quantise(y.astype(np.float32).astype(np.float64))
    for data, sc in ((m.v8, m.v_scale), (m.k8, m.k_scale)):
        got = data.view(torch.uint8).cpu().numpy().transpose(0, 2, 1, 3)
        # dimensions from 16 on are not rotated; the first 16 of the keys are, by the angle 0 (x * 1 - x' * 0 is
        # x where the partner is finite)
        part = slice(16, 128) if data is m.k8 else slice(0, 128)
        nan = (codes & 0x7F) == 0x7F
        same = (got == codes) | (nan & ((got & 0x7F) == 0x7F)) | (((got | codes) & 0x7F) == 0)
        assert same[..., part].all()
        assert np.array_equal(sc.cpu().numpy().transpose(0, 2, 1, 3), scale)
    k, v = m.unstep_kv_read_mx8(0, 1)
    want = mx8.values(codes, scale)
    assert np.array_equal(np.isnan(want), np.isnan(v.double().cpu().numpy()))
    assert np.array_equal(np.nan_to_num(v.double().cpu().numpy()), np.nan_to_num(want))
    assert u.unstep_mx8_dequantize(q8[:, :0], qs[:, :0]).shape == (1, 0, H, 128)


def test_append_replayed_from_a_graph_and_on_another_stream():
    B, H, gh, gw, C = 1, 3, 4, 5, 2
    a, b = u.CacheMX8(B, H, gh, gw, 0, 4), u.CacheMX8(B, H, gh, gw, 0, 4)
    _, buf = chunk(B, C * gh * gw, H, 1, "plain")
    n = C * gh * gw
    cos, sin = torch.empty(n, 64, device="cuda"), torch.empty(n, 64, device="cuda")
    q8 = torch.empty(B, n, H, 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    qs = torch.empty(B, n, H, 4, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        u.unstep_rotary_tables(0, C, gh, gw, out=(cos, sin))
        a.unstep_kv_append_mx8(0, C, *buf, cos, sin, layout="half", q8=q8, q_scale=qs)
    side = torch.cuda.Stream()
    for r in range(3):
        _, new = chunk(B, n, H, 100 + r, "plain")
        for t, x in zip(buf, new):
            t.copy_(x)
        torch.cuda.synchronize()
        g.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side) if r == 1 else torch.cuda.stream(torch.cuda.current_stream()):
            c2, s2 = u.unstep_rotary_tables(0, C, gh, gw, stream=side)
            w8, ws = b.unstep_kv_append_mx8(0, C, *new, c2, s2, layout="half", stream=side)
        torch.cuda.synchronize()
        for x, y in ((a.k8, b.k8), (a.v8, b.v8), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale), (q8, w8), (qs, ws)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("scale,eps", [(2.0 ** 60, 0.0), (2.0 ** -62, 0.0), (2.0 ** 55, 1e-6), (2.0 ** -40, 1e-6), (2.0 ** -70, 0.0)])
def test_normalisation_of_very_large_and_small_tokens(scale, eps):
    """Statistics outside the range of the fast path, beside ordinary ones in the same work-group."""
    B, H, gh, gw = 1, 3, 2, 4
    g = np.random.default_rng(11)
    x = g.standard_normal((B, gh * gw, H, 128))
    x[:, 1::2] *= scale
    bits = [f32_to_bf16_bits(x), f32_to_bf16_bits(x[:, ::-1]), f32_to_bf16_bits(x)]
    c, s = (np.ascontiguousarray(t, np.float32) for t in mx8.tables(0, 1, gh, gw, (44, 42, 42)))
    w, wd = weights(H, 5)
    flat = lambda t: t.reshape(B, gh * gw, H * 128)  # noqa: E731
    want = [mx8.rotate(rmsnorm.rms_norm_bf16(flat(bits[i]), w[i], eps).reshape(x.shape), c, s, False) for i in range(2)]
    b = u.Cache(B, H, gh, gw, 0, 1)
    q = b.unstep_kv_append_rotary(0, 1, *(dev(t) for t in bits), torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(),
                                  q_norm_weight=wd[0], k_norm_weight=wd[1], norm_eps=eps)
    assert np.array_equal(host(q), f32_to_bf16_bits(want[0]))
    assert np.array_equal(host(b.k), f32_to_bf16_bits(want[1]).transpose(0, 2, 1, 3))
