"""Pins of the quantised format's and the rotary options' oracle: torch's own e4m3 conversion, closed
forms, the half-step bound, and complex multiplication."""
import math

import numpy as np
import pytest
import torch

from oracle import mx8, rope, tables
from oracle.numerics import f32_to_bf16_bits


def test_e4m3_numbers_are_torchs():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = mx8.e4m3_value(codes.numpy())
    assert np.array_equal(np.isnan(want), np.isnan(got))
    assert np.array_equal(want[~np.isnan(want)], got[~np.isnan(got)])


def test_e4m3_rounding_is_torchs():
    g = torch.Generator().manual_seed(1)
    z = torch.cat([torch.randn(200000, generator=g) * 30, torch.randn(50000, generator=g) * 0.02,
                   torch.tensor(mx8.E4M3, dtype=torch.float32),
                   torch.tensor((mx8.E4M3[1:] + mx8.E4M3[:-1]) / 2, dtype=torch.float32)]).clamp(-448, 448)
    want = z.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(mx8.e4m3_code(z.double().numpy()), want)


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0000001, 1), (896.0, 1), (1.75, -8), (1.7500001, -7), (1.0, -8), (0.0, -100),
                                   (2.0 ** -92, -100), (2.0 ** -90, -98), (3.38e38, 120), (2.0 ** -149, -100)])
def test_block_exponent(top, e):
    assert mx8.exponent(top) == e


def test_held_values_are_within_half_a_step():
    y = np.random.default_rng(2).standard_normal((500, 128)) * np.exp2(np.random.default_rng(3).integers(-40, 40, (500, 1)))
    c, s = mx8.quantise(y)
    v = mx8.values(c, s)
    top = np.abs(y.reshape(500, 4, 32)).max(-1).repeat(32, -1)
    # half a step: 2^-4 of the value, at least half of the smallest step 2^-9 of the block's scale (<= top / 224)
    assert np.all(np.abs(v - y) <= np.maximum(np.abs(y) * 2.0 ** -4, top / 224 * 2.0 ** -10))
    assert np.array_equal(v, f32_to_f64_bf16(v))
    bad = y.copy()
    bad[0, 3], bad[1, 40], bad[2, 127] = np.inf, -np.inf, np.nan
    cb, sb = mx8.quantise(bad)
    assert np.isnan(mx8.values(cb, sb)[[0, 1, 2], [3, 40, 127]]).all() and np.isnan(mx8.values(cb, sb)).sum() == 3


def f32_to_f64_bf16(v):
    return (f32_to_bf16_bits(v).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("pairs", [8, 32, 48, 64])
def test_rotation_is_complex_multiplication(half, pairs):
    rng = np.random.default_rng(pairs)
    x = f32_to_bf16_bits(rng.standard_normal((5, 3, 128)))
    ang = rng.uniform(0, 100, (5, pairs))
    c, s = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    y = mx8.rotate(x, c, s, half)
    xf = f32_to_f64_bf16_bits(x)
    z = (xf[..., :pairs] + 1j * xf[..., pairs:2 * pairs]) if half else (xf[..., 0:2 * pairs:2] + 1j * xf[..., 1:2 * pairs:2])
    w = z * np.exp(1j * ang)[:, None]
    got = (y[..., :pairs] + 1j * y[..., pairs:2 * pairs]) if half else (y[..., 0:2 * pairs:2] + 1j * y[..., 1:2 * pairs:2])
    assert np.abs(got - w).max() < 2.0 ** -21 * np.abs(z).max()
    assert np.array_equal(y[..., 2 * pairs:], xf[..., 2 * pairs:])
    if not half and pairs == 64:
        assert np.array_equal(f32_to_bf16_bits(y), rope.rope_bf16(x, c, s))


def f32_to_f64_bf16_bits(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def test_unscaled_tables_are_the_models():
    c, s = mx8.tables(6, 3, 4, 5, (44, 42, 42))
    wc, ws = tables.rope_tables(6, 3, 4, 5)
    assert np.array_equal(c.astype(np.float32), wc) and np.array_equal(s.astype(np.float32), ws)


def test_scalings():
    d, s = (64, 32, 32), 8.0
    plain = mx8.frequencies(d)
    lin = mx8.frequencies(d, scaling="linear", factor=s)
    base = mx8.frequencies(d, scaling="base", factor=s)
    parts = mx8.frequencies(d, scaling="parts", factor=s, trained=1024.0)
    for f in (lin, base, parts):
        assert np.array_equal(f[32:], plain[32:])                  # rows and columns are not scaled
    assert np.allclose(lin[:32], plain[:32] / s)
    assert base[0] == plain[0] and math.isclose(base[31], plain[31] / s, rel_tol=1e-12)
    turns = 1024.0 * plain[:32] / (2 * math.pi)
    assert np.array_equal(parts[:32][turns >= 32], plain[:32][turns >= 32])
    assert np.allclose(parts[:32][turns <= 1], plain[:32][turns <= 1] / s)
    assert np.all(parts[:32] <= plain[:32]) and np.all(parts[:32] >= plain[:32] / s * (1 - 1e-12))
