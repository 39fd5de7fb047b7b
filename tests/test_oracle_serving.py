"""Pins of oracle/serving.py: against torch's own casts, closed forms and a
plain softmax."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as OS


def test_fp8_grid_is_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = OS.grid("fp8")
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
    assert np.array_equal(np.signbit(got[~np.isnan(want)]), np.signbit(want[~np.isnan(want)]))


def test_fp4_grid():
    up = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert OS.grid("fp4").tolist() == up + [-x for x in up]


@pytest.mark.parametrize("kind", ["fp8", "int8", "fp4"])
def test_exponent_is_the_smallest(kind):
    rng = np.random.default_rng(0)
    top = OS.TOP[kind]
    for a in np.concatenate([np.exp(rng.uniform(-60, 60, 200)), [top, np.nextafter(top, 2 * top), top / 2, 1.0, 2.0 ** -126]]):
        e = OS.exponent(float(a), kind)
        assert a <= top * 2.0 ** e and (e == -126 or a > top * 2.0 ** (e - 1))
    assert OS.exponent(0.0, kind) == -126


def test_fp8_codes_are_torchs_casts():
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(20, 128, generator=g) * 10).to(torch.bfloat16)
    for row in x:
        codes, scales = OS.quantise(row.double().numpy(), "fp8")
        e = torch.from_numpy(scales - 127).repeat_interleave(32)
        want = (row.double() * torch.exp2(-e.double())).float().to(torch.float8_e4m3fn).view(torch.uint8)
        assert np.array_equal(codes, want.numpy())


def test_int8_codes_and_values():
    row = np.zeros(128)
    row[:4] = [127.0, 63.5, 64.5, -0.5]           # a scale of 1: ties go to the even code
    row[32:34] = [254.0, 3.0]                     # a scale of 2: 1.5 to 2
    codes, scales = OS.quantise(row, "int8")
    assert scales.tolist() == [127, 128, 1, 1]
    assert codes[:4].tolist() == [127, 64, 64, 0] and codes[32:34].tolist() == [127, 2]
    assert OS.value(codes, scales, "int8")[32:34].tolist() == [254.0, 4.0]


def test_not_finite_groups():
    row = np.ones(128)
    row[40], row[70] = np.nan, -np.inf
    codes, scales = OS.quantise(row, "fp4")
    v = OS.value(codes, scales, "fp4")
    assert scales.tolist()[1:3] == [255, 255] and np.isnan(v[32:96]).all() and (v[:32] == 1).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_is_a_complex_product(layout):
    rng = np.random.default_rng(2)
    x, pos = rng.standard_normal((5, 2, 128)), np.array([0, 1, 7, 1000, 2 ** 20])
    f = OS.frequencies(64)
    a, b = OS.pairs(64, layout)
    y = OS.rope(x, pos, f, layout, m=1.5)
    want = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, None, None] * f)
    assert np.allclose(y[..., a] + 1j * y[..., b], want, atol=1e-9)
    assert np.array_equal(y[..., 64:], x[..., 64:])
    back = OS.rope(y, pos, f, layout, m=1 / 1.5, inverse=True)
    assert np.allclose(back, x, atol=1e-9)


def test_frequencies():
    f = OS.frequencies(128, 1e4)
    assert f[0] == 1 and math.isclose(f[32], 1e-2)
    assert np.allclose(OS.frequencies(128, 1e4, "linear", 4.0), f / 4)
    ntk = OS.frequencies(128, 1e4, "ntk", 8.0)
    assert ntk[0] == 1 and math.isclose(ntk[-1], f[-1] / 8)            # the slowest pair is stretched by the factor
    parts = OS.frequencies(128, 1e4, "parts", 8.0, orig_len=4096, beta_fast=32, beta_slow=1)
    turns = 4096 * f / (2 * math.pi)
    assert np.allclose(parts[turns > 32], f[turns > 32]) and np.allclose(parts[turns < 1], f[turns < 1] / 8)


def test_attend_is_a_softmax():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((128,), (50, 128), (50, 128)))
    sees = torch.rand(50, generator=g) < 0.5
    o, lse, spread, bound = OS.attend(q.numpy(), k.numpy(), v.numpy(), sees.numpy(), 0.1)
    z = torch.where(sees, k @ q * 0.1, -math.inf)
    assert np.allclose(o, (torch.softmax(z, 0) @ v).numpy()) and math.isclose(lse, float(torch.logsumexp(z, 0)))
    assert (spread > 0).all() and bound > 0
    o, lse, _, _ = OS.attend(q.numpy(), k.numpy(), v.numpy(), np.zeros(50, bool), 0.1)
    assert (o == 0).all() and lse == -np.inf
