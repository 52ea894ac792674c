"""Pins of the oracle's microscaling blocks (n5): the element values against torch's own 8-bit type and the format's table, the
scale against its definition, the rounding against its bound and its ties."""
import numpy as np
import pytest
import torch

import oracle

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
TOP = {oracle.MXFP8: 448.0, oracle.MXFP4: 6.0}
FMTS = [oracle.MXFP8, oracle.MXFP4]


def _one(code, s, fmt):
    """The value of one element code."""
    c = np.zeros(32 if fmt == oracle.MXFP8 else 16, np.uint8)
    c[0] = code
    return oracle.mx_values(c, np.array([s], np.uint8), fmt)[0]


def test_element_values():
    for c in range(16):
        assert _one(c, 127, oracle.MXFP4) == (-1 if c >= 8 else 1) * E2M1[c % 8]
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    for c in range(256):
        got = _one(c, 127, oracle.MXFP8)
        assert got == want[c] or (np.isnan(got) and np.isnan(want[c]) and c % 128 == 127)
    assert _one(1, 0, oracle.MXFP4) == 2.0 ** -128 and _one(7, 254, oracle.MXFP4) == 6 * 2.0 ** 127
    assert np.isnan(_one(0, 255, oracle.MXFP4)) and np.isnan(_one(0, 255, oracle.MXFP8))


def _blocks(seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((400, 32)) * np.exp2(rng.integers(-30, 30, (400, 1)).astype(np.float64))
    x[::7] *= np.exp2(rng.integers(-12, 12, x[::7].shape).astype(np.float64))  # a wide range inside the block
    return x.astype(np.float32)


@pytest.mark.parametrize("fmt", FMTS)
def test_scale_is_the_smallest_that_clamps_nothing_and_values_are_within_half_a_step(fmt):
    x = _blocks(1)
    code, s = oracle.mx_quantise(x, fmt)
    back = oracle.mx_values(code, s, fmt)
    amax, unit = np.abs(x.astype(np.float64)).max(1), np.exp2(s[:, 0].astype(np.float64) - 127)
    assert np.all(amax <= TOP[fmt] * unit) and np.all(amax > TOP[fmt] * unit / 2)
    mant, small = (3, 2.0 ** -6) if fmt == oracle.MXFP8 else (1, 1.0)
    y = np.abs(back) / unit[:, None]
    step = np.exp2(np.floor(np.log2(np.maximum(np.maximum(y, np.abs(x) / unit[:, None]), small))) - mant)
    assert np.all(np.abs(back - x) <= step / 2 * unit[:, None])


@pytest.mark.parametrize("fmt", FMTS)
def test_what_is_held_quantises_to_itself(fmt):
    x = _blocks(2)
    code, s = oracle.mx_quantise(x, fmt)
    back = oracle.mx_values(code, s, fmt).astype(np.float32)
    again, s2 = oracle.mx_quantise(back, fmt)
    assert np.array_equal(oracle.mx_values(again, s2, fmt), back)


def test_ties_borders_and_blocks_that_are_not_finite():
    x = np.zeros((1, 32), np.float32)
    x[0, :12] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, -0.0, 0.2500001]
    code, s = oracle.mx_quantise(x, oracle.MXFP4)
    c = np.stack((code & 15, code >> 4), -1).reshape(1, 32)[0]
    assert s[0, 0] == 127 and c[:12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 14, 8, 1]
    x[0, 0] = np.nextafter(np.float32(6.0), np.float32(7.0))
    assert oracle.mx_quantise(x, oracle.MXFP4)[1][0, 0] == 128
    x[0, 0] = 448.0
    assert oracle.mx_quantise(x, oracle.MXFP8)[1][0, 0] == 127
    x[0, 0] = np.nextafter(np.float32(448.0), np.float32(449.0))
    assert oracle.mx_quantise(x, oracle.MXFP8)[1][0, 0] == 128
    for bad in (np.nan, np.inf, -np.inf):
        x[0, 5] = bad
        for fmt in FMTS:
            code, s = oracle.mx_quantise(x, fmt)
            assert s[0, 0] == 255 and not code.any() and np.isnan(oracle.mx_values(code, s, fmt)).all()
    for fmt in FMTS:
        code, s = oracle.mx_quantise(np.zeros((1, 32), np.float32), fmt)
        assert s[0, 0] == 0 and not oracle.mx_values(code, s, fmt).any()
        tiny = np.full((1, 32), 2.0 ** -140, np.float32)
        assert oracle.mx_quantise(tiny, fmt)[1][0, 0] == 0
        big = np.full((1, 32), np.finfo(np.float32).max, np.float32)
        code, s = oracle.mx_quantise(big, fmt)
        assert s[0, 0] < 255 and np.all(oracle.mx_values(code, s, fmt) <= 2.0 ** 128)
