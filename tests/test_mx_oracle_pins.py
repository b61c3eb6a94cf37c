"""Pins of the oracle of the 8- and 4-bit cache (oracle/mx.py): hand-made codes, the definition
of the shared power, and torch's own e4m3."""
import numpy as np
import pytest
import torch

from oracle import mx


def test_elements():
    e = mx.elements(4)
    assert e[:8].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6] and (e[8:] == -e[:8]).all()
    e = mx.elements(8)
    assert (e[1], e[8], e[0x38], e[0x7e]) == (2.0 ** -9, 2.0 ** -6, 1.0, 448.0)
    other = torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(e, other, equal_nan=True)


@pytest.mark.parametrize("bits", (8, 4))
def test_the_shared_power_is_the_least_that_holds_the_largest(bits):
    r = np.random.default_rng(1)
    x = r.standard_normal((300, 64)) * 2.0 ** r.integers(-100, 100, (300, 1))
    code, scale = mx.quantise(x, bits)
    top = np.abs(x).reshape(300, 2, 32).max(-1)
    power = 2.0 ** (scale.astype(float) - 127)
    assert (top <= mx.LARGEST[bits] * power).all() and (top > mx.LARGEST[bits] * power / 2).all()
    off = np.abs(mx.values(code, scale, bits) - x).reshape(300, 2, 32)
    unit, least = {8: (2.0 ** -4, 2.0 ** -10), 4: (0.25, 0.25)}[bits]
    assert (off <= np.maximum(np.abs(x).reshape(300, 2, 32) * unit, power[..., None] * least)).all()


def test_eight_bits_round_as_torch_does():
    x = np.random.default_rng(2).standard_normal((500, 32)).astype(np.float32)
    x[:, 0] = 7.0  # power -6 everywhere: 448 2^-6 = 7
    x = np.clip(x, -7, 7)
    code, scale = mx.quantise(x, 8)
    assert (scale == 121).all()
    want = torch.tensor(x * 64).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(code, want)


@pytest.mark.parametrize("bits", (8, 4))
def test_ties_zeros_and_what_is_not_finite(bits):
    table = mx.elements(bits)[:(1 << (bits - 1)) - (bits == 8)]
    middle = (table[1:] + table[:-1]) / 2
    for i in range(0, len(middle), 31):
        part = middle[i:i + 31]
        x = np.zeros(32)
        x[0], x[1:1 + len(part)] = table[-1], -part
        code, scale = mx.quantise(x, bits)
        assert scale == 127
        half = 1 << (bits - 1)
        assert [c - half for c in code[1:1 + len(part)]] == \
            [j + j % 2 for j in range(i, i + len(part))]
    code, scale = mx.quantise(np.array([0.0, -0.0] * 16), bits)
    assert scale == 10 and code.tolist() == [0, 1 << (bits - 1)] * 16
    for bad in (np.nan, np.inf, -np.inf, 3.4e38):
        code, scale = mx.quantise(np.array([1.0] * 31 + [bad]), bits)
        assert scale == 255 and not code.any() and np.isnan(mx.values(code, scale, bits)).all()
    _, scale = mx.quantise(np.full(32, {8: 3.29e38, 4: 2.97e38}[bits]), bits)
    assert scale == {8: 247, 4: 253}[bits]


def test_packing():
    code = np.arange(64).astype(np.uint8) % 16
    assert mx.pack(code, 4)[:3].tolist() == [0x10, 0x32, 0x54]
    assert np.array_equal(mx.unpack(mx.pack(code, 4), 4), code)
