"""Keys and values in 8 or 4 bits (include/dsa3d_mx.h) in plain numpy and float64: the nearest
element is found by looking at all of them; used by the tests only."""
from __future__ import annotations

import numpy as np

BLOCK = 32
LEAST = -117                  # the least power of two that is written
LARGEST = {8: 448.0, 4: 6.0}
NOT_FINITE = 255


def elements(bits):
    """The element of each code; NaN where a code stands for none."""
    behind, bias = (3, 7) if bits == 8 else (1, 1)
    half = 1 << (bits - 1)
    x = np.zeros(2 * half)
    for c in range(2 * half):
        e, m = (c % half) >> behind, c & ((1 << behind) - 1)
        lead = 1 << behind if e else 0
        x[c] = (-1.0 if c >= half else 1.0) * (lead + m) * 2.0 ** (max(e, 1) - bias - behind)
    if bits == 8:
        x[0x7f] = x[0xff] = np.nan
    return x


def quantise(x, bits):
    """x [..., channels] -> (codes [..., channels], scale bytes [..., channels / 32]), uint8."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    table = elements(bits)[:(1 << (bits - 1)) - (bits == 8)]
    finite = np.isfinite(blocks).all(-1)
    size = np.where(finite[..., None], np.abs(blocks), 0.0)
    top = size.max(-1)
    power = np.full(top.shape, LEAST)
    for e in range(LEAST, 128):  # the least that holds the largest
        power = np.where(top > table[-1] * 2.0 ** e, e + 1, power)
    y = size / 2.0 ** power[..., None].astype(np.float64)
    above = np.clip(np.searchsorted(table, y), 0, len(table) - 1)
    below = np.maximum(above - 1, 0)
    up, down = table[above] - y, y - table[below]
    code = np.where((up < down) | ((up == down) & (above % 2 == 0)) | (above == 0), above, below)
    over = (table[code] * 2.0 ** power[..., None].astype(np.float64) >= 2.0 ** 128).any(-1)
    none = ~finite | over
    code = np.where(none[..., None], 0, code + (np.signbit(blocks).astype(int) << (bits - 1)))
    scale = np.where(none, NOT_FINITE, power + 127)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def values(codes, scales, bits):
    """What codes and scale bytes stand for, in float64."""
    power = np.where(scales == NOT_FINITE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return elements(bits)[codes] * np.repeat(power, BLOCK, -1)


def pack(codes, bits):
    """Codes as the cache holds them: two 4-bit ones to a byte, the even channel in its low half."""
    return codes if bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(held, bits):
    if bits == 8:
        return held
    return np.stack((held & 15, held >> 4), -1).reshape(*held.shape[:-1], -1)


def places(pages, held, lengths, page_size, num_pages):
    """(packed row, page, row of the page) of every new token that has a place."""
    at = 0
    for b, (n, m) in enumerate(zip(lengths, held)):
        for i in range(n):
            j = m - n + i
            if 0 <= j < pages.shape[1] * page_size and 0 <= pages[b, j // page_size] < num_pages:
                yield at + i, pages[b, j // page_size], j % page_size
        at += n
