"""The 8-bit KV cache in 64 bits, from its definition, for the tests: which number a code stands for, and which code and exponent a
row of bf16 numbers gets (nearest of all 127 magnitudes, found by search)."""
import numpy as np

PAGE, D = 16, 128


def _magnitude(c):
    e, m = c >> 3, c & 7
    return m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)


MAGNITUDES = np.array([_magnitude(c) for c in range(127)])                   # ascending; 126 is 448
VALUES = np.concatenate([MAGNITUDES, [np.nan], -MAGNITUDES, [np.nan]])       # of the 256 codes


def quantize(x):
    """x [..., 128] float64 (bf16 numbers) -> codes uint8 [..., 128], exponents int8 [...]."""
    finite = np.isfinite(x)
    top = np.where(finite, np.abs(x), 0.0).max(-1)
    e = np.full(top.shape, -110)
    for k in range(-110, 121):                                               # the smallest that is large enough
        e = np.where((top > 448.0 * 2.0 ** k), k + 1, e)
    with np.errstate(invalid="ignore"):
        y = np.abs(x) / 2.0 ** e[..., None].astype(np.float64)
    y = np.where(np.isnan(y), 0.0, np.minimum(y, np.where(e == 120, 240.0, 448.0)[..., None]))
    hi = np.searchsorted(MAGNITUDES, y).clip(1, 126)
    below, above = y - MAGNITUDES[hi - 1], MAGNITUDES[hi] - y
    code = np.where((below < above) | ((below == above) & ((hi - 1) % 2 == 0)), hi - 1, hi)
    code = np.where(np.isnan(x), 127, code + 128 * (np.signbit(x) & ~np.isnan(x)))
    return code.astype(np.uint8), e.astype(np.int8)


def keys(codes, exponents):
    """codes [pages, Hkv, 16, 128], exponents [pages, Hkv, 2, 16] -> the keys' values."""
    return VALUES[codes] * np.exp2(exponents[:, :, 0, :, None].astype(np.float64))


def values(codes, exponents):
    return VALUES[codes] * np.exp2(exponents[:, :, 1, None, :].astype(np.float64))


def store(k, v, ex, page, slot, k_row, v_row):
    """Rows [Hkv, 128] of one token into codes and exponents (in place)."""
    k[page, :, slot, :], ex[page, :, 0, slot] = quantize(k_row)
    v[page, :, :, slot], ex[page, :, 1, slot] = quantize(v_row)
