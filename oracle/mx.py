"""The quantised rows of include/sangam_kvq.h written out with numpy in float64:
blocks of 32 dims, codes of e4m3 (8 bits) or e2m1 (4 bits) under a shared power
of two.

TEST INFRASTRUCTURE ONLY: nothing on the product path imports it.

The codes' values are listed one by one and a value goes to the nearest of
them, so that nothing here rounds by arithmetic.
"""
import numpy as np

BLOCK = 32
NAN_SCALE = 255
MIN_SCALE = 10


def code_values(fmt: str) -> np.ndarray:
    """Values of the codes without a sign bit, ascending (code = index)."""
    bits, exponents, bias = (3, 16, 7) if fmt == "e4m3" else (1, 4, 1)
    out = []
    for e in range(exponents):
        for f in range(1 << bits):
            frac = f / (1 << bits)
            out.append((1.0 + frac) * 2.0 ** (e - bias) if e > 0 else frac * 2.0 ** (1 - bias))
    return np.asarray(out[:-1] if fmt == "e4m3" else out)  # (the last e4m3 code is NaN)


def from_bf16(bits: np.ndarray) -> np.ndarray:
    with np.errstate(invalid="ignore"):  # (NaN patterns)
        return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16_exact(x: np.ndarray) -> np.ndarray:
    """bf16 bits of values that are bf16 numbers (or NaN); 2^128, which codes of
    values next to it can stand for, is infinity there."""
    x = np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)
    f = x.astype(np.float32)
    bits = f.view(np.uint32)
    out = np.where(np.isnan(f), 0x7FC0, bits >> 16).astype(np.uint16)
    assert np.array_equal(from_bf16(out), x, equal_nan=True)
    return out


def quantise(x: np.ndarray, fmt: str):
    """Codes (uint8: one per value, or two e2m1 codes, the even dim in the low
    half) and scale bytes of rows x [..., D] (float64)."""
    b = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, BLOCK))
    table = code_values(fmt)
    largest = np.abs(b).max(-1)  # NaN where the block holds one
    bad = ~np.isfinite(largest)
    takes = table[-1] * 2.0 ** (np.arange(MIN_SCALE, 255) - 127.0)  # the largest that each byte takes
    scale = MIN_SCALE + np.searchsorted(takes, np.where(bad, 0.0, largest), side="left")
    y = np.where(bad[..., None], 0.0, b) * 2.0 ** (127 - scale)[..., None]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(table, a, side="left"), 1, len(table) - 1)
    lo = hi - 1
    up, down = table[hi] - a, a - table[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == table[hi], hi, code)
    code = code + np.where(np.signbit(y), len(table) + (fmt == "e4m3"), 0)
    code = np.where(bad[..., None], 0, code).reshape(x.shape).astype(np.uint8)
    if fmt == "e2m1":
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    return code, np.where(bad, NAN_SCALE, scale).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    """What codes and scale bytes stand for, float64 [..., D]."""
    table = code_values(fmt)
    c = np.asarray(codes, np.int64)
    if fmt == "e2m1":
        c = np.stack([c & 15, c >> 4], -1).reshape(c.shape[:-1] + (-1,))
    else:
        table = np.append(table, np.nan)
    both = np.concatenate([table, -table])
    v = both[c].reshape(c.shape[:-1] + (-1, BLOCK))
    s = np.asarray(scales, np.int64)
    power = np.where(s == NAN_SCALE, np.nan, 2.0 ** (s - 127.0))
    return (v * power[..., None]).reshape(c.shape)
