"""The 4-bit store's rounding (nibbles_of in csrc/tsq_cache4.cu) on the CPU: one fused product and addition with an inverse that is 2^-20 too large gives round(x / s), halves away from zero, for
every 16-bit x and every scale of seven significant bits with |x / s| up to 128."""
import numpy as np
import pytest

f32 = np.float32
MAGIC = 12582912.0


def patterns(fmt):
    if fmt == "f16":
        return np.arange(1, 0x7c00, dtype=np.uint16).view(np.float16).astype(f32)
    return (np.arange(0x2000, 0x6000, dtype=np.uint32) << 16).view(f32)      # 2^-63 .. 2^64


def rounded(x, inverse):
    """fma(x, inverse, 1.5 * 2^23) less the addend: the exact product (35 bits) plus the addend is exact in long double, and is rounded once."""
    return (np.longdouble(x) * np.longdouble(inverse) + np.longdouble(MAGIC)).astype(f32).astype(np.float64) - MAGIC


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
@pytest.mark.parametrize("ulp", [-1, 0, 1])                                  # the reciprocal may be one unit off
def test_every_quotient(fmt, ulp):
    x = patterns(fmt)
    halves = 0
    for exponent in (-38, -24, -9, -1, 0, 5, 12):
        for m in range(64, 128):
            s = f32(m * 2.0 ** exponent / 128)
            inverse = ((f32(1) / s).view(np.int32) + ulp).view(f32) * f32(1 + 2.0 ** -20)
            quotient = x.astype(np.float64) / np.float64(s)                  # a half is exact here, and nothing else is near one
            use = x[quotient <= 128]
            want = np.floor(quotient[quotient <= 128] + 0.5)
            halves += int((quotient[quotient <= 128] % 1 == 0.5).sum())
            assert np.array_equal(rounded(use, inverse), want) and np.array_equal(rounded(-use, inverse), -want)
    assert halves > 1000


def test_nibbles_are_numbers_where_they_stand():
    """to_linear_bits (csrc/tsq_cache_device.cuh): the lower eleven bits of a binary16 number count in one unit, 2^-24, whether the eleventh is set or not."""
    n = np.arange(2048, dtype=np.uint16)
    assert np.array_equal(n.view(np.float16).astype(np.float64), n * 2.0 ** -24)
    words = np.arange(65536, dtype=np.uint32)
    for shifted, first in ((words << 3, 0), (words >> 5, 2)):
        for mask, unit, k in ((0x0078, 2.0 ** -21, first), (0x0780, 2.0 ** -17, first + 1)):
            got = (shifted & mask).astype(np.uint16).view(np.float16).astype(np.float64)
            assert np.array_equal(got, (words >> (4 * k) & 15) * unit)
