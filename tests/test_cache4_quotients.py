"""The 4-bit store's arithmetic (Grid4, nibbles_of in csrc/tsq_cache4.cu) in whole numbers on the CPU, with the zero-point in the addend and the codes cut off at 15."""
import numpy as np
import pytest

from tests._cache4 import store_ref

f32, i64 = np.float32, np.int64
MAGIC = 12582912


def test_how_near_a_quotient_comes_to_a_half():
    """x of eleven bits and s of seven, |x / s| up to 128: x / s is k + 1/2 or at least 1 / ((2 k + 1) times s's 7-bit number) of itself away, which is above 2^-15; an inverse that is between 2^-21 and
    2^-19 too large stays in front of it.  The nearest there is lies within 2^-14.9."""
    x, nearest = np.arange(1024, 2048, dtype=i64), 1.0
    for s in range(64, 128):
        for d in range(-11, 4):                                          # x / s = X / S * 2^d
            top, bottom = (x << d, i64(s)) if d >= 0 else (x, i64(s) << -d)
            odd = 2 * (top // bottom) + 1                                # of the half that follows the quotient's whole part: x / s against odd / 2
            off = np.abs(2 * top - odd * bottom)
            use = (top <= 128 * bottom) & (off > 0)
            nearest = min(nearest, float((off[use] / (odd * bottom)[use]).min(initial=1.0)))
    assert 2.0 ** -15 < nearest < 2.0 ** -14.9


@pytest.mark.parametrize("ulp", [-1, 0, 1])                              # the reciprocal may be one unit off
@pytest.mark.parametrize("zero", [-128, -127, -15, -8, 0, 1, 20, 128])
def test_one_fused_operation_for_every_quotient(zero, ulp):
    """fma(x, inverse, magic - zero) = magic + round(x / s) - zero for both signs of x.  Only the numbers of x and s and the difference of their exponents count: powers of two go through the
    reciprocal, the products and the fused operation unchanged (scales are 2^-40 to 2^124, inverses normal numbers), and quotients below a sixteenth round to 0 beside the addend.  In whole
    numbers: the product has 35 bits and the addend is a whole number, so the sum is rounded once, halves to even."""
    x = np.arange(1024, 2048, dtype=i64)                                 # binary16's; bfloat16's eight bits are among them
    for s in range(64, 128):
        inverse = ((f32(1) / f32(s)).view(np.int32) + ulp).view(f32) * f32(1 + 2.0 ** -20)
        fraction, power = np.frexp(inverse)
        number, power = i64(fraction * f32(2 ** 24)), int(power) - 24    # inverse = number * 2^power
        for d in range(-7, 4):
            # |x / s| = x * 2^d / s, up to 128
            top, bottom = (x << d, i64(s)) if d >= 0 else (x, i64(s) << -d)
            use = top <= 128 * bottom
            quotient = (2 * top + bottom) // (2 * bottom)                # rounded, halves up
            shift = -(power + d)
            for sign in (1, -1):
                exact = (i64(MAGIC - zero) << shift) + sign * x * number
                down = exact >> shift
                rest = exact - (down << shift)
                half = i64(1) << (shift - 1)
                got = down + ((rest > half) | ((rest == half) & (down % 2 == 1)))
                assert np.array_equal(got[use] - MAGIC, (sign * quotient - zero)[use])
                assert (got[use] >= 1 << 23).all() and (got[use] < 1 << 24).all()


def codes_of(x):
    """Rows of finite numbers within 2^126 as store4_kernel has them, binary32 throughout, packed codes taken from the low halves of the sums."""
    lo, hi = x.min(-1), x.max(-1)
    step = np.maximum(np.maximum((hi - lo).astype(f32) / f32(15), np.maximum(np.abs(lo), np.abs(hi)) * f32(0.0078125)), f32(2.0 ** -40))
    bits = (step.view(np.int32) + 0x1ffff) & ~0x1ffff
    inverse = (f32(1) / bits.view(f32)) * f32(1 + 2.0 ** -20)
    fused = lambda a, b, c: (np.longdouble(a) * np.longdouble(b) + np.longdouble(c)).astype(f32)  # noqa: E731
    zero = fused(lo, inverse, f32(MAGIC)) - f32(MAGIC)
    sums = fused(x, inverse[:, None], (f32(MAGIC) - zero)[:, None])
    code = np.minimum(sums.view(np.int32) & 0xffff, 15).astype(np.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, (bits.view(np.uint32) >> 16 | (zero.astype(np.int32).view(np.uint32) << 16)).view(np.int32)


@pytest.mark.parametrize("fmt", ["f16", "bf16"])
def test_whole_rows(fmt):
    """Ranges on both sides of 0, above and below it, of one number, of numbers half a step from a code; scales over the type's whole range."""
    r = np.random.default_rng(7)
    rows = r.standard_normal((4000, 64))
    rows[1000:2000] += 8 * r.standard_normal((1000, 1))
    rows[2000:2500] = rows[2000:2500, :1]
    rows[2500:3000] = r.integers(-40, 41, (500, 64)) * (r.integers(64, 128, (500, 1)) / 2.0)
    rows *= 2.0 ** r.integers(*((-14, 11) if fmt == "f16" else (-40, 117)), (4000, 1))
    with np.errstate(over="ignore"):
        x = np.clip(rows, -65504, 65504).astype(np.float16).astype(f32) if fmt == "f16" else (rows.astype(f32).view(np.uint32) & np.uint32(0xffff0000)).view(f32)
    x = x[np.abs(x).max(-1) <= 2.0 ** 126]                               # rows with larger numbers go another way (nibbles_of_any)
    assert len(x) > 3900
    codes, words = codes_of(x)
    want_codes, want_words = store_ref(x)
    assert np.array_equal(words, want_words) and np.array_equal(codes, want_codes)
    assert len(np.unique(words >> 16)) > 100 and (codes & 15 == 15).any()
