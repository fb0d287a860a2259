"""What the paged 4-bit cache gives back at the ends of the range: compared as it is, with infinities and NaN told apart from large numbers and zeros."""
import math

import pytest
import torch

from tests._cache4 import Setup4, numbers, scales, word_of

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def check(s, slots):
    """Every number to the bit; NaN where the definition has NaN and nowhere else."""
    slots = s.ints(slots)
    k, v = (torch.full((len(slots), s.H, s.D), 3.0, dtype=s.dtype, device="cuda") for _ in range(2))
    s.cache.load(slots, k, v)
    there = (slots >= 0) & (slots < s.pages * s.P)
    at, most = torch.where(there, slots, 0).long(), torch.finfo(s.dtype).max
    for got, codes, grid in ((k, s.k_codes, s.k_grid), (v, s.v_codes, s.v_grid)):
        want = numbers(codes[at // s.P, :, at % s.P], grid[at // s.P, :, at % s.P]).clamp(-most, most).to(s.dtype)
        want = torch.where(there[:, None, None], want, torch.zeros_like(want))
        none = want.isnan()
        assert torch.equal(got.isnan(), none) and not bool(got.isinf().any())
        assert torch.equal(got[~none], want[~none])
    return k, v


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_of_the_largest_numbers_come_back_finite(dtype, D):
    s = Setup4(dtype, [40], kv_heads=2, head_dim=D, page=16, seed=70)
    most = torch.finfo(dtype).max
    x = s.rows(40, 2)
    x[0], x[1] = most, -most                                            # in binary16: 128 * 512
    x[2], x[2, :, ::3] = most, -most
    x[3], x[3, :, 1] = most, 0.0
    slots = s.slots_of(0, 0, 40)
    s.cache.store(x, -x, s.ints(slots))
    k, v = check(s, slots)
    assert bool(k[:4].isfinite().all()) and bool(v[:4].isfinite().all())
    if dtype == F16:
        at = slots[0]
        assert float(scales(s.k_grid[at // 16, 0, at % 16])) == 512.0 and bool((k[0] == most).all()) and bool((k[1] == -most).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale,zero", [(2.0 ** 127, 100), (2.0 ** 127, -100), (2.0 ** 126, -8), (3.0 * 2.0 ** 126, -1), (512.0, 113), (65504 / 1000, 1000), (2.0 ** 60, -7), (math.inf, -7), (math.nan, 0)])
def test_scales_beyond_the_type(dtype, scale, zero):
    s = Setup4(dtype, [20], kv_heads=2, head_dim=64, page=16, seed=71)
    word = int(word_of(torch.tensor([scale]), torch.tensor([zero])))
    s.k_grid[int(s.table[0, 0]), :, 3:9], s.v_grid[int(s.table[0, 1]), 1, 2] = word, word
    check(s, s.slots_of(0, 0, 20))


def test_slots_outside_are_zero_and_rubbish_is_what_it_is():
    # pages that no request holds have NaN and infinite scales; none of them stands in for a slot outside the cache
    s = Setup4(F16, [20], kv_heads=1, head_dim=64, page=16, seed=72)
    for page in range(s.pages):
        s.k_grid[page], s.v_grid[page] = (int(word_of(torch.tensor([bad]), torch.tensor([5]))) for bad in (math.nan, math.inf))
    total = s.pages * s.P
    k, v = check(s, [-1, total, 0, total - 1, -2 ** 31, 2 ** 31 - 1, total + 5])
    assert bool((k[[0, 1, 4, 5, 6]] == 0).all()) and bool((v[[0, 1, 4, 5, 6]] == 0).all()) and bool(k[2].isnan().all()) and bool(k[3].isnan().all())
