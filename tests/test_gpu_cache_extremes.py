"""Attention over the paged 8-bit cache at the ends of its arguments' ranges."""
import math

import pytest
import torch

from tests._cache import HALF_STEP, Setup
from tests.test_gpu_cache import check_attention

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])
@pytest.mark.parametrize("log2_scale", [0, 10, 14, 18, 22, 30, 60, 100])
@pytest.mark.parametrize("winner,others,sign", [(127, 40, 1), (127, 40, -1), (60, 127, 1)])
def test_scores_far_from_zero(dtype, added, log2_scale, winner, others, sign):
    """One key's score is above the others' by more than 2^8 at any of these scales, at 60 against 127 with every score below zero: a row is that
    key's value.  The weight of it may be off by half a step of binary16, as all weights; where binary32 has no place left for fractions of a score,
    it still is the one weight."""
    held = 400
    s = Setup(dtype, [held], 2, 64, 16, seed=31)
    g = torch.Generator().manual_seed(5)
    every = s.table[0, :(held + 15) // 16].long()
    s.k_scale[every] = 0.031
    for where in [0, 70, 200, held - added]:                            # every row sees them
        s.k_codes[every] = -others if others > winner else torch.randint(-others, others, s.k_codes[every].shape, generator=g).to(torch.int8).cuda()
        s.k_codes[int(s.table[0, where // 16]), :, where % 16] = (-winner if others > winner else winner)
        q = torch.rand((added, 6, 1), generator=g) * 3 + 2              # each row in its own place of its binade
        q = (q * sign).to(dtype).expand(added, 6, 64).contiguous().cuda()
        out = torch.full_like(q, 5.0)
        ws = s.cache.workspace(added, 6, 1, added)
        s.cache.attention(q, s.ints([0, added]), s.ints([held]), s.table, out, ws, added, scale=sign * 2.0 ** log2_scale)
        page = int(s.table[0, where // 16])
        want = (s.v_codes[page, :, where % 16].double() * s.v_scale[page].double()[:, None]).repeat_interleave(3, 0)[None]
        assert bool(((out.double() - want).abs() <= (2.0 ** -11 + HALF_STEP[dtype] + 2.0 ** -16) * want.abs() + 2.0 ** -24).all()), (where, out[0, :, :4], want[0, :, :4])


@pytest.mark.parametrize("added", [1, 40])
def test_queries_below_bfloat16_s_normal_range(added):
    s = Setup(BF16, [130, 77], 2, 64, 16, seed=32)
    g = torch.Generator().manual_seed(6)
    q = (torch.randn((2 * added, 4, 64), generator=g, dtype=torch.float64) * 2.0 ** -128).to(BF16).cuda()
    assert 0.0 < float(q.double().abs().max()) < 2.0 ** -125
    check_attention(s, [added, added], 2, q=q, pad=0, scale=2.0 ** 127)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added,first", [(1, 322), (5, 320), (40, 304)])   # of the page, in the first request: its earlier rows do not see it
@pytest.mark.parametrize("of", ["k_scale", "v_scale"])
def test_a_page_whose_scale_is_no_number_spoils_the_rows_that_see_it(dtype, added, first, of):
    s = Setup(dtype, [323, 90], 2, 128, 16, seed=33)
    T = 2 * added
    q = s.rows(T, 6)
    args = (s.ints([0, added, T]), s.ints([323, 90]), s.table)
    ws = s.cache.workspace(T, 6, 2, added)
    clean, out = torch.zeros_like(q), torch.zeros_like(q)
    s.cache.attention(q, *args, clean, ws, added)
    getattr(s, of)[int(s.table[0, first // 16]), 1] = math.nan
    s.cache.attention(q, *args, out, ws, added)
    spoilt = torch.zeros((T, 6), dtype=torch.bool, device="cuda")
    spoilt[max(0, first - (323 - added)):added, 3:] = True
    assert torch.equal(out.isnan().all(-1), spoilt) and torch.equal(out.isnan().any(-1), spoilt) and torch.equal(out[~spoilt], clean[~spoilt])
