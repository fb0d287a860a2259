"""The paged 4-bit cache's attention where neighbouring tokens are of very different sizes: what a row sees does not depend on tokens that it does not see, nor on tokens without weight."""
import math

import pytest
import torch

from tests._cache import HALF_STEP
from tests._cache4 import Setup4, attention_ref, check_attention, numbers, scales, word_of, zeros

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def enlarge(s, grid, i, token, log2):
    page, place = int(s.table[i, token // s.P]), token % s.P
    word = grid[page, :, place]
    grid[page, :, place] = word_of(scales(word) * 2.0 ** log2, zeros(word))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,group", [(128, 64, 2), (64, 16, 3), (64, 128, 16)])
@pytest.mark.parametrize("of", ["k_grid", "v_grid"])
@pytest.mark.parametrize("log2", [2, 5, 12, 18, 25, 60])
def test_rows_that_do_not_see_a_larger_token(dtype, D, P, group, of, log2):
    """Later tokens of a row's page, some in its sixteen neighbours, whose scales are 2^log2 times the others'.  The tolerance goes by what a row sees (attention_ref)."""
    s = Setup4(dtype, [200, 77, 130], 2, D, P, seed=60)
    for i, token in ((0, 100), (0, 149), (0, 198), (1, 76), (1, 40), (2, 129), (2, 112)):
        enlarge(s, getattr(s, of), i, token, log2)
    check_attention(s, [199, 60, 30], group)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("of", ["k_grid", "v_grid"])
@pytest.mark.parametrize("scale", [2.0 ** 119, 2.0 ** 121, 2.0 ** 127])
def test_rows_that_do_not_see_a_token_at_the_end_of_the_range(dtype, D, of, scale):
    s = Setup4(dtype, [90, 40], 1, D, 16, seed=61)
    q = s.rows(100, 4)
    out, ws = torch.zeros_like(q), s.cache.workspace(100, 4, 2, 60)
    getattr(s, of)[int(s.table[0, 4]), :, 7] = word_of(torch.tensor([scale]), torch.tensor([-3])).cuda()  # token 71, which row 41 of 0 .. 59 is
    s.cache.attention(q, s.ints([0, 60, 100]), s.ints([90, 40]), s.table, out, ws, 60)
    want, tol = attention_ref(s, q, [0, 60, 100], [90, 40], D ** -0.5)
    blind = torch.ones(100, dtype=torch.bool)
    blind[41:60] = False
    assert bool(((out.double().cpu() - want).abs() <= tol)[blind].all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])                              # the row kernel, the tile kernel
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("of", ["k_grid", "v_grid"])
@pytest.mark.parametrize("log2", [3, 6, 18, 25, 60])
def test_tokens_without_weight_beside_others(dtype, added, causal, of, log2):
    """Every key gives the same score but those of a few tokens, whose weights are under 2^-90: a row is the mean of the others' values, each in its own measure.

    Tolerance: weights half a step of binary16 of their own (2^-11; they are equal, and the values' scales lie within 2^6 of one another, so none is below the normal range) and 2^-16 for their
    exponents, which are below 128 before the reference is taken off (three roundings of 2^-18), the exponential and the quotient; the sums a rounding of 2^-23 for each 16 tokens; all of the values'
    sizes.  The row its rounding."""
    held = 300
    s = Setup4(dtype, [held], 2, 64, 16, seed=62)
    every = s.table[0, :(held + 15) // 16].long()
    s.k_grid[every] = word_of(torch.tensor([0.5]), torch.tensor([-5])).cuda()
    s.k_codes[every] = 10 * 17                                          # 2.5
    alone = [0, 37, 133, held - 41]
    for t in alone:
        page, place = int(s.table[0, t // 16]), t % 16
        s.k_codes[page, :, place] = 0                                   # -2.5, or less
        enlarge(s, getattr(s, of), 0, t, log2)
    q = (torch.rand((added, 4, 1), generator=s.g) + 2).to(dtype).expand(added, 4, 64).contiguous().cuda()
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(added, 4, 1, added)
    s.cache.attention(q, s.ints([0, added]), s.ints([held]), s.table, out, ws, added, scale=0.125, causal=causal)
    v = numbers(s.v_codes[every], s.v_grid[every]).transpose(0, 1).reshape(2, -1, 64)
    size = (scales(s.v_grid[every]).double() * (15 + zeros(s.v_grid[every]).abs())).transpose(0, 1).reshape(2, -1)
    for j in range(added):
        seen = [t for t in range(held - added + j + 1 if causal else held) if t not in alone]
        # 64 * 5 * (2 to 3) / 8 nats or more below the others: what the large ones add is 2^60 * 16 * 2^-115 at most
        for h in range(2):
            want, most = v[h, seen].mean(0), size[h, seen].mean() * (2.0 ** -11 + 2.0 ** -16 + (held / 16 + 8) * 2.0 ** -23)
            off = (out[j, 2 * h:2 * h + 2].double() - want).abs()
            assert bool((off <= most + HALF_STEP[dtype] * (want.abs() + most) + 2.0 ** -24).all()), (j, h, float(off.max()), float(most))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("log2", [7, 30])
def test_absent_pages_beside_large_tokens(dtype, added, causal, log2):
    s = Setup4(dtype, [300, 130], 2, 64, 16, seed=64)
    for i, token in ((0, 3), (0, 70), (0, 97), (1, 33), (1, 110)):
        enlarge(s, s.v_grid, i, token, log2)
        enlarge(s, s.k_grid, i, token, -log2)
    table = s.table.clone()
    table[0, 5], table[0, 7], table[0, 8:12], table[1, 3] = -1, s.pages, -1, -2 ** 31
    check_attention(s, [added, added], 3, table=table, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])
@pytest.mark.parametrize("of,bad", [("k_grid", math.nan), ("v_grid", math.nan), ("k_grid", math.inf), ("v_grid", math.inf)])
def test_a_scale_that_is_no_number_beside_large_tokens(dtype, added, of, bad):
    """The rows that see the token are NaN, and no others; its neighbours count as they do elsewhere."""
    s = Setup4(dtype, [200, 90], 2, 64, 16, seed=65)
    q = s.rows(2 * added, 4)
    first = 200 - added + added // 2                                    # the first request's row added // 2
    for token in (first - 3, first + 1, 20):
        if token < 200:
            enlarge(s, s.v_grid, 0, token, 9)
    getattr(s, of)[int(s.table[0, first // 16]), :, first % 16] = int(word_of(torch.tensor([bad]), torch.tensor([-7])))
    out, ws = torch.zeros_like(q), s.cache.workspace(2 * added, 4, 2, added)
    s.cache.attention(q, s.ints([0, added, 2 * added]), s.ints([200, 90]), s.table, out, ws, added)
    want, tol = attention_ref(s, q, [0, added, 2 * added], [200, 90], 64 ** -0.5)
    spoilt = torch.zeros(2 * added, dtype=torch.bool)
    spoilt[added // 2:added] = True
    got = out.double().cpu()
    assert bool(got[spoilt].isnan().all()) and bool(((got - want).abs() <= tol)[~spoilt].all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])
@pytest.mark.parametrize("log2", [-60, -20, None])
def test_a_token_of_zeros_that_has_nearly_all_the_weight(dtype, added, log2):
    """A token of zeros has 2^21.6 times the others' weight and a scale of 2^log2 (None: 0), which keeps its product with the weight near theirs or below: a row is what they add, each in its own measure.

    Tolerance: as above, by what each of them adds; the zeros count in the softmax's sum alone."""
    held, token = 300, 37
    s = Setup4(dtype, [held], 1, 64, 16, seed=67)
    every = s.table[0, :(held + 15) // 16].long()
    s.k_grid[every] = word_of(torch.tensor([0.5]), torch.tensor([-5])).cuda()
    s.k_codes[every] = 5 * 17                                           # 0
    s.v_grid[every] = word_of(scales(s.v_grid[every]) * (2.0 ** 12 if dtype == F16 else 1.0), zeros(s.v_grid[every]))  # rows in the type's normal range
    page, place = int(s.table[0, token // 16]), token % 16
    s.k_codes[page, :, place], s.v_codes[page, :, place] = 8 * 17, 0    # 1.5
    s.v_grid[page, :, place] = 0 if log2 is None else int(word_of(torch.tensor([2.0 ** log2]), torch.tensor([0])))
    q = torch.full((added, 3, 64), 1.25, dtype=dtype, device="cuda")    # scores of 15 and 0
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(added, 3, 1, added)
    s.cache.attention(q, s.ints([0, added]), s.ints([held]), s.table, out, ws, added, scale=0.125, causal=False)
    v = numbers(s.v_codes[every], s.v_grid[every])[:, 0].reshape(-1, 64)[:held]
    size = (scales(s.v_grid[every]).double() * (15 + zeros(s.v_grid[every]).abs()))[:, 0].reshape(-1)[:held]
    p = torch.ones(held, dtype=torch.float64, device="cuda")
    p[token] = math.exp(15.0)
    p /= p.sum()
    want, most = p @ v, (p @ size) * (2.0 ** -11 + 2.0 ** -16 + (held / 16 + 8) * 2.0 ** -23)
    assert bool(((out.double() - want).abs() <= most + HALF_STEP[dtype] * (want.abs() + most) + (2.0 ** -25 if dtype == F16 else 0.0)).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])
@pytest.mark.parametrize("log2_scale", [0, 18, 22, 30, 60])
def test_scores_far_from_zero_beside_small_keys(dtype, added, log2_scale):
    """One key is 2^6 times its neighbours and its score above theirs by more than 2^8: a row is that key's value, whose weight may be off by half a step of binary16."""
    held = 300
    s = Setup4(dtype, [held], 2, 64, 16, seed=66)
    every = s.table[0, :(held + 15) // 16].long()
    s.k_grid[every] = word_of(torch.tensor([2.0 ** -5]), torch.tensor([0])).cuda()
    s.k_codes[every] = 5 * 17
    for where in (0, 70, held - added):                                 # every row sees them; each is 16 times the one before
        page, place = int(s.table[0, where // 16]), where % 16
        s.k_grid[page, :, place] = word_of(torch.tensor([2.0 * 16.0 ** (where > 0) * 16.0 ** (where > 70)]), torch.tensor([0])).cuda()
        s.k_codes[page, :, place] = 15 * 17
        q = (torch.rand((added, 6, 1), generator=s.g) * 3 + 2).to(dtype).expand(added, 6, 64).contiguous().cuda()
        out = torch.full_like(q, 5.0)
        ws = s.cache.workspace(added, 6, 1, added)
        s.cache.attention(q, s.ints([0, added]), s.ints([held]), s.table, out, ws, added, scale=2.0 ** log2_scale)
        want = numbers(s.v_codes[page, :, place], s.v_grid[page, :, place]).repeat_interleave(3, 0)[None]
        size = (scales(s.v_grid[page, :, place]).double() * (15 + zeros(s.v_grid[page, :, place]).abs())).repeat_interleave(3, 0)[None, :, None]
        assert bool(((out.double() - want).abs() <= (HALF_STEP[dtype] + 2.0 ** -16) * want.abs() + 2.0 ** -10.9 * size + 2.0 ** -24).all()), where
