"""The paged 4-bit cache on the GPU against plain references: store and load (to the bit), attention and cross attention (64 bits)."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2511_04002_b200 import binding as B
from tests._cache import HALF_STEP
from tests._cache4 import Setup4, attention_ref, check_attention, numbers, scales, store_ref, word_of, zeros

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


# ---- store and load ----

def check_store(s, x_k, x_v, slots):
    want = []
    for codes, grid, x in ((s.k_codes, s.k_grid, x_k), (s.v_codes, s.v_grid, x_v)):
        c, w = codes.cpu().numpy().copy(), grid.cpu().numpy().copy()
        new_c, new_w = store_ref(x.float().cpu().numpy())
        for t, slot in enumerate(slots):
            if 0 <= slot < s.pages * s.P:
                c[slot // s.P, :, slot % s.P], w[slot // s.P, :, slot % s.P] = new_c[t], new_w[t]
        want.append((c, w))
    s.cache.store(x_k, x_v, s.ints(slots))
    for (c, w), codes, grid in zip(want, (s.k_codes, s.v_codes), (s.k_grid, s.v_grid)):
        assert np.array_equal(grid.cpu().numpy(), w)
        assert np.array_equal(codes.cpu().numpy(), c)


def check_load(s, slots, into=None):
    slots = s.ints(slots)
    k, v = into or (torch.full((len(slots), s.H, s.D), 3.0, dtype=s.dtype, device="cuda") for _ in range(2))
    s.cache.load(slots, k, v)
    there = (slots >= 0) & (slots < s.pages * s.P)
    at = torch.where(there, slots, 0).long()
    most = torch.finfo(s.dtype).max
    for got, codes, grid in ((k, s.k_codes, s.k_grid), (v, s.v_codes, s.v_grid)):
        want = numbers(codes[at // s.P, :, at % s.P], grid[at // s.P, :, at % s.P]).clamp(-most, most).to(s.dtype)   # exact in 64 bits, and in 32
        want = torch.where(there[:, None, None], want, torch.zeros_like(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    return k, v


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_store_and_load(dtype, D, P):
    s = Setup4(dtype, [1, 2 * P, 3 * P + 5, 40, 300], kv_heads=3, head_dim=D, page=P, seed=P + D)
    slots = []
    for i, lo, hi in [(0, 0, 1), (1, 0, 2 * P), (2, P - 3, 3 * P + 5), (3, 33, 40), (4, 7, 300)]:
        slots += s.slots_of(i, lo, hi) + [-1, s.pages * P + 4]
    random.Random(P).shuffle(slots)                                     # rows go by themselves
    x_k, x_v = s.rows(len(slots), 3), s.rows(len(slots), 3, 0.2)
    x_k[5:9] *= 20.0
    x_v[9:30] += 3.0                                                    # ranges that do not reach 0
    x_v[30:40] -= 50.0
    check_store(s, x_k, x_v, slots)
    check_load(s, slots + list(reversed(slots)))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 2000])
def test_store_and_load_of_every_kind_of_block(dtype, tokens):
    s = Setup4(dtype, [2100], kv_heads=5, head_dim=64 if tokens % 2 else 128, page=32, seed=tokens)
    slots = s.slots_of(0, 2100 - tokens, 2100)
    check_store(s, s.rows(tokens, 5), s.rows(tokens, 5), slots)
    check_load(s, slots)


@pytest.mark.parametrize("H,D", [(1, 64), (17, 128), (131, 128), (40, 64)])
def test_store_and_load_of_many_heads(H, D):
    s = Setup4(BF16, [70, 9], kv_heads=H, head_dim=D, page=16, seed=H)
    slots = s.slots_of(0, 3, 70) + [-1] + s.slots_of(1, 0, 9)
    check_store(s, s.rows(len(slots), H), s.rows(len(slots), H), slots)
    check_load(s, slots[::-1] * 2)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_store_of_values_that_are_no_numbers_zeros_and_extremes(dtype, D):
    s = Setup4(dtype, [90], kv_heads=2, head_dim=D, page=16, seed=5)
    x = s.rows(90, 2)
    x[0, 0, 3], x[1, 1, 5], x[2, 0, 7] = math.nan, math.inf, -math.inf
    x[3, 0, :], x[4, 1, :], x[5, 0, :] = math.nan, math.inf, -math.inf  # rows without a finite number
    x[6, 0, ::2], x[6, 0, 1::2] = math.inf, -math.inf
    x[16:20] = 0.0
    x[20:24] = -0.0
    x[24] = 5.0                                                         # one number throughout
    x[25] = -1.0 / 3
    x[26], x[26, :, D // 2] = 7.0, 7.03125
    most = torch.finfo(dtype).max
    x[30] = most
    x[31], x[31, :, ::3] = most, -most                                  # a range that binary32 does not hold, in bfloat16
    x[32, :, 1] = most
    x[33, :, 2] = -most
    x[34], x[34, 0, 5] = most, math.nan
    x[40:44] = torch.finfo(dtype).tiny
    x[44], x[44, :, 0] = torch.finfo(dtype).smallest_normal * 2.0 ** -5, 0.0
    x[45:50] *= 2.0 ** -10
    check_store(s, x, -x, s.slots_of(0, 0, 90))
    check_load(s, s.slots_of(0, 0, 90))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_store_of_halves(dtype):
    # numbers that lie exactly between two codes: odd multiples of half a scale, which the ends of the range set
    s = Setup4(dtype, [300], kv_heads=2, head_dim=64, page=64, seed=6)
    half = torch.randint(64, 128, (300, 2, 1), generator=s.g).float() * torch.exp2(torch.randint(-14, 2, (300, 2, 1), generator=s.g).float()) / 2
    lo = -torch.randint(0, 16, (300, 2, 1), generator=s.g)
    x = (torch.randint(0, 31, (300, 2, 64), generator=s.g) + 2 * lo) * half
    x[..., :1], x[..., 1:2] = 2 * lo * half, (2 * lo + 30) * half
    x = x.to(dtype).cuda()
    exact = (x.double().cpu() / (2 * half)) % 1
    assert float((exact == 0.5).float().mean()) > 0.1
    check_store(s, x, -x, s.slots_of(0, 0, 300))


def test_what_is_stored_is_within_half_a_step():
    s = Setup4(BF16, [500], kv_heads=4, head_dim=128, page=64, seed=7)
    x, slots = s.rows(500, 4, 2.0), s.slots_of(0, 0, 500)
    s.cache.store(x, x, s.ints(slots))
    at = s.ints(slots).long()
    step = scales(s.k_grid[at // 64, :, at % 64]).double()[..., None]
    off = (numbers(s.k_codes[at // 64, :, at % 64], s.k_grid[at // 64, :, at % 64]) - x.double()).abs()
    # the zero-point is a whole number of steps: the largest number may lie half a step past the last code's half
    assert bool((off <= step).all()) and float((off > 0.5 * step).float().mean()) < 0.01


@pytest.mark.parametrize("D", [64, 128])
def test_rows_inside_wider_tensors_and_between_32_byte_boundaries(D):
    s = Setup4(F16, [90], kv_heads=3, head_dim=D, page=16, seed=8)
    slots = s.slots_of(0, 0, 90)
    wide = s.rows(90, 3 + 3 + 2)
    check_store(s, wide[:, 3:6], wide[:, :3], slots)
    into, v = s.rows(90, 8), torch.zeros((90, 3, D), dtype=F16, device="cuda")
    before = into.clone()
    check_load(s, slots, (into[:, 4:7], v))
    assert torch.equal(into[:, :4], before[:, :4]) and torch.equal(into[:, 7:], before[:, 7:])
    one, two = (torch.zeros(90 * 3 * D + 16, dtype=F16, device="cuda") for _ in range(2))
    k, v = one[8:8 + 90 * 3 * D].view(90, 3, D), two[16:].view(90, 3, D)
    k.copy_(wide[:, :3])
    check_store(s, k, wide[:, 2:5], slots)
    check_load(s, slots, (k, v))
    assert bool((one[:8] == 0).all()) and bool((one[8 + 90 * 3 * D:] == 0).all()) and bool((two[:16] == 0).all())


def test_a_scale_that_is_no_number_is_read_back_as_none():
    s = Setup4(F16, [20], kv_heads=1, head_dim=64, page=16, seed=9)
    slot = s.slots_of(0, 3, 4)[0]
    s.k_grid[slot // 16, 0, slot % 16] = int(word_of(torch.tensor([math.nan]), torch.tensor([-3])))
    k, v = torch.zeros((20, 1, 64), dtype=F16, device="cuda"), torch.zeros((20, 1, 64), dtype=F16, device="cuda")
    s.cache.load(s.ints(s.slots_of(0, 0, 20)), k, v)
    assert bool(k[3].isnan().all()) and bool(k[:3].isfinite().all()) and bool(k[4:].isfinite().all()) and bool(v.isfinite().all())


# ---- attention ----

@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group", [(64, 16, 2, 1), (128, 64, 2, 4), (128, 16, 1, 7), (64, 128, 3, 16), (128, 32, 5, 2), (64, 64, 1, 3)])
def test_attention_of_single_tokens(causal, dtype, D, P, H, group):
    held = [1, 2, P - 1, P, P + 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 1027]
    check_attention(Setup4(dtype, held, H, D, P, seed=H), [1] * len(held), group, causal=causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,added", [(128, 64, 2, 4, [1, 4, 0, 2, 3]), (64, 16, 2, 8, [2, 1, 1, 0, 2]), (128, 16, 3, 5, [3, 3, 1, 2, 3]),
                                               (128, 128, 1, 1, [16, 9, 13, 1, 0]), (64, 32, 2, 7, [2, 2, 2, 1, 2])])
def test_attention_of_drafted_tokens(causal, dtype, D, P, H, group, added):
    check_attention(Setup4(dtype, [16, 700, 33, 129, 2100], H, D, P, seed=group), added, group, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,added", [(128, 64, 2, 8, [6, 5, 1, 3, 6]), (64, 16, 1, 16, [3, 2, 1, 0, 3]), (128, 16, 1, 3, [16, 9, 13, 11, 7]), (64, 128, 2, 1, [16, 33, 48, 17, 1]),
                                               (128, 32, 2, 7, [7, 7, 1, 2, 7]), (64, 64, 1, 49, [1, 1, 1, 1, 1])])
def test_attention_around_the_most_rows_of_the_row_kernel(dtype, D, P, H, group, added):
    # 48 rows in tiles of 16, the last one full or not; 49
    check_attention(Setup4(dtype, [16, 700, 50, 129, 2100], H, D, P, seed=group), added, group)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,held,added", [
    (128, 64, 1, 4, [300], [300]), (64, 16, 2, 1, [129, 128, 127], [129, 100, 1]), (128, 32, 2, 7, [500, 37, 1, 260], [30, 37, 1, 0]),
    (64, 128, 1, 64, [90, 400], [20, 5]), (128, 16, 1, 33, [64, 257], [9, 17]), (128, 128, 2, 2, [1500], [40]), (64, 64, 3, 16, [200, 641], [70, 129])])
def test_attention_of_prompts(causal, dtype, D, P, H, group, held, added):
    check_attention(Setup4(dtype, held, H, D, P, seed=D), added, group, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [[1, 1, 1, 1], [3, 2, 1, 3], [200, 50, 90, 3]])
def test_cross_attention_of_more_rows_than_states(dtype, added):
    # a request without states: its rows are zero
    out = check_attention(Setup4(dtype, [40, 0, 77, 1], 2, 64, 16, seed=10), added, 3, causal=False)
    assert bool((out[added[0]:added[0] + added[1]] == 0).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("added", [[3, 1, 2, 2], [40, 20, 70, 33]])
def test_rows_that_see_nothing_are_zero(causal, added):
    # more rows than tokens, no tokens at all, a table without pages
    s = Setup4(BF16, [40, 40, 80, 40], 2, 128, 16, seed=8)
    table = s.table.clone()
    table[3] = -1
    out = check_attention(s, added, 4, lengths=[2, 0, 80, 40], table=table, causal=causal)
    assert bool((out[added[0]:added[0] + added[1]] == 0).all()) and bool((out[sum(added[:3]):sum(added)] == 0).all())
    assert bool((out[0] == 0).all()) == causal


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("added", [1, 50])
@pytest.mark.parametrize("P", [16, 32])
def test_pages_outside_the_cache_are_not_seen(causal, added, P):
    s = Setup4(F16, [400, 200], 2, 64, P, seed=9)
    table = s.table.clone()
    table[0, 3], table[0, 7], table[1, 0], table[1, 6] = -1, s.pages, -2 ** 31, 2 ** 31 - 1
    table[0, 10:12] = -1                                                # a whole step of the row kernel
    check_attention(s, [added, added], 2, table=table, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("added", [1, 5, 40, 150])
def test_rows_of_requests_longer_than_their_table(dtype, causal, added):
    # the table ends at 80, 80 and 64 keys; positions go by the whole length
    s = Setup4(dtype, [170, 100, 64], 2, 64, 16, seed=43)
    check_attention(s, [added, min(added, 100), min(added, 64)], 3, table=s.table[:, :5].contiguous(), causal=causal)


@pytest.mark.parametrize("added", [1, 40])
def test_a_table_without_entries(added):
    s = Setup4(F16, [100], 1, 64, 16, seed=26)
    q = s.rows(added, 2)
    out = torch.full_like(q, 5.0)
    s.cache.attention(q, s.ints([0, added]), s.ints([100]), s.table[:, :0].contiguous(), out, s.cache.workspace(added, 2, 1, added), added)
    assert bool((out == 0).all())


@pytest.mark.parametrize("causal", [True, False])
def test_rows_past_max_query_are_left_alone(causal):
    s = Setup4(F16, [100, 64], 1, 64, 16, seed=11)
    q = s.rows(60, 2)
    part = torch.full_like(q, 5.0)
    ws = s.cache.workspace(60, 2, 2, 40)
    s.cache.attention(q, s.ints([0, 40, 60]), s.ints([100, 64]), s.table, part, ws, 30, causal=causal)
    want, tol = attention_ref(s, q, [0, 40, 60], [100, 64], 64 ** -0.5, causal)
    same = [t for t in range(60) if t < 30 or t >= 40]
    assert bool(((part.double().cpu() - want).abs() <= tol)[same].all()) and bool((part[30:40] == 5.0).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 33])
def test_large_and_small_queries_scales_and_a_negative_factor(dtype, added):
    s = Setup4(dtype, [130, 77], 2, 128, 32, seed=12)
    tokens = 2 * added
    q = s.rows(tokens, 4)
    q *= torch.exp2(torch.arange(tokens * 4, device="cuda").view(tokens, 4, 1) % 9 - 6.0).to(dtype)
    q[0, 0] = 0.0
    check_attention(s, [added, added], 2, q=q, pad=0)
    check_attention(s, [added, added], 2, q=q, pad=0, scale=-0.3)
    check_attention(s, [added, added], 2, q=q, pad=0, scale=0.0)
    page = int(s.table[0, 1])                                           # tokens side by side whose numbers are of very different sizes
    s.v_grid[page] = word_of(scales(s.v_grid[page]) * torch.exp2(torch.arange(32, device="cuda") % 16 - 8.0), zeros(s.v_grid[page]))
    s.k_grid[page] = word_of(scales(s.k_grid[page]) * torch.exp2(-(torch.arange(32, device="cuda") % 12.0)), zeros(s.k_grid[page]))
    s.v_grid[int(s.table[0, 2])] = word_of(torch.zeros(1), torch.tensor([-4])).cuda()
    s.k_grid[int(s.table[1, 0])] = word_of(torch.zeros(1), torch.tensor([-4])).cuda()
    check_attention(s, [added, added], 2, q=q, pad=0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 33])
@pytest.mark.parametrize("zero", [(0, 1), (-15, -14), (20, 100), (-128, 129), (-1000, 1001)])
def test_zero_points_anywhere(dtype, added, zero):
    # ranges that do not reach 0: codes' sums and the zero-points' cancel, operands are rounded
    check_attention(Setup4(dtype, [130, 77, 260], 2, 64, 16, seed=14, zero=zero), [added] * 3, 2, scale=0.125 / (1 + max(abs(z) for z in zero)))


@pytest.mark.parametrize("added", [1, 5, 60])
def test_tokens_of_zeros_and_of_one_number(added):
    # stored: pages of zeros, tokens of one number throughout, tokens of tiny and of large numbers side by side
    s = Setup4(BF16, [200, 90], 2, 64, 16, seed=15)
    slots = s.slots_of(0, 0, 200) + s.slots_of(1, 0, 90)
    k, v = s.rows(290, 2), s.rows(290, 2)
    k[16:48], v[32:64] = 0.0, 0.0
    v[70], v[71], k[72], v[200], k[201] = 5.0, -0.001, 3.0, 0.0, 0.0
    v[80:90] *= 2.0 ** -12
    v[85] *= 2.0 ** 16
    check_store(s, k, v, slots)
    check_attention(s, [added, added], 3)
    check_attention(s, [added, added], 3, causal=False)


@pytest.mark.parametrize("added", [1, 33])
@pytest.mark.parametrize("log2_k,log2_v", [(-30, 100), (20, -38), (60, 60), (-20, -20)])
def test_scales_far_from_one(added, log2_k, log2_v):
    s = Setup4(BF16, [300, 77], 2, 128, 32, seed=16)
    used = s.table[0, :10].long()
    s.k_grid[used], s.v_grid[used] = word_of(scales(s.k_grid[used]) * 2.0 ** log2_k, zeros(s.k_grid[used])), word_of(scales(s.v_grid[used]) * 2.0 ** log2_v, zeros(s.v_grid[used]))
    tail = int(s.table[0, 9])                                           # its places behind the request stay rubbish
    s.k_grid[tail, :, 300 % 32:] = int(word_of(torch.tensor([math.nan]), torch.tensor([5])))
    s.v_grid[tail, :, 300 % 32:] = int(word_of(torch.tensor([math.inf]), torch.tensor([5])))
    check_attention(s, [added, added], 2, scale=128 ** -0.5 * 2.0 ** -max(log2_k, 0))


@pytest.mark.parametrize("added", [1, 33])
def test_a_query_that_is_no_number_spoils_its_own_row_alone(added):
    s = Setup4(BF16, [130, 77], 2, 64, 16, seed=13)
    q = s.rows(2 * added, 8)
    ws = s.cache.workspace(2 * added, 8, 2, added)
    args = (s.ints([0, added, 2 * added]), s.ints([130, 77]), s.table)
    clean, out = torch.zeros_like(q), torch.zeros_like(q)
    s.cache.attention(q, *args, clean, ws, added)
    q[0, 1, 5], q[added, 6, 0] = math.nan, math.inf
    s.cache.attention(q, *args, out, ws, added)
    want = torch.zeros((2 * added, 8), dtype=torch.bool, device="cuda")
    want[0, 1] = want[added, 6] = True
    assert torch.equal(out.isnan().any(-1), want) and torch.equal(out[~want], clean[~want])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added,first", [(1, 322), (5, 320), (40, 304)])  # the token: the first request's earlier rows do not see it
@pytest.mark.parametrize("of", ["k_grid", "v_grid"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_token_whose_scale_is_no_number_spoils_the_rows_that_see_it(dtype, added, first, of, bad):
    s = Setup4(dtype, [323, 90], 2, 128, 16, seed=33)
    T = 2 * added
    q = s.rows(T, 6)
    args = (s.ints([0, added, T]), s.ints([323, 90]), s.table)
    ws = s.cache.workspace(T, 6, 2, added)
    clean, out = torch.zeros_like(q), torch.zeros_like(q)
    s.cache.attention(q, *args, clean, ws, added)
    getattr(s, of)[int(s.table[0, first // 16]), 1, first % 16] = int(word_of(torch.tensor([bad]), torch.tensor([-7])))
    s.cache.attention(q, *args, out, ws, added)
    spoilt = torch.zeros((T, 6), dtype=torch.bool, device="cuda")
    spoilt[max(0, first - (323 - added)):added, 3:] = True
    assert torch.equal(out.isnan().all(-1), spoilt) and torch.equal(out.isnan().any(-1), spoilt)
    want, tol = attention_ref(s, q, [0, added, T], [323, 90], 128 ** -0.5)
    rest = ~spoilt.cpu()
    assert bool(((out.double().cpu() - clean.double().cpu()).abs() <= 2 * tol.nan_to_num(posinf=0.0))[rest].all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])
@pytest.mark.parametrize("log2_scale", [0, 10, 18, 22, 30, 60, 90])
@pytest.mark.parametrize("winner,others,sign", [(15, 5, 1), (15, 5, -1), (2, 14, 1)])
def test_scores_far_from_zero(dtype, added, log2_scale, winner, others, sign):
    """One key's score is above the others' by more than 2^8 at any of these scales: a row is that key's value, whose weight may be off by half a step of binary16."""
    held = 400
    s = Setup4(dtype, [held], 2, 64, 16, seed=31)
    g = torch.Generator().manual_seed(5)
    every = s.table[0, :(held + 15) // 16].long()
    for where in [0, 70, 200, held - added]:                            # every row sees them
        zero = 0 if others < winner else -15                            # keys above 0, or below
        s.k_grid[every] = word_of(torch.tensor([0.5]), torch.tensor([zero])).cuda()
        s.k_codes[every] = others * 17
        page, place = int(s.table[0, where // 16]), where % 16
        s.k_codes[page, :, place] = winner * 17
        q = torch.rand((added, 6, 1), generator=g) * 3 + 2              # each row in its own place of its binade
        if zero:
            q = -q                                                      # (2 - 15) against (14 - 15): the larger magnitude wins
        q = (q * sign).to(dtype).expand(added, 6, 64).contiguous().cuda()
        out = torch.full_like(q, 5.0)
        ws = s.cache.workspace(added, 6, 1, added)
        s.cache.attention(q, s.ints([0, added]), s.ints([held]), s.table, out, ws, added, scale=sign * 2.0 ** log2_scale)
        want = numbers(s.v_codes[page, :, place], s.v_grid[page, :, place]).repeat_interleave(3, 0)[None]
        size = (scales(s.v_grid[page, :, place]).double() * (15 + zeros(s.v_grid[page, :, place]).abs())).repeat_interleave(3, 0)[None, :, None]
        assert bool(((out.double() - want).abs() <= (HALF_STEP[dtype] + 2.0 ** -16) * want.abs() + 2.0 ** -10.9 * size + 2.0 ** -24).all()), where


@pytest.mark.parametrize("added", [1, 40])
def test_queries_below_bfloat16_s_normal_range(added):
    s = Setup4(BF16, [130, 77], 2, 64, 16, seed=32)
    q = (torch.randn((2 * added, 4, 64), generator=s.g, dtype=torch.float64) * 2.0 ** -128).to(BF16).cuda()
    assert 0.0 < float(q.double().abs().max()) < 2.0 ** -125
    check_attention(s, [added, added], 2, q=q, pad=0, scale=2.0 ** 125)


@pytest.mark.parametrize("added", [1, 5, 40])
def test_queries_and_rows_inside_wider_tensors(added):
    s = Setup4(F16, [90, 200], 2, 64, 16, seed=14)
    T = 2 * added
    wide, into = s.rows(T, 12), s.rows(T, 10)
    before = into.clone()
    ws = s.cache.workspace(T, 4, 2, added)
    args = (s.ints([0, added, T]), s.ints([90, 200]), s.table)
    want = torch.zeros((T, 4, 64), dtype=F16, device="cuda")
    s.cache.attention(wide[:, 3:7].contiguous(), *args, want, ws, added)
    s.cache.attention(wide[:, 3:7], *args, into[:, 5:9], ws, added)
    assert torch.equal(into[:, 5:9], want) and torch.equal(into[:, :5], before[:, :5]) and torch.equal(into[:, 9:], before[:, 9:])


# ---- shares ----

def check_parts(dtype, held, added, D, P, H, group, causal=True):
    """Every key has the same weight and every stretch of 32 tokens its own mark in the values (one number that is not 0), so that a part that is lost or counted twice shows in the row.  Weights
    are 1 and the sums whole numbers below 2^24, so exact; the quotient and its product take a rounding of binary32 each, the row one of its type, with its subnormal numbers' half step."""
    s = Setup4(dtype, held, H, D, P, seed=sum(held) % 1000)
    pages = [s.table[i, :(n + P - 1) // P].long() for i, n in enumerate(held)]
    for mine in pages:
        s.v_grid[mine] = word_of(torch.tensor([0.5]), torch.tensor([0])).cuda()
        unit = torch.arange(mine.numel() * P, device="cuda") // 32
        for h in range(H):
            code = torch.zeros((unit.numel(), D), dtype=torch.uint8, device="cuda")
            code[torch.arange(unit.numel()), (unit + 3 * h) % D] = (1 + unit // D % 15).to(torch.uint8)
            s.v_codes[mine, h] = (code[:, 0::2] | code[:, 1::2] << 4).view(mine.numel(), P, D // 2)
    T = sum(added)
    starts = [sum(added[:i]) for i in range(len(added) + 1)]
    q = s.rows(T, H * group)
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(T, H * group, len(added), max(added))
    s.cache.attention(q, s.ints(starts), s.ints(held), s.table, out, ws, max(added), scale=0.0, causal=causal)
    want = torch.zeros((T, H * group, D), dtype=torch.float64)
    t = 0
    for n, a in zip(held, added):
        unit = torch.arange(n) // 32
        value = (1 + unit // D % 15).double() * 0.5
        for j in range(a):
            see = n - a + j + 1 if causal else n
            for h in range(H):
                sums = torch.bincount((unit[:see] + 3 * h) % D, weights=value[:see], minlength=D)
                want[t, h * group:(h + 1) * group] = sums / max(see, 1)
            t += 1
    off = (out.double().cpu() - want).abs()
    assert bool((off <= (HALF_STEP[dtype] + 2.0 ** -22) * want + 2.0 ** -25).all()), float((off / want.clamp(min=2.0 ** -14)).max())
    assert s.cache.workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added,group", [(1, 1), (4, 5), (3, 16)])
@pytest.mark.parametrize("keys", [128 * n + more for n, more in ((6, 1), (13, 128), (14, 3), (15, 17), (252, 64), (253, 1), (254, 95), (255, 128), (470, 2), (625, 0), (1700, 9))])
def test_parts_of_one_tile_of_few_rows(dtype, added, group, keys):
    check_parts(dtype, [keys], [added], 128 if keys % 2 else 64, 64, 1, group)


@pytest.mark.parametrize("added,group", [(9, 8), (300, 1), (5, 64)])
@pytest.mark.parametrize("keys", [400, 1280, 1413, 5000, 40000])
def test_parts_of_tiles_of_many_rows(added, group, keys):
    check_parts(BF16, [keys], [added], 128 if keys % 2 else 64, 32, 1, group, causal=keys != 5000)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,held,added", [
    (64, 16, 2, 3, [9000, 1, 130, 0, 20000, 64], [1, 1, 1, 0, 1, 1]), (128, 64, 5, 1, [3000, 7000, 65], [8, 3, 1]), (128, 128, 3, 7, [12000, 500, 3000], [2, 1, 4]),
    (64, 128, 2, 5, [20000, 300, 3], [30, 70, 3]), (128, 16, 5, 2, [4000, 129, 1000, 0, 6000], [100, 129, 1, 0, 17]), (64, 64, 8, 16, [700, 2500, 64, 900], [16, 33, 20, 1])])
def test_parts_of_tiles_of_several_requests(dtype, D, P, H, group, held, added):
    check_parts(dtype, held, added, D, P, H, group)
    check_parts(dtype, held, added, D, P, H, group, causal=False)


def test_parts_of_many_equal_requests():
    n = 37                                                              # shares begin and end anywhere in a request
    check_parts(F16, [2048] * n, [1] * n, 64, 64, 3, 4)
    check_parts(BF16, [1100] * n, [33] * n, 128, 64, 1, 2)


@pytest.mark.parametrize("most", [1, 2, 30])
def test_many_short_requests(most):
    # more requests than a CTA has threads, some without a token, some without a row, at the ends too
    r = random.Random(most)
    n = 1500
    held = [0] + [r.choice([0, 1, 2, 17, 40, 65, 200]) for _ in range(n - 2)] + [0]
    added = [min(h, r.choice([0, 1, 1, most])) for h in held]
    s = Setup4(BF16, held, 1, 64, 16, seed=21)
    starts = [sum(added[:i]) for i in range(n + 1)]
    q = s.rows(starts[-1] + 2, 2, 1.5)
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(q.shape[0], 2, n, most)
    s.cache.attention(q, s.ints(starts), s.ints(held), s.table, out, ws, most)
    for i in sorted(r.sample(range(n), 120)):                           # the reference is slow
        part = Setup4.__new__(Setup4)
        part.__dict__ = dict(s.__dict__, table=s.table[i:i + 1])
        want, tol = attention_ref(part, q[starts[i]:starts[i + 1]], [0, added[i]], [held[i]], 64 ** -0.5)
        assert bool(((out[starts[i]:starts[i + 1]].double().cpu() - want).abs() <= tol).all()), i
    assert bool(out.isfinite().all()) and bool((out[starts[-1]:] == 5.0).all()) and s.cache.workspace_status(ws) == 0


# ---- streams, graphs, workspaces ----

@pytest.mark.parametrize("added", [1, 2, 60])
def test_on_another_stream_and_in_graphs_that_share_a_workspace(added):
    held = [900, 130, 61]
    s = Setup4(BF16, held, 2, 128, 64, seed=15)
    T = 3 * added
    q = s.rows(T, 8)
    starts, lengths = s.ints([0, added, 2 * added, T]), s.ints(held)
    ws = s.cache.workspace(T, 8, 3, added)
    want = torch.zeros_like(q)
    s.cache.attention(q, starts, lengths, s.table, want, ws, added)
    torch.cuda.synchronize()
    side, outs, graphs = torch.cuda.Stream(), [torch.zeros_like(q) for _ in range(3)], []
    side.wait_stream(torch.cuda.current_stream())
    s.cache.attention(q, starts, lengths, s.table, outs[0], ws, added, stream=side)
    side.synchronize()
    for o in outs[1:]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.cache.attention(q, starts, lengths, s.table, o, ws, added)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)
    # lengths are read on the GPU: a replay follows them
    lengths.copy_(s.ints([450, 129, 1]))
    graphs[0].replay()
    s.cache.attention(q, starts, lengths, s.table, want, ws, added)
    torch.cuda.synchronize()
    assert torch.equal(outs[1], want)


@pytest.mark.parametrize("added", [1, 50])
def test_two_calls_at_once(added):
    """Two streams, a workspace each: calls that may run at the same time, on whatever part of the GPU the other leaves."""
    s = Setup4(F16, [3000, 700, 90], 2, 64 if added == 1 else 128, 32, seed=22)
    T = 3 * added
    starts, lengths = s.ints([0, added, 2 * added, T]), s.ints(s.held)
    qs = [s.rows(T, 8) for _ in range(2)]
    wss = [s.cache.workspace(T, 8, 3, added) for _ in range(2)]
    want, got, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for q, ws in zip(qs, wss):
        o = torch.zeros_like(q)
        s.cache.attention(q, starts, lengths, s.table, o, ws, added)
        want.append(o)
        got.append([torch.zeros_like(q) for _ in range(6)])
    torch.cuda.synchronize()
    for k in range(6):
        for q, ws, o, st in zip(qs, wss, got, streams):
            s.cache.attention(q, starts, lengths, s.table, o[k], ws, added, stream=st)
    torch.cuda.synchronize()
    for w, o in zip(want, got):
        assert all(torch.equal(x, w) for x in o)
    assert [s.cache.workspace_status(ws) for ws in wss] == [0, 0]


def test_one_workspace_for_calls_of_every_kind_in_turn():
    from tests._cache import Setup
    s, eight = Setup4(BF16, [2000, 300], 1, 64, 16, seed=23), Setup(BF16, [2000, 300], 1, 64, 16, seed=23)
    ws = s.cache.workspace(400, 4, 2, 200)                              # the larger of the two
    for added in (1, 200, 3, 100, 1):
        for t in (s, eight):
            q = t.rows(2 * added, 4)
            args = (q, t.ints([0, added, 2 * added]), t.ints(t.held), t.table)
            out, want = torch.zeros_like(q), torch.zeros_like(q)
            t.cache.attention(*args, out, ws, added)
            t.cache.attention(*args, want, t.cache.workspace(2 * added, 4, 2, added), added)
            assert torch.equal(out, want)


@pytest.mark.parametrize("added", [1, 40])
def test_a_workspace_whose_wait_ran_out_is_not_used_before_an_init(added):
    """The state is planted: TSQ_ERR_TIMEOUT in the status, counters of parts that stand between calls."""
    s = Setup4(F16, [5000, 300], 2, 64, 16, seed=34)
    T = 2 * added
    q = s.rows(T, 4)
    args = (q, s.ints([0, added, T]), s.ints(s.held), s.table)
    ws = s.cache.workspace(T, 4, 2, added)
    want, out = torch.zeros_like(q), torch.full_like(q, 5.0)
    s.cache.attention(*args, want, ws, added)
    words = ws[:4096].view(torch.int32)
    words[0] = 7
    words[4:200] = 1
    before = words.clone()
    s.cache.attention(*args, out, ws, added)
    assert s.cache.workspace_status(ws) == 7 and bool((out == 5.0).all()) and torch.equal(words, before)
    s.cache.workspace_init(ws)
    for _ in range(2):
        s.cache.attention(*args, out, ws, added)
        assert torch.equal(out, want)
    assert s.cache.workspace_status(ws) == 0


def test_refusals_through_the_binding():
    s = Setup4(F16, [40], 2, 64, 16, seed=24)
    q, out = s.rows(1, 4), s.rows(1, 4)
    args = (s.ints([0, 1]), s.ints([40]), s.table)
    ws = s.cache.workspace(1, 4, 1, 1)
    for bad in (dict(q=q.to(BF16)), dict(q=q[..., :32]), dict(q=q.cpu()), dict(out=out[:, :2]), dict(ws=ws.view(torch.int32)), dict(max_query="x")):
        a = dict(q=q, out=out, ws=ws, max_query=1)
        a.update(bad)
        with pytest.raises((AssertionError, TypeError)):
            s.cache.attention(a["q"], *args, a["out"], a["ws"], a["max_query"])
    for bad in (dict(ws=ws[:-16]), dict(max_query=0), dict(scale=math.nan)):
        a = dict(ws=ws, max_query=1, scale=None)
        a.update(bad)
        with pytest.raises(B.TsqError):
            s.cache.attention(q, *args, out, a["ws"], a["max_query"], scale=a["scale"])
    with pytest.raises(B.TsqError):                                     # five query heads for two key heads
        s.cache.attention(s.rows(1, 5), *args, s.rows(1, 5), ws, 1)
    with pytest.raises(AssertionError):
        s.cache.store(s.rows(3, 2), s.rows(3, 2), s.ints([1, 2]))
    with pytest.raises(AssertionError):
        s.cache.load(s.ints([[1], [2]]), s.rows(2, 2), s.rows(2, 2))
    with pytest.raises(AssertionError):
        B.Cache4(F16, s.k_codes, s.v_codes[:1], s.k_grid, s.v_grid)
    with pytest.raises(AssertionError):
        B.Cache4(F16, s.k_codes.view(torch.int8), s.v_codes, s.k_grid, s.v_grid)
    with pytest.raises(AssertionError):
        B.Cache4(F16, s.k_codes, s.v_codes, s.k_grid[..., :8].contiguous(), s.v_grid)


@pytest.mark.parametrize("added", [1, 20])
def test_offsets_past_32_bits(added):
    # 4.6 GB of codes each; the pages in use are the last ones
    s = Setup4(F16, [300, 40], 8, 128, 128, seed=16, least_pages=70000)
    assert s.k_codes.numel() > 2 ** 32 and int(s.table[0, 0]) * 8 * 128 * 64 > 2 ** 32
    slots = s.slots_of(0, 300 - added, 300) + s.slots_of(1, 40 - added, 40)
    x_k, x_v = s.rows(2 * added, 8), s.rows(2 * added, 8)
    s.cache.store(x_k, x_v, s.ints(slots))
    at = s.ints(slots).long()
    for x, codes, grid in ((x_k, s.k_codes, s.k_grid), (x_v, s.v_codes, s.v_grid)):
        c, w = store_ref(x.float().cpu().numpy())
        assert np.array_equal(codes[at // 128, :, at % 128].cpu().numpy(), c) and np.array_equal(grid[at // 128, :, at % 128].cpu().numpy(), w)
    check_load(s, slots)
    check_attention(s, [added, added], 4)


# ---- together ----

@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_request_from_its_prompt_to_its_tenth_token(dtype):
    """The operators together, as a server has them: prompts, then a token a step; attention at each against the cache as it stands, and cross attention over states that were stored once."""
    H, D, P, group, width = 2, 64, 16, 4, 12
    s = Setup4(dtype, [0, 0, 0], H, D, P, seed=17, spare=60)
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    held, prompt, free = [0, 0, 0], [37, 1, 80], s.free
    # the encoders' states
    states, state_table = [50, 0, 129], torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    start, state_lengths, slots, taken = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 3, sum(states), 1))
    B.cache_slots(P, s.ints([0, 0, 0]), s.ints(states), free, start, state_lengths, state_table, slots, taken)
    s.cache.store(s.rows(sum(states), H), s.rows(sum(states), H), slots)
    free = free[int(taken):]
    ws = s.cache.workspace(200, H * group, 3, 80)
    for step in range(11):
        added = prompt if step == 0 else [1, 1, 0 if step == 4 else 1]
        T = sum(added) + 2
        starts, lengths, slots, taken = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 3, T, 1))
        B.cache_slots(P, s.ints(held), s.ints(added), free, starts, lengths, table, slots, taken)
        free = free[int(taken):]
        k, v, q = s.rows(T, H, 1.0 + step % 3), s.rows(T, H), s.rows(T, H * group)
        s.cache.store(k, v, slots)
        out, cross = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
        s.cache.attention(q, starts, lengths, table, out, ws, max(added))
        s.cache.attention(q, starts, state_lengths, state_table, cross, ws, max(added), causal=False)
        held = [h + a for h, a in zip(held, added)]
        assert lengths.cpu().tolist() == held
        for got, of, n, causal in ((out, table, held, True), (cross, state_table, states, False)):
            want, tol = attention_ref(s, q, starts.cpu().tolist(), n, D ** -0.5, causal, of)
            assert bool(((got.double().cpu() - want).abs() <= tol)[:T - 2].all()) and bool((got[T - 2:] == 5.0).all())
        back_k, back_v = check_load(s, slots.tolist())
        at = slots[:T - 2].long()
        for x, back, grid in ((k, back_k, s.k_grid), (v, back_v, s.v_grid)):   # a step at most: an end of the range may lie half a step past the last code's half
            step_of = scales(grid[at // P, :, at % P])[..., None]
            assert bool(((back[:T - 2].float() - x[:T - 2].float()).abs() <= step_of * 1.0001 + HALF_STEP[dtype] * (x[:T - 2].abs().float() + step_of)).all())
    assert s.cache.workspace_status(ws) == 0


@pytest.mark.parametrize("dtype,rows", [(F16, 7), (BF16, 200)])         # through the row kernel, through the tile kernel
def test_a_captured_step(dtype, rows):
    """Slots, store, attention and load captured into a graph and replayed, against the same calls made one by one."""
    P, H, D, group, width = 16, 2, 64, 4, 20

    class Side:
        def __init__(self):
            self.s = s = Setup4(dtype, [0, 0, 0], H, D, P, seed=50, spare=60)
            ints = lambda n, v=0: torch.full((n,), v, dtype=torch.int32, device="cuda")  # noqa: E731
            self.held, self.added, self.free = ints(3), ints(3), ints(200)
            self.starts, self.lengths, self.slots, self.taken = ints(4), ints(3), ints(rows, -1), ints(1)
            self.table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
            self.k, self.v, self.back_k, self.back_v = (torch.zeros((rows, H, D), dtype=dtype, device="cuda") for _ in range(4))
            self.q, self.out = (torch.zeros((rows, H * group, D), dtype=dtype, device="cuda") for _ in range(2))
            self.ws = s.cache.workspace(rows, H * group, 3, rows)

        def calls(self):
            B.cache_slots(P, self.held, self.added, self.free, self.starts, self.lengths, self.table, self.slots, self.taken)
            self.s.cache.store(self.k, self.v, self.slots)
            self.s.cache.attention(self.q, self.starts, self.lengths, self.table, self.out, self.ws, rows)
            self.s.cache.load(self.slots, self.back_k, self.back_v)

        def results(self):
            return [t.clone() for t in (self.starts, self.lengths, self.table, self.slots, self.taken, self.out[:int(self.starts[-1])], self.back_k, self.back_v,
                                        self.s.k_codes, self.s.v_codes, self.s.k_grid, self.s.v_grid)]

    eager, replayed = sides = [Side() for _ in range(2)]
    g = torch.Generator().manual_seed(51)
    for side in sides:                                                  # the first calls, before the capture
        side.calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.calls()
    held, order, used, share = [0, 0, 0], torch.randperm(60, generator=g).to(torch.int32), 0, rows // 3
    for added in ([share, 1, share + 1], [1, share, 0], [0, 0, 0], [share, share, share], [1, 1, 1], [0, 1, 2]):
        k, v, q = (torch.randn(t.shape, generator=g).to(dtype).cuda() for t in (eager.k, eager.v, eager.q))
        free = torch.full((200,), -1, dtype=torch.int32)
        free[:60 - used] = order[used:]
        for side in sides:
            for to, what in ((side.held, torch.tensor(held)), (side.added, torch.tensor(added)), (side.free, free), (side.k, k), (side.v, v), (side.q, q)):
                to.copy_(what)
        eager.calls()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager.results(), replayed.results()):
            assert torch.equal(x, y)
        assert bool(eager.out.isfinite().all()) and bool((eager.back_k[:sum(added)] != 0).any() or not sum(added))
        held = [h + a for h, a in zip(held, added)]
        used += int(eager.taken)
    assert [side.s.cache.workspace_status(side.ws) for side in sides] == [0, 0]


def test_a_cache_that_is_taken_over_and_handed_on():
    """Rows that the codec decodes go into the cache; rows that it gives back go through the codec like any others."""
    T, H, D, P = 200, 4, 64, 32
    s = Setup4(F16, [T], H, D, P, seed=42)
    sent = torch.cat([s.rows(T, H).view(T, H * D), s.rows(T, H).view(T, H * D)])   # keys, then values
    plan = B.Plan(F16, H * D, 2 * T, 6.0, [2, 4, 8], 0.2)
    blob, ws = plan.alloc(2 * T)
    rows, again = torch.empty_like(sent), torch.empty_like(sent)
    plan.encode(sent, blob, ws)
    plan.decode(blob, 2 * T, rows, ws)
    slots = s.slots_of(0, 0, T)
    check_store(s, rows[:T].view(T, H, D), rows[T:].view(T, H, D), slots)
    check_attention(s, [1], 4)
    check_attention(s, [20], 4)
    k, v = check_load(s, slots)
    back = torch.cat([k.view(T, H * D), v.view(T, H * D)])
    plan.encode(back, blob, ws)
    plan.decode(blob, 2 * T, again, ws)
    assert plan.workspace_status(ws) == (0, 0)
    big = back.abs() >= 6.0
    assert torch.equal(again[big], back[big])
