"""The paged 8-bit cache on the GPU against plain references: block tables and slots, store and load (to the bit), attention (64 bits)."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2511_04002_b200 import binding as B
from tests._cache import HALF_STEP, Setup, attention_ref, slots_ref, store_ref

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


# ---- block tables and slots ----

def run_slots(P, held, added, free, table, tokens):
    dev = lambda v, shape=None: torch.tensor(v, dtype=torch.int32).reshape(shape or (len(v),)).cuda()  # noqa: E731
    S = len(held)
    width = len(table[0]) if S else 0
    t = dev([e for r in table for e in r], (S, width))
    start, lengths = (torch.full((n,), -9, dtype=torch.int32, device="cuda") for n in (S + 1, S))
    slots, taken = torch.full((tokens,), -9, dtype=torch.int32, device="cuda"), torch.full((1,), -9, dtype=torch.int32, device="cuda")
    args = (P, dev(held), dev(added), dev(free), start, lengths, t, slots, taken)
    B.cache_slots(*args)
    first = [x.cpu().tolist() for x in (start, lengths, t, slots, taken)]
    B.cache_slots(*args)                                                # again over its own results
    assert first == [x.cpu().tolist() for x in (start, lengths, t, slots, taken)]
    return first


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("seed", range(4))
def test_slots(P, seed):
    r = random.Random(seed)
    S = [1, 7, 300, 1500][seed]
    held = [r.choice([0, 1, P - 1, P, P + 1, r.randint(0, 5 * P)]) for _ in range(S)]
    added = [r.choice([0, 1, 1, P, r.randint(0, 3 * P)]) for _ in range(S)]
    width = 9
    need = sum((h + a + P - 1) // P - (h + P - 1) // P for h, a in zip(held, added))
    free = list(range(5000, 5000 + need + 3))
    r.shuffle(free)
    table = [[1000 + 9 * i + e if e * P < held[i] else -5 for e in range(width)] for i in range(S)]
    tokens = sum(added) + [0, 13, 5, 1][seed]
    got = run_slots(P, held, added, free, table, tokens)
    want = slots_ref(P, held, added, free, table, tokens)
    assert got[0] == want[0] and got[1] == want[1] and got[2] == want[2] and got[3] == want[3] and got[4] == [want[4]]
    assert want[4] == need


def test_slots_without_enough_pages_width_or_rows():
    P = 16
    held, added = [10, 0, 40, 5], [40, 33, 0, 100]
    table = [[7, -1, -1, -1], [-1] * 4, [8, 9, 10, -1], [11, -1, -1, -1]]
    # three free pages for fifteen; four entries for the last request's seven; fewer rows than tokens
    for free, tokens in (([30, 31, 32], 173), (list(range(30, 60)), 90), ([], 200)):
        got = run_slots(P, held, added, free, table, tokens)
        want = slots_ref(P, held, added, free, table, tokens)
        assert [got[0], got[1], got[2], got[3], got[4][0]] == list(want)


def test_slots_of_nothing_and_of_negative_lengths():
    assert run_slots(16, [], [], [1], [], 3) == [[0], [], [], [-1, -1, -1], [0]]
    got = run_slots(16, [-5, 3], [2, -7], [4], [[-1], [2]], 4)
    assert got == [[0, 2, 2], [2, 3], [[4], [2]], [64, 65, -1, -1], [1]]


# ---- store and load ----

def check_store(s, x_k, x_v, slots):
    want = []
    for codes, scale, x in ((s.k_codes, s.k_scale, x_k), (s.v_codes, s.v_scale, x_v)):
        c, f = codes.cpu().numpy().copy(), scale.cpu().numpy().copy()
        store_ref(c, f, x.float().cpu().numpy(), slots)
        want.append((c, f))
    s.cache.store(x_k, x_v, s.ints(slots))
    for (c, f), codes, scale in zip(want, (s.k_codes, s.v_codes), (s.k_scale, s.v_scale)):
        assert np.array_equal(codes.cpu().numpy(), c)
        assert np.array_equal(scale.cpu().numpy().view(np.uint32), f.view(np.uint32))


def check_load(s, slots):
    slots = s.ints(slots)
    k, v = (torch.full((len(slots), s.H, s.D), 3.0, dtype=s.dtype, device="cuda") for _ in range(2))
    s.cache.load(slots, k, v)
    there = (slots >= 0) & (slots < s.pages * s.P)
    at = torch.where(there, slots, 0).long()
    for got, codes, scale in ((k, s.k_codes, s.k_scale), (v, s.v_codes, s.v_scale)):
        want = (codes[at // s.P, :, at % s.P].float() * scale[at // s.P][..., None]).to(s.dtype)
        want = torch.where(there[:, None, None], want, torch.zeros_like(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_store_and_load(dtype, D, P):
    held = [1, 2 * P, 3 * P + 5, 40, 300]
    s = Setup(dtype, held, kv_heads=3, head_dim=D, page=P, seed=P + D)
    # one token; two whole pages; from inside a page over its end; a page's last tokens; a long one; rows without a slot between them
    parts = [(0, 0, 1), (1, 0, 2 * P), (2, P - 3, 3 * P + 5), (3, 33, 40), (4, 7, 300)]
    slots = []
    for i, lo, hi in parts:
        slots += s.slots_of(i, lo, hi) + [-1, s.pages * P + 4]
    x_k, x_v = s.rows(len(slots), 3), s.rows(len(slots), 3, 0.2)
    x_k[5:9] *= 20.0                                                    # some pages' scales grow
    check_store(s, x_k, x_v, slots)
    check_load(s, slots + list(reversed(slots)))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_store_token_by_token_grows_the_scale(dtype):
    s = Setup(dtype, [40], kv_heads=2, head_dim=64, page=16, seed=3)
    for p in range(40):
        check_store(s, s.rows(1, 2, 0.1 * (1 + p % 16)), s.rows(1, 2, 1.0 / (1 + p)), s.slots_of(0, p, p + 1))
    check_load(s, s.slots_of(0, 0, 40))


def test_store_of_a_batch_of_single_tokens():
    held = [1 + 13 * i % 70 for i in range(200)]
    s = Setup(BF16, held, kv_heads=8, head_dim=128, page=64, seed=4)
    slots = [t for i, h in enumerate(held) for t in s.slots_of(i, h - 1, h)]
    check_store(s, s.rows(200, 8), s.rows(200, 8), slots)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_store_of_a_prompt_in_blocks(dtype):
    # several tokens for each CTA: runs that begin and end anywhere in a CTA's block, and rows without a slot
    s = Setup(dtype, [1500, 700], kv_heads=8, head_dim=128, page=32, seed=25)
    slots = s.slots_of(0, 3, 1500) + [-1] * 5 + s.slots_of(1, 650, 700) + [-1]
    check_store(s, s.rows(len(slots), 8), s.rows(len(slots), 8), slots)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_store_of_values_that_are_no_numbers_zeros_and_extremes(dtype):
    s = Setup(dtype, [48, 20], kv_heads=2, head_dim=64, page=16, seed=5)
    x = s.rows(68, 2)
    x[0, 0, 3], x[1, 1, 5], x[2, 0, 7] = math.nan, math.inf, -math.inf
    x[16:32] = 0.0                                                      # a whole page
    x[32:48, 1] = math.inf                                              # a page of one head without a finite value
    x[48:50] = torch.finfo(dtype).max
    x[50:68] = torch.finfo(dtype).tiny
    check_store(s, x, -x, s.slots_of(0, 0, 48) + s.slots_of(1, 0, 20))


def test_rows_of_a_wider_tensor():
    s = Setup(F16, [50], kv_heads=2, head_dim=64, page=32, seed=6)
    wide = s.rows(50, 2 + 2 + 4)                                        # values, keys and something else of each token
    check_store(s, wide[:, 2:4], wide[:, :2], s.slots_of(0, 0, 50))
    k, v = s.rows(50, 8), torch.zeros((50, 2, 64), dtype=F16, device="cuda")
    before = k.clone()
    s.cache.load(s.ints(s.slots_of(0, 0, 50)), k[:, 3:5], v)
    want = torch.zeros_like(v)
    s.cache.load(s.ints(s.slots_of(0, 0, 50)), want, v)
    assert torch.equal(k[:, 3:5], want) and torch.equal(k[:, :3], before[:, :3]) and torch.equal(k[:, 5:], before[:, 5:])


@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_begin_between_32_byte_boundaries(D):
    s = Setup(BF16, [90], kv_heads=3, head_dim=D, page=16, seed=27)
    slots = s.slots_of(0, 0, 90)
    one, two = (torch.zeros(90 * 3 * D + 16, dtype=BF16, device="cuda") for _ in range(2))
    k, v = one[8:8 + 90 * 3 * D].view(90, 3, D), two[16:].view(90, 3, D)
    want_k, want_v = torch.zeros_like(k), torch.zeros_like(v)
    s.cache.load(s.ints(slots), want_k.contiguous(), want_v)
    x = s.rows(90, 3)
    k.copy_(x)
    check_store(s, k, x, slots)
    s.cache.load(s.ints(slots), k, v)
    at = s.ints(slots).long()
    for got, codes, scale in ((k, s.k_codes, s.k_scale), (v, s.v_codes, s.v_scale)):
        assert torch.equal(got, (codes[at // s.P, :, at % s.P].float() * scale[at // s.P][..., None]).to(BF16))
    assert bool((one[:8] == 0).all()) and bool((one[8 + 90 * 3 * D:] == 0).all()) and bool((two[:16] == 0).all())


# ---- attention ----

def check_attention(s, added, group, scale=None, lengths=None, table=None, q=None, pad=3, max_query=None, **kw):
    lengths = s.held if lengths is None else lengths
    starts = [0]
    for a in added:
        starts.append(starts[-1] + a)
    q = s.rows(starts[-1] + pad, s.H * group, 1.5) if q is None else q
    out = torch.full(q.shape, 5.0, dtype=s.dtype, device="cuda")
    most = max(added + [1]) if max_query is None else max_query
    ws = s.cache.workspace(q.shape[0], q.shape[1], len(added), most)
    args = (q, s.ints(starts), s.ints(lengths), s.table if table is None else table, out, ws, most)
    s.cache.attention(*args, scale=scale, **kw)
    torch.cuda.synchronize()
    assert s.cache.workspace_status(ws) == 0
    want, tol = attention_ref(s, q, starts, lengths, s.D ** -0.5 if scale is None else scale, table)
    got = out.double().cpu()
    assert bool((got[starts[-1]:] == 5.0).all()), "rows behind the last request's"
    if starts[-1]:
        most_value = torch.finfo(s.dtype).max                           # past it a row rounds to infinity
        off = (got.clamp(-most_value, most_value) - want.clamp(-most_value, most_value)).abs()[:starts[-1]]
        assert bool((off <= tol[:starts[-1]]).all()), "largest excess %g" % float((off - tol[:starts[-1]]).nan_to_num(nan=math.inf).max())
    again = torch.full_like(out, 5.0)
    s.cache.attention(*args[:4], again, *args[5:], scale=scale, **kw)
    assert torch.equal(out, again), "the same inputs give the same bits"
    return out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group", [(64, 16, 2, 1), (128, 64, 2, 4), (128, 16, 1, 7), (64, 128, 3, 16), (128, 32, 5, 2), (64, 64, 1, 3)])
def test_attention_of_single_tokens(dtype, D, P, H, group):
    held = [1, 2, P - 1, P, P + 1, 63, 64, 65, 300, 1027]
    check_attention(Setup(dtype, held, H, D, P, seed=H), [1] * len(held), group)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,added", [(128, 64, 2, 4, [1, 4, 0, 2, 3]), (64, 16, 2, 8, [2, 1, 1, 0, 2]), (128, 16, 3, 5, [3, 3, 1, 2, 3]),
                                               (128, 128, 1, 1, [16, 9, 13, 1, 0]), (64, 32, 2, 7, [2, 2, 2, 1, 2])])
def test_attention_of_drafted_tokens(dtype, D, P, H, group, added):
    held = [16, 700, 33, 129, 2100]
    check_attention(Setup(dtype, held, H, D, P, seed=group), added, group)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,held,added", [
    (128, 64, 1, 4, [300], [300]), (64, 16, 2, 1, [129, 128, 127], [129, 100, 1]), (128, 32, 2, 7, [500, 37, 1, 260], [30, 37, 1, 0]),
    (64, 128, 1, 64, [90, 400], [20, 5]), (128, 16, 1, 33, [64, 257], [9, 17]), (128, 128, 2, 2, [1500], [40]), (64, 64, 3, 16, [200, 641], [70, 129])])
def test_attention_of_prompts(dtype, D, P, H, group, held, added):
    check_attention(Setup(dtype, held, H, D, P, seed=D), added, group)


@pytest.mark.parametrize("added", [[3, 1, 2, 2], [40, 20, 70, 33]])
def test_rows_that_see_nothing_are_zero(added):
    # more rows than tokens, no tokens at all, a table without pages
    s = Setup(BF16, [40, 40, 80, 40], 2, 128, 16, seed=8)
    table = s.table.clone()
    table[3] = -1
    out = check_attention(s, added, 4, lengths=[2, 0, 80, 40], table=table)
    assert bool((out[added[0] - 3 if added[0] > 3 else 0] == 0).all()) and bool((out[added[0]] == 0).all())


@pytest.mark.parametrize("added", [1, 50])
def test_pages_outside_the_cache_are_not_seen(added):
    s = Setup(F16, [400, 200], 2, 64, 32, seed=9)
    table = s.table.clone()
    table[0, 3], table[0, 7], table[1, 0], table[1, 6] = -1, s.pages, -2 ** 31, 2 ** 31 - 1
    check_attention(s, [added, added], 2, table=table)


@pytest.mark.parametrize("added", [1, 40])
def test_a_table_without_entries(added):
    s = Setup(F16, [100], 1, 64, 16, seed=26)
    q = s.rows(added, 2)
    out = torch.full_like(q, 5.0)
    s.cache.attention(q, s.ints([0, added]), s.ints([100]), s.table[:, :0].contiguous(), out, s.cache.workspace(added, 2, 1, added), added)
    assert bool((out == 0).all())


def test_slots_of_the_most_requests():
    n = 8192
    held, added = [i * 7 % 50 for i in range(n)], [i * 5 % 3 for i in range(n)]
    need = sum((h + a + 15) // 16 - (h + 15) // 16 for h, a in zip(held, added))
    free, table = list(range(70000, 70000 + need)), [[9 * i + e if 16 * e < held[i] else -5 for e in range(4)] for i in range(n)]
    got, want = run_slots(16, held, added, free, table, sum(added) + 1), slots_ref(16, held, added, free, table, sum(added) + 1)
    assert [got[0], got[1], got[2], got[3], got[4][0]] == list(want)


@pytest.mark.parametrize("added", [1, 40])
def test_lengths_past_the_table_end_with_it(added):
    s = Setup(F16, [100, 64], 1, 64, 16, seed=10)
    table = s.table[:, :5].contiguous()
    starts, most = [0, added, 2 * added], added
    q = s.rows(2 * added, 2)
    ws = s.cache.workspace(2 * added, 2, 2, most)
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    s.cache.attention(q, s.ints(starts), s.ints([100, 64]), table, out, ws, most)
    assert bool(out.isfinite().all())
    if added == 1:                                                      # position 99 sees all 80 tokens of the table
        s.cache.attention(q, s.ints(starts), s.ints([80, 64]), table, want, ws, most)
        assert torch.equal(out, want)


def test_rows_past_max_query_are_left_alone():
    s = Setup(F16, [100, 64], 1, 64, 16, seed=11)
    q = s.rows(60, 2)
    full, part = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
    ws = s.cache.workspace(60, 2, 2, 40)
    s.cache.attention(q, s.ints([0, 40, 60]), s.ints([100, 64]), s.table, full, ws, 40)
    s.cache.attention(q, s.ints([0, 40, 60]), s.ints([100, 64]), s.table, part, ws, 30)
    same = [t for t in range(60) if t < 30 or t >= 40]
    near = 4 * HALF_STEP[F16] * full[same].abs().float() + 2e-3         # another split of the sums: both are within the tolerance of check_attention
    assert bool(((full[same].float() - part[same].float()).abs() <= near).all()) and bool((part[30:40] == 5.0).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 33])
def test_large_and_small_queries_scales_and_a_negative_factor(dtype, added):
    held = [130, 77]
    s = Setup(dtype, held, 2, 128, 32, seed=12)
    tokens = 2 * added
    q = s.rows(tokens, 4)
    q *= torch.exp2(torch.arange(tokens * 4, device="cuda").view(tokens, 4, 1) % 9 - 6.0).to(dtype)
    q[0, 0] = 0.0
    check_attention(s, [added, added], 2, q=q, pad=0)
    check_attention(s, [added, added], 2, q=q, pad=0, scale=-0.3)
    check_attention(s, [added, added], 2, q=q, pad=0, scale=0.0)
    s.v_scale[s.table[0, 1]] *= 2.0 ** 20                               # values of very different sizes
    s.v_scale[s.table[0, 2]] = 0.0
    s.k_scale[s.table[1, 0]] = 0.0
    check_attention(s, [added, added], 2, q=q, pad=0)


@pytest.mark.parametrize("added", [1, 33])
def test_a_query_that_is_no_number_spoils_its_own_row_alone(added):
    s = Setup(BF16, [130, 77], 2, 64, 16, seed=13)
    q = s.rows(2 * added, 8)
    ws = s.cache.workspace(2 * added, 8, 2, added)
    args = (s.ints([0, added, 2 * added]), s.ints([130, 77]), s.table)
    clean, out = torch.zeros_like(q), torch.zeros_like(q)
    s.cache.attention(q, *args, clean, ws, added)
    q[0, 1, 5], q[added, 6, 0] = math.nan, math.inf
    s.cache.attention(q, *args, out, ws, added)
    spoilt = out.isnan().any(-1)
    want = torch.zeros_like(spoilt)
    want[0, 1] = want[added, 6] = True
    assert torch.equal(spoilt, want) and torch.equal(out[~want], clean[~want])


@pytest.mark.parametrize("added", [1, 5, 40])
def test_queries_and_rows_inside_wider_tensors(added):
    s = Setup(F16, [90, 200], 2, 64, 16, seed=14)
    T = 2 * added
    wide, into = s.rows(T, 12), s.rows(T, 10)
    before = into.clone()
    ws = s.cache.workspace(T, 4, 2, added)
    args = (s.ints([0, added, T]), s.ints([90, 200]), s.table)
    want = torch.zeros((T, 4, 64), dtype=F16, device="cuda")
    s.cache.attention(wide[:, 3:7].contiguous(), *args, want, ws, added)
    s.cache.attention(wide[:, 3:7], *args, into[:, 5:9], ws, added)
    assert torch.equal(into[:, 5:9], want) and torch.equal(into[:, :5], before[:, :5]) and torch.equal(into[:, 9:], before[:, 9:])


@pytest.mark.parametrize("added", [1, 2, 60])
def test_on_another_stream_and_in_graphs_that_share_a_workspace(added):
    held = [900, 130, 61]
    s = Setup(BF16, held, 2, 128, 64, seed=15)
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


@pytest.mark.parametrize("D,P,H,group,held,added", [
    (64, 16, 1, 2, [40000], [1]), (128, 64, 1, 1, [9000], [1]), (64, 32, 2, 5, [20000, 3], [3, 1]), (128, 128, 1, 8, [12000, 64, 1], [2, 1, 1]),      # up to 592 parts of a tile
    (64, 64, 1, 1, [20000], [40]), (128, 16, 1, 5, [5000, 10], [30, 8]), (64, 128, 1, 64, [9000], [1]), (128, 32, 2, 3, [4000, 130], [100, 130])])
def test_long_requests_whose_tiles_many_shares_have_parts_of(D, P, H, group, held, added):
    check_attention(Setup(F16, held, H, D, P, seed=20), added, group)


@pytest.mark.parametrize("group,most", [(1, 1), (4, 2), (2, 30)])
def test_many_short_requests(group, most):
    # more requests than a CTA has threads, some without a token, some without a row, at the ends too
    r = random.Random(most)
    n = 1500
    held = [0] + [r.choice([0, 1, 2, 17, 40, 65, 200]) for _ in range(n - 2)] + [0]
    added = [min(h, r.choice([0, 1, 1, most])) for h in held]
    s = Setup(BF16, held, 1, 64, 16, seed=21)
    starts = [0]
    for a in added:
        starts.append(starts[-1] + a)
    q = s.rows(starts[-1] + 2, group, 1.5)
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(q.shape[0], group, n, most)
    s.cache.attention(q, s.ints(starts), s.ints(held), s.table, out, ws, most)
    some = sorted(r.sample(range(n), 150))                              # the reference is slow: rows of 150 of them, and that every row is finite
    for i in some:
        part = Setup.__new__(Setup)
        part.__dict__ = dict(s.__dict__, table=s.table[i:i + 1])
        want, tol = attention_ref(part, q[starts[i]:starts[i + 1]], [0, added[i]], [held[i]], 64 ** -0.5)
        assert bool(((out[starts[i]:starts[i + 1]].double().cpu() - want).abs() <= tol).all()), i
    assert bool(out.isfinite().all()) and bool((out[starts[-1]:] == 5.0).all()) and s.cache.workspace_status(ws) == 0


@pytest.mark.parametrize("added", [1, 50])
def test_two_calls_at_once(added):
    """Two streams, a workspace each: calls that may run at the same time, on whatever part of the GPU the other leaves."""
    held = [3000, 700, 90]
    s = Setup(F16, held, 2, 64 if added == 1 else 128, 32, seed=22)
    T = 3 * added
    starts, lengths = s.ints([0, added, 2 * added, T]), s.ints(held)
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


def test_one_workspace_for_calls_of_either_kind_in_turn():
    held = [2000, 300]
    s = Setup(BF16, held, 1, 64, 16, seed=23)
    ws = s.cache.workspace(400, 4, 2, 200)                              # the larger of the two
    for added in (1, 200, 3, 100, 1):
        q = s.rows(2 * added, 4)
        args = (q, s.ints([0, added, 2 * added]), s.ints(held), s.table)
        out, want = torch.zeros_like(q), torch.zeros_like(q)
        s.cache.attention(*args, out, ws, added)
        s.cache.attention(*args, want, s.cache.workspace(2 * added, 4, 2, added), added)
        assert torch.equal(out, want)


def test_refusals_through_the_binding():
    s = Setup(F16, [40], 2, 64, 16, seed=24)
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
        B.cache_slots(16, s.ints([1, 2]), s.ints([1]), s.free, s.ints([0, 0, 0]), s.ints([0, 0]), s.ints([[0], [0]]), s.ints([0, 0]), s.ints([0]))
    with pytest.raises(AssertionError):
        B.Cache(F16, s.k_codes, s.v_codes[:1], s.k_scale, s.v_scale)


def test_arrays_that_begin_anywhere():
    # slots, tables and lengths are only aligned to their four bytes
    whole = [torch.full((n + 1,), -9, dtype=torch.int32, device="cuda") for n in (4, 3, 21, 300, 1)]
    start, lengths, table, slots, taken = (w[1:] for w in whole)
    table = table.view(3, 7)
    held, added = [5, 0, 30], [100, 64, 1]
    free = torch.arange(50, 80, dtype=torch.int32, device="cuda")[1:]
    ints = lambda v: torch.tensor([0] + v, dtype=torch.int32, device="cuda")[1:]  # noqa: E731
    first = [[3] + [-9] * 6, [-9] * 7, [1, 2] + [-9] * 5]
    table.copy_(torch.tensor(first))
    B.cache_slots(16, ints(held), ints(added), free, start, lengths, table, slots, taken)
    want = slots_ref(16, held, added, free.cpu().tolist(), first, 300)
    assert [start.tolist(), lengths.tolist(), table.tolist(), slots.tolist(), int(taken)] == list(want)
    assert all(int(w[0]) == -9 for w in whole)


@pytest.mark.parametrize("added", [1, 20])
def test_offsets_past_32_bits(added):
    # 5.4 GB of codes each; the pages in use are the last ones
    s = Setup(F16, [300, 40], 8, 128, 128, seed=16, least_pages=41000)
    assert s.k_codes.numel() > 2 ** 32 and int(s.table[0, 0]) * 8 * 128 * 128 > 2 ** 32
    slots = s.slots_of(0, 300 - added, 300) + s.slots_of(1, 40 - added, 40)
    x_k, x_v = s.rows(2 * added, 8), s.rows(2 * added, 8)
    pages = sorted({t // 128 for t in slots})
    small = [c[pages].cpu().numpy().copy() for c in (s.k_codes, s.k_scale, s.v_codes, s.v_scale)]
    local = [pages.index(t // 128) * 128 + t % 128 for t in slots]
    store_ref(small[0], small[1], x_k.float().cpu().numpy(), local)
    store_ref(small[2], small[3], x_v.float().cpu().numpy(), local)
    s.cache.store(x_k, x_v, s.ints(slots))
    for got, want in zip((s.k_codes, s.k_scale, s.v_codes, s.v_scale), small):
        assert np.array_equal(got[pages].cpu().numpy(), want)
    check_load(s, slots)
    check_attention(s, [added, added], 4)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_request_from_its_prompt_to_its_tenth_token(dtype):
    """The operators together, as a server has them: prompts, then a token a step; attention at each against the cache as it stands."""
    H, D, P, group, width = 2, 64, 16, 4, 12
    s = Setup(dtype, [0, 0, 0], H, D, P, seed=17, spare=30)
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    held, prompt = [0, 0, 0], [37, 1, 80]
    free = s.free
    ws = s.cache.workspace(200, H * group, 3, 80)
    for step in range(11):
        added = prompt if step == 0 else [1, 1, 0 if step == 4 else 1]
        T = sum(added) + 2
        starts, lengths, slots, taken = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 3, T, 1))
        B.cache_slots(P, s.ints(held), s.ints(added), free, starts, lengths, table, slots, taken)
        free = free[int(taken):]
        k, v, q = s.rows(T, H, 1.0 + step % 3), s.rows(T, H), s.rows(T, H * group)
        s.cache.store(k, v, slots)
        out = torch.full_like(q, 5.0)
        s.cache.attention(q, starts, lengths, table, out, ws, max(added))
        held = [h + a for h, a in zip(held, added)]
        assert lengths.cpu().tolist() == held
        want, tol = attention_ref(s, q, starts.cpu().tolist(), held, D ** -0.5, table)
        assert bool(((out.double().cpu() - want).abs() <= tol)[:T - 2].all()) and bool((out[T - 2:] == 5.0).all())
        # what was stored is within half a step of its page's scale
        back_k, back_v = torch.zeros_like(k), torch.zeros_like(v)
        s.cache.load(slots, back_k, back_v)
        step_of = s.k_scale[(slots[:T - 2] // P).long()][..., None]
        near = step_of * 0.5001 + HALF_STEP[dtype] * (k[:T - 2].abs().float() + step_of)
        assert bool(((back_k[:T - 2].float() - k[:T - 2].float()).abs() <= near).all())


def test_codes_that_the_codec_sends_on():
    """A cache handed on: the rows that load gives go through the codec like any others."""
    s = Setup(F16, [64], 8, 128, 64, seed=18)
    k, v = (torch.zeros((64, 8, 128), dtype=F16, device="cuda") for _ in range(2))
    s.cache.load(s.ints(s.slots_of(0, 0, 64)), k, v)
    plan = B.Plan(F16, 1024, 64, 6.0, [2, 4, 8], 0.2)
    blob, ws = plan.alloc(64)
    y = torch.empty((64, 1024), dtype=F16, device="cuda")
    plan.encode(k.view(64, 1024), blob, ws)
    plan.decode(blob, 64, y, ws)
    assert plan.workspace_status(ws) == (0, 0)
    big = k.view(64, 1024).abs() >= 6.0
    assert torch.equal(y[big], k.view(64, 1024)[big])
