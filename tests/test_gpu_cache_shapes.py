"""Store and load of the paged 8-bit cache, to the bit, at the launch shapes that large steps and wide caches take; the hand-over from the codec; tables shorter than their requests."""
import pytest
import torch

from paper_2511_04002_b200 import binding as B
from tests._cache import Setup
from tests.test_gpu_cache import check_attention, check_load, check_store

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def some_rows(s, n):
    x = s.rows(n, s.H)
    x *= torch.exp(0.5 * torch.randn((n, 1, 1), generator=s.g)).cuda().to(x.dtype)
    return x


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("P", [16, 128])
def test_store_and_load_of_a_large_prompt(dtype, P):
    # 64 tokens for each CTA of the store, four for each thread of the load; runs that cross a CTA's 32nd and 64th token, with rows between them that have no slot
    s = Setup(dtype, [5000, 333, 70], kv_heads=8, head_dim=128, page=P, seed=40 + P)
    slots = s.slots_of(0, 5, 2000) + [-1] * 7 + s.slots_of(1, 300, 333) + s.slots_of(0, 2000 // P * P + P, 5000) + [-1] + s.slots_of(2, 0, 70)
    check_store(s, some_rows(s, len(slots)), some_rows(s, len(slots)), slots)
    for n in (len(slots), len(slots) - 1, len(slots) - 7, 4097):        # whole and partly filled last blocks
        check_load(s, slots[:n])
    check_load(s, list(reversed(slots)) + slots[:100])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,D", [(17, 128), (17, 64), (33, 64), (40, 64), (40, 128), (131, 128)])
def test_store_and_load_of_many_heads(dtype, H, D):
    # from 17 heads of 128 (33 of 64) a token has more chunks than the load's CTA has threads
    s = Setup(dtype, [700, 90, 1], kv_heads=H, head_dim=D, page=32, seed=H)
    slots = s.slots_of(0, 3, 700) + [-1] + s.slots_of(1, 30, 90) + s.slots_of(2, 0, 1) + [s.pages * 32]
    check_store(s, some_rows(s, len(slots)), some_rows(s, len(slots)), slots)
    check_load(s, slots)
    check_load(s, slots[5:600:7])
    check_load(s, slots * 3)


@pytest.mark.parametrize("tokens", [1, 2, 31, 295, 296, 297, 591, 593, 2367, 2369, 3001])
def test_load_of_every_kind_of_block(tokens):
    # 5 heads of 64: six tokens of a CTA's threads at once, and from one token to 24 for a CTA
    s = Setup(BF16, [3100], kv_heads=5, head_dim=64, page=64, seed=41)
    check_load(s, s.slots_of(0, 3100 - tokens, 3100))


def test_a_cache_that_is_taken_over():
    """What a receiver does first: rows that the codec decodes go into the cache, and a step goes on from there."""
    T, H, D, P = 200, 4, 64, 32
    s = Setup(F16, [T], H, D, P, seed=42)
    sent = torch.cat([s.rows(T, H).view(T, H * D), s.rows(T, H).view(T, H * D)])   # keys, then values
    plan = B.Plan(F16, H * D, 2 * T, 6.0, [2, 4, 8], 0.2)
    blob, ws = plan.alloc(2 * T)
    rows = torch.empty_like(sent)
    plan.encode(sent, blob, ws)
    plan.decode(blob, 2 * T, rows, ws)
    assert plan.workspace_status(ws) == (0, 0)
    k, v = rows[:T].view(T, H, D), rows[T:].view(T, H, D)
    check_store(s, k, v, s.slots_of(0, 0, T))
    check_attention(s, [1], 4)
    check_attention(s, [20], 4)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 5, 40, 150])
def test_rows_of_requests_longer_than_their_table(dtype, added):
    # the table ends at 80, 80 and 64 keys; positions go by the whole length
    s = Setup(dtype, [170, 100, 64], 2, 64, 16, seed=43)
    table = s.table[:, :5].contiguous()
    check_attention(s, [added, min(added, 100), min(added, 64)], 3, table=table)
