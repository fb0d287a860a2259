"""Attention over the paged 8-bit cache where a row's keys are shared out over many CTAs: every key has the same weight and every stretch of 64 keys its own mark in the
values, so that a part that is lost or counted twice shows in the row."""
import pytest
import torch

from tests._cache import HALF_STEP, Setup

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
SCALE = 0.5                                                             # of every value page


def mark(s, held):
    """Token p of a request has one value other than 0, at dimension (p / 64 + 3 head) mod D: 64 and more, by how often that dimension has come round."""
    s.v_codes.zero_()
    for i, n in enumerate(held):
        pages = s.table[i, :(n + s.P - 1) // s.P].long()
        s.v_scale[pages] = SCALE
        unit = torch.arange(pages.numel() * s.P, device="cuda") // 64
        for h in range(s.H):
            codes = torch.zeros((unit.numel(), s.D), dtype=torch.int8, device="cuda")
            codes[torch.arange(unit.numel()), (unit + 3 * h) % s.D] = (64 + unit // s.D % 60).to(torch.int8)
            s.v_codes[pages, h] = codes.view(pages.numel(), s.P, s.D)


def marked_means(s, held, added, group):
    want = torch.zeros((sum(added), s.H * group, s.D), dtype=torch.float64)
    t = 0
    for n, a in zip(held, added):
        unit = torch.arange(n) // 64
        value = (64 + unit // s.D % 60).double() * SCALE
        for j in range(a):
            see = n - a + j + 1
            for h in range(s.H):
                sums = torch.bincount((unit[:see] + 3 * h) % s.D, weights=value[:see], minlength=s.D)
                want[t, h * group:(h + 1) * group] = sums / max(see, 1)
            t += 1
    return want


def check_parts(dtype, held, added, D, P, H, group):
    """The weights are 1, the sums of codes and of weights whole numbers below 2^24 and so exact; the quotient and its product take a rounding of binary32 each, the row one
    of its type, with its subnormal numbers' half step (2^-25)."""
    s = Setup(dtype, held, H, D, P, seed=sum(held) % 1000)
    mark(s, held)
    T = sum(added)
    starts = [sum(added[:i]) for i in range(len(added) + 1)]
    q = s.rows(T, H * group)
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(T, H * group, len(added), max(added))
    s.cache.attention(q, s.ints(starts), s.ints(held), s.table, out, ws, max(added), scale=0.0)
    want = marked_means(s, held, added, group)
    off = (out.double().cpu() - want).abs()
    assert bool((off <= (HALF_STEP[dtype] + 2.0 ** -22) * want + 2.0 ** -25).all()), float((off / want.clamp(min=2.0 ** -14)).max())
    assert s.cache.workspace_status(ws) == 0


# one request and one key head: the row kernel has as many parts as 64-key units and two more, as far as its CTAs go (592, 444 for more than 8 rows)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added,group", [(1, 1), (4, 5)])
@pytest.mark.parametrize("keys", [64 * n + more for n, more in ((12, 1), (13, 64), (14, 3), (15, 17), (252, 64), (253, 1), (254, 5), (255, 64), (470, 2), (625, 0), (1700, 9))])
def test_parts_of_one_tile_of_few_rows(dtype, added, group, keys):
    check_parts(dtype, [keys], [added], 128 if keys % 2 else 64, 64, 1, group)


# the tile kernel: steps of 128 keys and four more, at most sixteen parts of a tile on the average
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added,group", [(9, 8), (40, 1), (300, 1), (5, 64)])
@pytest.mark.parametrize("keys", [400, 1280, 1285, 1413, 2001, 5000, 40000, 100001])
def test_parts_of_tiles_of_many_rows(dtype, added, group, keys):
    check_parts(dtype, [keys], [added], 128 if keys % 2 else 64, 32, 1, group)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,P,H,group,held,added", [
    (64, 16, 2, 3, [9000, 1, 130, 0, 20000, 64], [1, 1, 1, 0, 1, 1]), (128, 64, 5, 1, [3000, 7000, 65], [8, 3, 1]), (128, 128, 3, 7, [12000, 500, 3000], [2, 1, 4]),
    (64, 128, 2, 5, [20000, 300, 3], [30, 70, 3]), (128, 16, 5, 2, [4000, 129, 1000, 0, 6000], [100, 129, 1, 0, 17]), (64, 64, 8, 16, [700, 2500, 64, 900], [16, 33, 20, 1])])
def test_parts_of_tiles_of_several_requests(dtype, D, P, H, group, held, added):
    check_parts(dtype, held, added, D, P, H, group)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_parts_of_many_equal_requests(dtype):
    n = 37                                                              # shares begin and end anywhere in a request
    check_parts(dtype, [2048] * n, [1] * n, 64, 64, 3, 4)
    check_parts(dtype, [1100] * n, [33] * n, 128, 64, 1, 2)
