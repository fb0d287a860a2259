"""Attention over both paged caches where scores are so far from zero that binary32 holds them in steps of 1 to 64: the reference that a row's weights are relative to follows every score that is above it by
more than the weights' range allows, whichever way the sum of reference and limit is rounded."""
import pytest
import torch

from tests._cache import Setup
from tests._cache4 import Setup4, numbers, word_of

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("width", [8, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("added", [1, 40])                              # the row kernels, the tile kernels
@pytest.mark.parametrize("log2_scale", [12, 13, 14, 15, 16, 17, 18, 19, 20])
def test_scores_that_rounding_sets_apart(width, dtype, added, log2_scale):
    """Every key has the same score, so what sets weights apart is how its sum with the logarithm of a value's scale is rounded.  A row lies between the least and the largest of the values (weights are
    rounded to binary16, half a step of which is 2^-11; the row's rounding is the values' own at most, so 2^-8), whatever the weights are."""
    held = [600] * (150 if added == 1 else 2)                           # of the row kernels a CTA has several steps
    s = (Setup if width == 8 else Setup4)(dtype, held, 2, 64, 16, seed=80 + log2_scale)
    pages = s.table[:, :38].long()
    later = (torch.arange(38, device="cuda") // 4).clamp(max=4).mul(4.5).round().expand(len(held), -1)  # so far above the first ones are the later pages' scales, in powers of two
    if width == 8:
        s.k_codes[pages] = 64
        s.k_scale[pages] = 2.0 ** -5                                    # 2
        s.v_scale[pages] = torch.exp2(later - 9)[..., None]
        v = s.v_codes.double() * s.v_scale.double()[..., None, None]
    else:
        s.k_grid[pages] = word_of(torch.tensor([0.5]), torch.tensor([-4])).cuda()
        s.k_codes[pages] = 8 * 17                                       # 2
        s.v_grid[pages] = word_of(torch.exp2(later.cpu() - 9), torch.tensor([-8])).cuda()[..., None, None]
        v = numbers(s.v_codes, s.v_grid)
    tokens = len(held) * added
    q = (torch.rand((tokens, 6, 1), generator=s.g) * 6 + 2).to(dtype).expand(tokens, 6, 64).contiguous().cuda()
    out = torch.full_like(q, 5.0)
    ws = s.cache.workspace(tokens, 6, len(held), added)
    starts = list(range(0, tokens + 1, added))
    s.cache.attention(q, s.ints(starts), s.ints(held), s.table, out, ws, added, scale=2.0 ** log2_scale)
    assert bool(out.isfinite().all())
    for i in range(0, len(held), 7):
        for h in range(2):
            x = v[pages[i], h].reshape(-1, 64)[:600]
            got, room = out[starts[i]:starts[i + 1], 3 * h:3 * h + 3].double(), x.abs().amax(0) * 2.0 ** -7
            assert bool((got >= x.amin(0) - room).all()) and bool((got <= x.amax(0) + room).all())
