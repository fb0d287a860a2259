"""Workspaces of attention over the paged 8-bit cache: what a wait that ran out leaves, and which tensors are taken."""
import pytest
import torch

from paper_2511_04002_b200 import binding as B
from tests._cache import Setup

pytestmark = pytest.mark.gpu
F16 = torch.float16


@pytest.mark.parametrize("added", [1, 40])
def test_a_workspace_whose_wait_ran_out_is_not_used_before_an_init(added):
    """The state is planted: TSQ_ERR_TIMEOUT in the status, counters of parts that stand between calls."""
    held = [5000, 300]
    s = Setup(F16, held, 2, 64, 16, seed=34)
    T = 2 * added
    q = s.rows(T, 4)
    args = (q, s.ints([0, added, T]), s.ints(held), s.table)
    ws = s.cache.workspace(T, 4, 2, added)
    want, out = torch.zeros_like(q), torch.full_like(q, 5.0)
    s.cache.attention(*args, want, ws, added)
    words = ws[:4096].view(torch.int32)
    words[0] = 7
    words[4:200] = 1
    before = words.clone()
    for _ in range(2):
        s.cache.attention(*args, out, ws, added)
    assert s.cache.workspace_status(ws) == 7 and bool((out == 5.0).all()) and torch.equal(words, before)
    s.cache.workspace_init(ws)
    assert s.cache.workspace_status(ws) == 0
    for _ in range(2):
        s.cache.attention(*args, out, ws, added)
        assert torch.equal(out, want)
    assert s.cache.workspace_status(ws) == 0


@pytest.mark.parametrize("call", ["workspace_init", "workspace_status"])
def test_tensors_that_are_no_workspace(call):
    s = Setup(F16, [40], 2, 64, 16, seed=35)
    ws = s.cache.workspace(1, 4, 1, 1)
    one = torch.zeros(1, dtype=torch.uint8, device="cuda")
    for bad in (ws.cpu(), ws.view(torch.int32), ws.view(torch.float32), ws[::2], one.expand(1 << 24), ws[:0]):
        with pytest.raises((AssertionError, B.TsqError)):
            getattr(s.cache, call)(bad)
    getattr(s.cache, call)(ws)
