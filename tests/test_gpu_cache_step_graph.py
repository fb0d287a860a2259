"""A whole step over the paged 8-bit cache (slots, store, attention, load) captured into a graph and replayed, against the same calls made one by one."""
import pytest
import torch

from paper_2511_04002_b200 import binding as B
from tests._cache import Setup

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


class Step:
    """Buffers of a step of at most `rows` rows and its four calls; lengths, pages and rows are read on the GPU."""

    def __init__(self, s, requests, rows, group, width):
        self.s, self.most = s, rows
        ints = lambda n, v=0: torch.full((n,), v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.held, self.added, self.free = ints(requests), ints(requests), ints(200)
        self.starts, self.lengths, self.slots, self.taken = ints(requests + 1), ints(requests), ints(rows, -1), ints(1)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        self.k, self.v, self.back_k, self.back_v = (torch.zeros((rows, s.H, s.D), dtype=s.dtype, device="cuda") for _ in range(4))
        self.q, self.out = (torch.zeros((rows, s.H * group, s.D), dtype=s.dtype, device="cuda") for _ in range(2))
        self.ws = s.cache.workspace(rows, s.H * group, requests, rows)

    def calls(self):
        B.cache_slots(self.s.P, self.held, self.added, self.free, self.starts, self.lengths, self.table, self.slots, self.taken)
        self.s.cache.store(self.k, self.v, self.slots)
        self.s.cache.attention(self.q, self.starts, self.lengths, self.table, self.out, self.ws, self.most)
        self.s.cache.load(self.slots, self.back_k, self.back_v)

    def results(self):
        s = self.s
        n = int(self.starts[-1])
        return [t.clone() for t in (self.starts, self.lengths, self.table, self.slots, self.taken, self.out[:n], self.back_k, self.back_v, s.k_codes, s.v_codes,
                                    torch.nan_to_num(s.k_scale), torch.nan_to_num(s.v_scale))]


@pytest.mark.parametrize("dtype,rows", [(F16, 7), (BF16, 200)])         # through the row kernel, through the tile kernel
def test_a_captured_step(dtype, rows):
    P, group, width = 16, 4, 20
    sides = [Step(Setup(dtype, [0, 0, 0], 2, 64, P, seed=50, spare=60), 3, rows, group, width) for _ in range(2)]
    eager, replayed = sides
    g = torch.Generator().manual_seed(51)
    for step in sides:                                                  # the first calls, before the capture
        step.calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.calls()
    held, order, used = [0, 0, 0], torch.randperm(60, generator=g).to(torch.int32), 0
    share = rows // 3
    for added in ([share, 1, share + 1], [1, share, 0], [0, 0, 0], [share, share, share], [1, 1, 1], [0, 1, 2]):
        k, v, q = (torch.randn(t.shape, generator=g).to(dtype).cuda() for t in (eager.k, eager.v, eager.q))
        free = torch.full((200,), -1, dtype=torch.int32)
        free[:60 - used] = order[used:]
        for step in sides:
            for to, what in ((step.held, torch.tensor(held)), (step.added, torch.tensor(added)), (step.free, free), (step.k, k), (step.v, v), (step.q, q)):
                to.copy_(what)
        eager.calls()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager.results(), replayed.results()):
            assert torch.equal(x, y)
        assert bool(eager.out.isfinite().all()) and bool((eager.back_k[:sum(added)] != 0).any() or not sum(added))
        held = [h + a for h, a in zip(held, added)]
        used += int(eager.taken)
        assert eager.lengths.tolist() == held
    assert [s.s.cache.workspace_status(s.ws) for s in sides] == [0, 0]
