"""What the tests of the paged cache share: caches with tables in a mixed order, and plain references of its calls."""
import math

import numpy as np
import torch

FLOOR = np.float32(2.0 ** -40)
HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


class Setup:
    """Requests with `held` tokens in the cache (this step's among them) over pages in a mixed order; what no request holds is rubbish: NaN and
    infinite scales, entries of the table that name no page."""

    def __init__(self, dtype, held, kv_heads=2, head_dim=64, page=16, seed=0, spare=3, least_pages=0):
        from paper_2511_04002_b200 import binding as B
        g = torch.Generator().manual_seed(seed)
        self.g, self.dtype, self.held, self.H, self.D, self.P = g, dtype, held, kv_heads, head_dim, page
        need = [(h + page - 1) // page for h in held]
        self.pages = max(sum(need) + spare, least_pages)
        order = torch.randperm(self.pages, generator=g)
        if least_pages:
            order = order.sort(descending=True).values                 # the far end of a large cache
        self.width = max(need + [0]) + 2
        table = torch.full((len(held), self.width), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            table[i, n:] = torch.tensor([-1, self.pages + 7])[torch.arange(self.width - n) % 2].to(torch.int32)
            at += n
        self.free = order[at:].to(torch.int32).cuda()
        self.table = table.cuda()
        shape = (self.pages, kv_heads, page, head_dim)
        self.k_codes, self.v_codes = (torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2))
        self.k_scale, self.v_scale = (torch.full(shape[:2], bad, device="cuda") for bad in (math.nan, math.inf))
        used = order[:at].cuda()
        for codes, scale in ((self.k_codes, self.k_scale), (self.v_codes, self.v_scale)):
            codes[used] = (torch.randn((at,) + shape[1:], generator=g) * 40).round().clamp(-127, 127).to(torch.int8).cuda()
            scale[used] = (0.03 * torch.exp(0.5 * torch.randn((at, kv_heads), generator=g))).cuda()
        self.cache = B.Cache(dtype, self.k_codes, self.v_codes, self.k_scale, self.v_scale)

    def ints(self, v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def rows(self, tokens, heads, scale=1.0):
        return (torch.randn((tokens, heads, self.D), generator=self.g) * scale).to(self.dtype).cuda()

    def slots_of(self, i, lo, hi):
        return [int(self.table[i, p // self.P]) * self.P + p % self.P for p in range(lo, hi)]


def attention_ref(s, q, starts, lengths, scale, table=None):
    """Rows in 64 bits, and how far a kernel that rounds weights to binary16 (relative to the largest of the row times the page's scale), sums in binary32
    and rounds the row once may be off: weights half a step (2^-11) and 2^-25 at the small end, each score's binary32 sum D + 8
    roundings of its terms' magnitudes, 2^-20 for the exponential, the sums and the quotient."""
    table = (s.table if table is None else table).cpu()
    out, tol = torch.full(q.shape, math.nan, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    G = q.shape[1] // s.H
    for i, L in enumerate(lengths):
        n = starts[i + 1] - starts[i]
        pages = [int(e) for e in table[i, : (L + s.P - 1) // s.P]]
        ok = torch.tensor([0 <= e < s.pages for e in pages], dtype=torch.bool).repeat_interleave(s.P)[:L]
        safe = torch.tensor([e if 0 <= e < s.pages else 0 for e in pages], dtype=torch.long, device="cuda")
        for h in range(s.H):
            k = (s.k_codes[safe, h].double() * s.k_scale[safe, h].double()[:, None, None]).reshape(-1, s.D)[:L].cpu()
            v = (s.v_codes[safe, h].double() * s.v_scale[safe, h].double()[:, None, None]).reshape(-1, s.D)[:L].cpu()
            k, v = torch.where(ok[:, None], k, 0.0), torch.where(ok[:, None], v, 0.0)
            for j in range(n):
                see = min(L, max(0, L - n + j + 1))
                rows = q[starts[i] + j, h * G:(h + 1) * G].double().cpu()
                live = ok[:see]
                if not bool(live.any()):
                    out[starts[i] + j, h * G:(h + 1) * G] = 0.0
                    continue
                score = (rows @ k[:see].t() * scale).masked_fill(~live, -math.inf)
                w = torch.softmax(score, -1)
                o = w @ v[:see]
                off = (rows.abs() @ k[:see].abs().t()).amax(-1, keepdim=True) * abs(scale) * (s.D + 8) * 2.0 ** -24
                near = w @ v[:see].abs() * (2.0 ** -11 + 2 * off + 2.0 ** -20)
                out[starts[i] + j, h * G:(h + 1) * G] = o
                tol[starts[i] + j, h * G:(h + 1) * G] = near + see * 2.0 ** -25 * v[:see].abs().max() + HALF_STEP[s.dtype] * (o.abs() + near) + 2.0 ** -25
    return out, tol


def store_ref(codes, scale, x, slots):
    """tsq_cache_store on numpy arrays: codes int8 [pages, heads, P, D], scale f32, x f32 [tokens, heads, D]; binary32 throughout."""
    pages, H, P, D = codes.shape
    t, n = 0, len(slots)
    one, top = np.float32(1), np.float32(127)
    while t < n:
        slot = int(slots[t])
        if not 0 <= slot < pages * P:
            t += 1
            continue
        page, o = divmod(slot, P)
        e = t + 1
        while e < n and int(slots[e]) == slot + e - t and o + e - t < P:
            e += 1
        for h in range(H):
            run = x[t:e, h].astype(np.float32)
            fine = np.abs(run[np.isfinite(run)])
            s = max(np.float32(fine.max() if fine.size else 0) / top, FLOOR)
            if o:
                s = max(s, scale[page, h])
                front = codes[page, h, :o].astype(np.float32) * (scale[page, h] / s)
                codes[page, h, :o] = np.clip(np.rint(front), -127, 127).astype(np.int8)
            with np.errstate(invalid="ignore", over="ignore"):
                c = np.clip(np.rint(run * (one / s)), -127, 127)
            codes[page, h, o:o + e - t] = np.where(np.isnan(c), 0, c).astype(np.int8)
            scale[page, h] = s
        t = e


def slots_ref(P, held, added, free, table, tokens):
    held, added = [max(h, 0) for h in held], [max(a, 0) for a in added]
    table = [list(r) for r in table]
    starts, lengths, slots, used = [0], [], [], 0
    for row, h, a in zip(table, held, added):
        for p in range(h, h + a):
            e = p // P
            if p % P == 0:
                if e < len(row):
                    row[e] = free[used] if used < len(free) else -1
                used += 1
            page = row[e] if e < len(row) else -1
            slots.append(page * P + p % P if page >= 0 else -1)
        starts.append(starts[-1] + a)
        lengths.append(h + a)
    return starts, lengths, table, (slots + [-1] * tokens)[:tokens], used
