"""What the tests of the paged 4-bit cache share: caches with tables in a mixed order, and plain references of its calls."""
import math

import numpy as np
import torch

from tests._cache import HALF_STEP, Setup

F16, BF16 = torch.float16, torch.bfloat16


def word_of(scale, zero):
    """int32 words from binary32 scales (cut to seven significant bits) and whole zero-points."""
    return zero.to(torch.int32) << 16 | scale.float().view(torch.int32) >> 17 << 1


def scales(grid):
    return (grid << 16).view(torch.float32)


def zeros(grid):
    return grid >> 16


def numbers(codes, grid):
    """What codes [..., D / 2] and words [...] stand for, in 64 bits."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return (code.double() + zeros(grid).double()[..., None]) * scales(grid).double()[..., None]


class Setup4(Setup):
    """As Setup, over a 4-bit cache.  What no request holds is rubbish: in the last page's places behind a request, too."""

    def __init__(self, dtype, held, kv_heads=2, head_dim=64, page=16, seed=0, spare=3, least_pages=0, zero=(-12, -2)):
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
        shape = (self.pages, kv_heads, page)
        self.k_codes, self.v_codes = (torch.full(shape + (head_dim // 2,), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.k_grid, self.v_grid = (word_of(torch.full(shape, bad), torch.full(shape, 999)).cuda() for bad in (math.nan, math.inf))
        used = order[:at].cuda()
        for codes, grid in ((self.k_codes, self.k_grid), (self.v_codes, self.v_grid)):
            codes[used] = torch.randint(0, 256, (at,) + shape[1:] + (head_dim // 2,), generator=g, dtype=torch.uint8).cuda()
            scale = 0.2 * torch.exp(0.5 * torch.randn((at,) + shape[1:], generator=g))
            grid[used] = word_of(scale, torch.randint(zero[0], zero[1], scale.shape, generator=g)).cuda()
        for i, h in enumerate(held):
            if h % page:
                self.k_grid[int(table[i, h // page]), :, h % page:] = int(word_of(torch.tensor([math.nan]), torch.tensor([-999])))
                self.v_grid[int(table[i, h // page]), :, h % page:] = int(word_of(torch.tensor([math.inf]), torch.tensor([-999])))
        self.cache = B.Cache4(dtype, self.k_codes, self.v_codes, self.k_grid, self.v_grid)


def attention_ref(s, q, starts, lengths, scale, causal=True, table=None):
    """Rows in 64 bits, and how far a kernel may be off that rounds weights to binary16 relative to the largest of the row times its token's scale, sums in binary32 and
    rounds the row once: weights half a step (2^-11) and 2^-25 at the small end; each score's binary32 sum D + 8 roundings of its terms' magnitudes, which are those of code times query and of
    zero-point times query apart; keys and values that are rounded to binary16 half a step of themselves and of their zero-point times the scale; the sums over the tokens one rounding of 2^-23 for each 16 of them and for each part; 2^-20 for the exponential
    and the quotient."""
    table = (s.table if table is None else table).cpu()
    out, tol = torch.full(q.shape, math.nan, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    G = q.shape[1] // s.H
    exact = lambda grid: bool(((zeros(grid) <= 0) & (zeros(grid) >= -15)).all())  # noqa: E731
    for i, L in enumerate(lengths):
        n = starts[i + 1] - starts[i]
        L = min(L, table.shape[1] * s.P)
        pages = [int(e) for e in table[i, : (L + s.P - 1) // s.P]]
        ok = torch.tensor([0 <= e < s.pages for e in pages], dtype=torch.bool).repeat_interleave(s.P)[:L]
        safe = torch.tensor([e if 0 <= e < s.pages else 0 for e in pages], dtype=torch.long, device="cuda")
        for h in range(s.H):
            def rows(codes, grid):
                x = numbers(codes[safe, h], grid[safe, h]).reshape(-1, s.D)[:L].cpu()
                step, zero = (f(grid[safe, h]).double().reshape(-1)[:L].cpu() for f in (scales, zeros))
                # the numbers, the size of a term of their sums, what two roundings to binary16 go by
                return torch.where(ok[:, None], x, 0.0), torch.where(ok, step * (15 + zero.abs()), 0.0), torch.where(ok[:, None], x.abs() + (step * zero.abs())[:, None], 0.0)
            (k, k_size, k_round), (v, v_size, v_round) = rows(s.k_codes, s.k_grid), rows(s.v_codes, s.v_grid)
            k_half = 0.0 if exact(s.k_grid[safe, h].reshape(-1)[:L]) else 2.0 ** -11
            v_half = 0.0 if exact(s.v_grid[safe, h].reshape(-1)[:L]) else 2.0 ** -11
            for j in range(n):
                see = min(L, max(0, lengths[i] - n + j + 1)) if causal else L
                x = q[starts[i] + j, h * G:(h + 1) * G].double().cpu()
                live = ok[:see]
                if not bool(live.any()):
                    out[starts[i] + j, h * G:(h + 1) * G] = 0.0
                    continue
                score = (x @ k[:see].t() * scale).masked_fill(~live, -math.inf)
                w = torch.softmax(score, -1)
                o = w @ v[:see]
                sums = x.abs().sum(-1, keepdim=True) * k_size[:see]
                off = ((sums * (s.D + 8) * 2.0 ** -24 + (x.abs() @ k_round[:see].t()) * k_half) * abs(scale)).amax(-1, keepdim=True)
                near = w @ v[:see].abs() * (2.0 ** -11 + 2 * off + 2.0 ** -20) + w @ v_round[:see] * v_half + (w @ v_size[:see])[:, None] * (see / 16 + 8) * 2.0 ** -23
                near = near + see * 2.0 ** -25 * v_size[:see].max()
                out[starts[i] + j, h * G:(h + 1) * G] = o
                tol[starts[i] + j, h * G:(h + 1) * G] = near + HALF_STEP[s.dtype] * (o.abs() + near) + 2.0 ** -25
    return out, tol


def check_attention(s, added, group, scale=None, lengths=None, table=None, q=None, pad=3, max_query=None, causal=True):
    lengths = s.held if lengths is None else lengths
    starts = [0]
    for a in added:
        starts.append(starts[-1] + a)
    q = s.rows(starts[-1] + pad, s.H * group, 1.5) if q is None else q
    out = torch.full(q.shape, 5.0, dtype=s.dtype, device="cuda")
    most = max(added + [1]) if max_query is None else max_query
    ws = s.cache.workspace(q.shape[0], q.shape[1], len(added), most)
    args = (q, s.ints(starts), s.ints(lengths), s.table if table is None else table, out, ws, most)
    s.cache.attention(*args, scale=scale, causal=causal)
    torch.cuda.synchronize()
    assert s.cache.workspace_status(ws) == 0
    want, tol = attention_ref(s, q, starts, lengths, s.D ** -0.5 if scale is None else scale, causal, table)
    got = out.double().cpu()
    assert bool((got[starts[-1]:] == 5.0).all()), "rows behind the last request's"
    if starts[-1]:
        most_value = torch.finfo(s.dtype).max                           # past it a row rounds to infinity
        off = (got.clamp(-most_value, most_value) - want.clamp(-most_value, most_value)).abs()[:starts[-1]]
        assert bool((off <= tol[:starts[-1]]).all()), "largest excess %g" % float((off - tol[:starts[-1]]).nan_to_num(nan=math.inf).max())
    again = torch.full_like(out, 5.0)
    s.cache.attention(*args[:4], again, *args[5:], scale=scale, causal=causal)
    assert torch.equal(out, again), "the same inputs give the same bits"
    return out


def up7(x):
    """The next binary32 number of seven significant bits."""
    return ((x.astype(np.float32).view(np.int32) + 0x1ffff) & ~0x1ffff).view(np.float32)


def nearest(x):
    return np.sign(x) * np.floor(np.abs(x) + 0.5)


def store_ref(x):
    """Codes [..., D / 2] and words of rows x f32 [..., D]: scales in binary32, quotients exact enough in 64 bits (a quotient that is no half is 2^-12 of it away from one)."""
    fine = np.isfinite(x)
    lo, hi = np.where(fine, x, np.inf).min(-1), np.where(fine, x, -np.inf).max(-1)
    none = lo > hi
    lo, hi = np.where(none, 0, lo).astype(np.float32), np.where(none, 0, hi).astype(np.float32)
    lo, hi = np.maximum(lo, np.float32(-2.0 ** 126)), np.minimum(hi, np.float32(2.0 ** 126))
    step = np.maximum(((hi - lo).astype(np.float32) / np.float32(15)).astype(np.float32), np.maximum(np.abs(lo), np.abs(hi)) * np.float32(2.0 ** -7))
    s = up7(np.maximum(step, np.float32(2.0 ** -40)))
    z = nearest(lo.astype(np.float64) / s.astype(np.float64))
    with np.errstate(invalid="ignore"):
        c = np.clip(nearest(x.astype(np.float64) / s.astype(np.float64)[..., None]) - z[..., None], 0, 15)
    c = np.where(np.isnan(x), 0, c).astype(np.uint8)
    word = (z.astype(np.int64) << 16 | (s.view(np.int32).astype(np.int64) >> 16)).astype(np.uint64).astype(np.uint32).view(np.int32)
    return c[..., 0::2] | c[..., 1::2] << 4, word
