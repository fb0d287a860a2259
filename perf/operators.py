"""Operators of the paged 8-bit key/value cache as their users have them done, as timed cases.

A server that takes over a request holds keys and values as whole numbers in [-127, 127] with one scale for each page of
tokens and head.  A step of it is made of three operators: block tables, slots and offsets from the requests' lengths
(`slots`); quantising a step's keys and values into the cache, and reading them back (`store`); attention of a step's
queries over the cache (`attend`).

    listed()             the cases that stand for the range
    draw(rng)            one more case of the same range
    prepare(case, seed)  inputs, cache and tables, as a program has them before the call
    run(state)           one pass: in elementary torch operations, or through the framework where `own` is true
    exact(case, seed)    the same outputs from the definition, in 64 bits
    work(case)           bytes and operations the pass cannot do without

Definition.  A cache has pages of P tokens; a slot is page * P + place.  Storing a run of neighbouring tokens at the
places o, o+1, ... of a page sets, for each head, a = the largest finite |x| of the run and the scale s to
max(a / 127, 2^-40), or to the larger of that and the scale the page had if o > 0; codes in front of o become
rint(code * (s_had / s)); a token's code is rint(x * (1 / s)), +-127 for infinities, 0 for NaN.  Query i of a request with n queries and
length L sits at position L - n + i and sees the keys up to its own position; a row that sees none is zero.
"""
from __future__ import annotations

import math
import random

import torch

own = False
FLOOR = 2.0 ** -40               # smallest scale of a page
MAX_SCORES = 32 * 8192 * 8192    # query heads x queries x keys of the largest attention case, requests padded to one length
MAX_KEYS = 64 * 8000 * 8 * 128   # elements of keys, padded likewise
MAX_STORED = 8192 * 8 * 128      # elements of keys of the largest store


def _case(op, sequences, held, added, kv_heads=8, group=4, head_dim=128, page=64, dtype="bf16", pad=0, **name):
    """held, added: (fewest, most) tokens that the requests have in the cache before the step, and bring in it.  group: query heads for
    each key head.  pad: rows behind the last request's, as in a batch of a fixed size."""
    return dict(name, op=op, sequences=sequences, held_lo=held[0], held_hi=held[1], added_lo=added[0], added_hi=added[1],
                kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, dtype=dtype, pad=pad)


def listed():
    return [
        # a decode step of 64 requests: one slot each, now and then a new page
        _case("slots", 64, (100, 4000), (1, 1), page=16, name="slots_step_64"),
        # the admission of a large batch: new prompts and continued ones, some without a token in this step
        _case("slots", 512, (0, 2000), (0, 1024), page=64, pad=1000, name="slots_batch_512"),
        # a decode step of 64 requests writes its keys and values
        _case("store", 64, (100, 2000), (1, 1), name="store_step_64x8x128_bf16"),
        # a whole prompt written at once
        _case("store", 1, (0, 0), (8192, 8192), name="store_prompt_8192x8x128_bf16"),
        # odd lengths that begin and end inside pages, an odd number of heads, short heads, padding rows
        _case("store", 7, (1, 700), (0, 333), kv_heads=5, head_dim=64, page=32, dtype="f16", pad=19, name="store_ragged_7x5x64_f16"),
        # one token of one short conversation: latency alone
        _case("attend", 1, (1000, 1000), (1, 1), name="attend_token_1001_bf16"),
        # a decode step of a batch of 64 requests of all lengths
        _case("attend", 64, (500, 8000), (1, 1), name="attend_step_64_bf16"),
        # one token of one long document, 64 query heads
        _case("attend", 1, (131071, 131071), (1, 1), group=8, page=128, name="attend_long_131072_bf16"),
        # drafted tokens to verify, a key head for each of 40 query heads, small pages
        _case("attend", 16, (1, 3001), (1, 5), kv_heads=40, group=1, page=16, dtype="f16", name="attend_drafts_16x40_f16"),
        # a whole prompt
        _case("attend", 1, (0, 0), (8192, 8192), name="attend_prompt_8192_bf16"),
        # prompts taken in chunks beside continued requests, 64 query heads
        _case("attend", 5, (0, 6000), (1, 900), group=8, dtype="f16", name="attend_chunks_5_f16"),
        # odd lengths, seven query heads for a key head, short heads, requests without a query, padding rows
        _case("attend", 9, (0, 1000), (0, 257), kv_heads=2, group=7, head_dim=64, page=32, pad=13, name="attend_ragged_9x14x64_bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["slots", "store", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    dtype, head_dim = rng.choice(["f16", "bf16"]), rng.choice([64, 128, 128])
    kv_heads, pad = rng.choice([1, 2, 5, 8, 8, 10, 32, 40]), rng.choice([0, 0, 5, 77])
    if op == "slots":
        sequences = _log_int(rng, 1, 512)
        most = _log_int(rng, 1, 1024)
        return _case(op, sequences, (0, _log_int(rng, 1, 4000)), (rng.choice([0, 1, most]), most), page=page, pad=pad)
    sequences = _log_int(rng, 1, 64)
    if op == "store":
        most = max(1, min(_log_int(rng, 1, 8192), MAX_STORED // (sequences * kv_heads * head_dim)))
        return _case(op, sequences, (0, _log_int(rng, 1, 2000)), (rng.choice([0, 1, most]), most), kv_heads, 1, head_dim, page, dtype, pad)
    group = rng.choice([1, 2, 4, 5, 7, 8, 16]) if kv_heads <= 10 else 1
    keys = min(_log_int(rng, 1, 131072), MAX_KEYS // (sequences * kv_heads * head_dim))
    most = rng.choice([1, rng.randint(1, 8), _log_int(rng, 8, 8192)])
    most = max(1, min(most, keys, MAX_SCORES // (sequences * kv_heads * group * keys)))
    held = max(0, keys - most)
    return _case(op, sequences, (rng.choice([0, held // 3, held]), held), (rng.choice([0, 1, most]), most), kv_heads, group, head_dim, page, dtype, pad)


def _spread(n, lo, hi):
    """n lengths from lo to hi in a mixed order."""
    return [lo + (hi - lo) * (i * 7919 % n) // max(n - 1, 1) if n > 1 else hi for i in range(n)]


def _lengths(case):
    held = _spread(case["sequences"], case["held_lo"], case["held_hi"])
    added = _spread(case["sequences"], case["added_lo"], case["added_hi"])[::-1]
    return held, added


def _dtype(case):
    return {"f16": torch.float16, "bf16": torch.bfloat16}[case["dtype"]]


class State:
    pass


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    held, added = _lengths(case)
    S, P, H, D = case["sequences"], case["page"], case["kv_heads"], case["head_dim"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = State()
    s.op, s.page, s.cache, s.ws = case["op"], P, None, None
    s.tokens = sum(added) + case["pad"]                                  # rows of the step, padding among them
    s.max_query, s.max_length = max(added), max(h + a for h, a in zip(held, added))
    s.held, s.added = _ints(held), _ints(added)
    starts = [0]
    for a in added:
        starts.append(starts[-1] + a)
    s.query_start, s.lengths = _ints(starts), _ints([h + a for h, a in zip(held, added)])
    width = (s.max_length + P - 1) // P + 3
    before, after = [(h + P - 1) // P for h in held], [(h + a + P - 1) // P for h, a in zip(held, added)]
    s.pages = sum(after) + 5
    order = torch.randperm(s.pages, generator=g, device="cuda").to(torch.int32)

    have = before if s.op == "slots" else after
    n_have = _ints(have)
    cols = torch.arange(width, device="cuda", dtype=torch.int32)[None, :]
    rank = (n_have.cumsum(0) - n_have)[:, None] + cols
    s.block_table = torch.where(cols < n_have[:, None], order[rank.clamp_(max=s.pages - 1)], -1).to(torch.int32).contiguous()
    if s.op == "slots":
        s.free_pages = order[sum(before):].contiguous()
        s.slots = torch.full((s.tokens,), -7, dtype=torch.int32, device="cuda")
        s.taken = torch.zeros(1, dtype=torch.int32, device="cuda")
        s.query_start, s.lengths = torch.zeros_like(s.query_start), torch.zeros_like(s.lengths)
        return s

    # keys and values of the tokens that are in the cache; what no request holds is left over from others
    s.k_codes = torch.empty((s.pages, H, P, D), dtype=torch.int8, device="cuda")
    s.v_codes = torch.empty_like(s.k_codes)
    for codes in (s.k_codes, s.v_codes):
        for p0 in range(0, s.pages, 256):
            part = codes[p0:p0 + 256]
            part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 36.0).round_().clamp_(-127, 127))
    s.k_scale = 0.03 * torch.exp(0.3 * torch.randn((s.pages, H), generator=g, device="cuda"))
    s.v_scale = 0.03 * torch.exp(0.3 * torch.randn((s.pages, H), generator=g, device="cuda"))
    s.k_scale[order[sum(have):].long()] = math.nan
    s.v_scale[order[sum(have):].long()] = math.inf

    def rows(heads):
        return torch.randn((s.tokens, heads, D), generator=g, device="cuda")

    if s.op == "attend":
        s.q = rows(H * case["group"]).to(_dtype(case))
        s.out = torch.full_like(s.q, 7.0)                                # rows behind the last request's keep this
        return s
    gain = torch.ones(H * D, device="cuda")
    gain[torch.randperm(H * D, generator=g, device="cuda")[:8]] = 8.0    # channels that stand out, in the keys alone
    spread = torch.exp(0.2 * torch.randn((s.tokens, 1, 1), generator=g, device="cuda"))
    s.k, s.v = (rows(H) * spread * gain.view(H, D)).to(_dtype(case)), (rows(H) * spread).to(_dtype(case))
    slots, touched = [], []
    table = s.block_table.cpu().tolist()
    for i, (h, a) in enumerate(zip(held, added)):
        slots += [table[i][p // P] * P + p % P for p in range(h, h + a)]
        touched += [table[i][p // P] * P + p % P for p in range(h // P * P, h + a)] if a else []
    s.slots = _ints(slots + [-1] * case["pad"])
    s.touched = _ints(touched)                                           # every token of the pages that the step writes to
    s.k_back = torch.zeros((len(touched), H, D), dtype=_dtype(case), device="cuda")
    s.v_back = torch.zeros_like(s.k_back)
    return s


def run(s):
    return {"slots": _slots, "store": _store, "attend": _attend}[s.op](s)


def _cache(s):
    from paper_2511_04002_b200 import binding as B
    if s.cache is None:                                                  # a program has one for as long as it has the cache
        dtype = s.q.dtype if s.op == "attend" else s.k.dtype
        s.cache = B.Cache(dtype, s.k_codes, s.v_codes, s.k_scale, s.v_scale)
    return s.cache


def _slots(s):
    if own:
        from paper_2511_04002_b200 import binding as B
        B.cache_slots(s.page, s.held, s.added, s.free_pages, s.query_start, s.lengths, s.block_table, s.slots, s.taken)
    else:
        P, held, added = s.page, s.held.long(), s.added.long()
        length = held + added
        ends = added.cumsum(0)
        first, last = (held + P - 1) // P, (length + P - 1) // P
        new = last - first
        rank0 = new.cumsum(0) - new
        cols = torch.arange(s.block_table.shape[1], device=held.device)[None, :]
        rank = rank0[:, None] + cols - first[:, None]
        fits = rank < s.free_pages.numel()
        page = torch.where(fits, s.free_pages[rank.clamp(0, s.free_pages.numel() - 1)].long(), -1)
        table = torch.where((cols >= first[:, None]) & (cols < last[:, None]), page, s.block_table.long())
        t = torch.arange(s.tokens, device=held.device)
        i = torch.searchsorted(ends, t, right=True).clamp_(max=held.numel() - 1)
        at = length[i] - ends[i] + t
        mine = table[i, (at // P).clamp(0, table.shape[1] - 1)]
        s.slots.copy_(torch.where((t < ends[-1]) & (mine >= 0), mine * P + at % P, -1))
        s.block_table.copy_(table)
        s.query_start[1:].copy_(ends)
        s.lengths.copy_(length)
        s.taken.copy_(new.sum())
    return {"query_start": s.query_start, "lengths": s.lengths, "block_table": s.block_table, "slots": s.slots, "taken": s.taken}


def _store_plain(x, codes, scale, slots, query_start):
    P, pages = codes.shape[2], codes.shape[0]
    x = x.float()
    live = slots >= 0
    page, place = slots.clamp(min=0).long() // P, slots.clamp(min=0).long() % P
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1) * live[:, None]                       # [tokens, heads]
    most = torch.zeros_like(scale).scatter_reduce(0, page[:, None].expand_as(top), top, "amax")
    begin = torch.full((pages,), P, device=x.device).scatter_reduce(0, page, torch.where(live, place, P), "amin")
    fresh, touched = (begin == 0)[:, None], (begin < P)[:, None]
    want = (most / torch.full_like(most, 127.0)).clamp(min=FLOOR)                                # a tensor: by a number, torch multiplies by 1 / 127
    after = torch.where(touched, torch.where(fresh, want, torch.maximum(scale, want)), scale)
    # the page in which each request goes on: codes in front of its first new token
    lead = query_start[:-1].long().clamp(max=slots.numel() - 1)
    some = (query_start[1:] > query_start[:-1]) & (slots[lead] >= 0)
    old, o = page[lead], torch.where(some, place[lead], 0)
    was = codes[old].float()                                                                     # [requests, heads, P, D]
    front = (torch.arange(P, device=x.device)[None, :] < o[:, None])[:, None, :, None]
    moved = torch.where(front, (was * (scale[old] / after[old])[:, :, None, None]).round(), was)
    # a request without a token in this step may name a page that another one has: nothing of it is written
    keep = torch.where(some, old, pages)
    grown = torch.cat([codes, codes[:1]]).index_put((keep,), moved.to(torch.int8))
    inverse = 1.0 / after[page]
    value = torch.where(x.isnan(), 0.0, (x * inverse[:, :, None]).round().clamp(-127, 127))
    grown[torch.where(live, page, pages), :, place] = value.to(torch.int8)
    codes.copy_(grown[:pages])
    scale.copy_(after)


def _load_plain(codes, scale, slots, out):
    page, place = slots.long() // codes.shape[2], slots.long() % codes.shape[2]
    out.copy_(codes[page, :, place].float() * scale[page][:, :, None])


def _store(s):
    if own:
        cache = _cache(s)
        cache.store(s.k, s.v, s.slots)
        cache.load(s.touched, s.k_back, s.v_back)
    else:
        _store_plain(s.k, s.k_codes, s.k_scale, s.slots, s.query_start)
        _store_plain(s.v, s.v_codes, s.v_scale, s.slots, s.query_start)
        _load_plain(s.k_codes, s.k_scale, s.touched, s.k_back)
        _load_plain(s.v_codes, s.v_scale, s.touched, s.v_back)
    return {"k": s.k_back, "v": s.v_back, "k_scale": s.k_scale, "v_scale": s.v_scale}


def _attend(s):
    if own:
        cache = _cache(s)
        if s.ws is None:
            s.ws = cache.workspace(s.tokens, s.q.shape[1], s.lengths.numel(), s.max_query)
        cache.attention(s.q, s.query_start, s.lengths, s.block_table, s.out, s.ws, s.max_query)
        return s.out
    S, P, L, Q = s.lengths.numel(), s.page, s.max_length, max(s.max_query, 1)
    H, D = s.k_codes.shape[1], s.k_codes.shape[3]
    length, start = s.lengths.long(), s.query_start.long()
    at = torch.arange(L, device=s.q.device)
    held = at[None, :] < length[:, None]                                                         # [S, L]
    page = s.block_table.long()[:, at // P].clamp(min=0)
    k = torch.where(held[:, :, None, None], s.k_codes[page, :, at % P].float() * s.k_scale[page][..., None], 0.0)
    v = torch.where(held[:, :, None, None], s.v_codes[page, :, at % P].float() * s.v_scale[page][..., None], 0.0)
    i = torch.arange(Q, device=s.q.device)
    count = start[1:] - start[:-1]
    q = s.q[(start[:-1, None] + i).clamp(max=s.tokens - 1)].float().view(S, Q, H, -1, D)
    score = torch.einsum("sqhgd,slhd->shgql", q, k) * (1.0 / math.sqrt(D))
    seen = held[:, None, :] & (at[None, None, :] <= (length - count)[:, None, None] + i[None, :, None])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.einsum("shgql,slhd->shgqd", score, v) / torch.where(total == 0, 1.0, total)
    t = torch.arange(s.tokens, device=s.q.device)
    of = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp_(max=S - 1)
    rows = o.permute(0, 3, 1, 2, 4)[of, (t - start[of]).clamp(0, Q - 1)].reshape(s.out.shape)
    s.out.copy_(torch.where((t < start[-1])[:, None, None], rows, s.out.float()))
    return s.out


def exact(case, seed):
    held, added = _lengths(case)
    s = prepare(case, seed)
    P, D, H = case["page"], case["head_dim"], case["kv_heads"]
    table = s.block_table.cpu().tolist()
    if s.op == "slots":
        free, used, slots, starts = s.free_pages.cpu().tolist(), 0, [], [0]
        for row, h, a in zip(table, held, added):
            for p in range(h, h + a):
                if p % P == 0:
                    row[p // P], used = free[used] if used < len(free) else -1, used + 1
                slots.append(row[p // P] * P + p % P if row[p // P] >= 0 else -1)
            starts.append(starts[-1] + a)
        return {"query_start": _ints(starts), "lengths": _ints([h + a for h, a in zip(held, added)]), "block_table": _ints(table),
                "slots": _ints(slots + [-1] * case["pad"]), "taken": _ints([used])}
    if s.op == "store":
        out = {}
        for name, x, codes, scale in (("k", s.k.double(), s.k_codes, s.k_scale), ("v", s.v.double(), s.v_codes, s.v_scale)):
            scale, back, t = scale.double(), [], 0
            for row, h, a in zip(table, held, added):
                p = h
                while p < h + a:
                    page, o = row[p // P], p % P
                    n = min(P - o, h + a - p)
                    part = x[t:t + n].transpose(0, 1)                                            # [heads, n, D]
                    new = (part.abs().amax((1, 2)) / 127.0).clamp(min=FLOOR)
                    if o:
                        new = torch.maximum(new, scale[page])
                        front = (codes[page, :, :o].double() * (scale[page] / new)[:, None, None]).round()
                        back.append((front * new[:, None, None]).transpose(0, 1))
                    back.append(((part / new[:, None, None]).round().clamp(-127, 127) * new[:, None, None]).transpose(0, 1))
                    scale[page] = new
                    p, t = p + n, t + n
            out[name] = torch.cat(back) if back else x[:0]
            out[name + "_scale"] = scale
        return out
    out = torch.full(s.q.shape, 7.0, dtype=torch.float64, device="cuda")
    t, G = 0, case["group"]
    for i, (h, a) in enumerate(zip(held, added)):
        L = h + a
        pages = s.block_table[i, :(L + P - 1) // P].long()
        for head in range(H if a else 0):
            k, v = ((c[pages, head].double() * f[pages, head].double()[:, None, None]).reshape(-1, D)[:L]
                    for c, f in ((s.k_codes, s.k_scale), (s.v_codes, s.v_scale)))
            hidden = torch.arange(L, device="cuda")[None, :] > h + torch.arange(a, device="cuda")[:, None]
            for j in range(head * G, (head + 1) * G):
                w = s.q[t:t + a, j].double() @ k.t() / math.sqrt(D)
                out[t:t + a, j] = torch.softmax(w.masked_fill_(hidden, -math.inf), -1) @ v
        t += a
    return out


def work(case):
    """slots: lengths in; offsets, slots, the new entries of the tables and their pages out.  store: keys and values in, codes and scales out
    and in again, values out; two operations to find the largest, two for the code, one back.  attend: queries, codes and scales in, rows out; two
    operations for each product in the scores and in the sums."""
    held, added = _lengths(case)
    S, P, H, D = case["sequences"], case["page"], case["kv_heads"], case["head_dim"]
    n, pairs = sum(added), list(zip(held, added))
    if case["op"] == "slots":
        new = sum((h + a + P - 1) // P - (h + P - 1) // P for h, a in pairs)
        return {"bytes": 4 * (2 * S + 2 * S + 1 + n + case["pad"] + 2 * new), "flops": 0}
    if case["op"] == "store":
        pages = sum((h + a + P - 1) // P - h // P for h, a in pairs if a)
        touched = sum(h % P + a for h, a in pairs if a)
        return {"bytes": 2 * H * (D * (2 * n + n + 3 * touched) + 8 * pages) + 4 * (n + case["pad"] + touched), "flops": 2 * H * D * (4 * n + touched)}
    keys = sum(h + a for h, a in pairs if a)
    pages = sum((h + a + P - 1) // P for h, a in pairs if a)
    seen = sum(a * h + a * (a + 1) // 2 for h, a in pairs)
    return {"bytes": 2 * H * (D * keys + 4 * pages) + 4 * H * case["group"] * D * n + 4 * (pages + 2 * S), "flops": 4 * D * H * case["group"] * seen}
