"""Operators of the paged 4-bit key/value cache as their users have them done, as timed cases.

A server that has more requests than its memory holds at 8 bits keeps keys and values as codes 0 .. 15 with a scale and a
zero-point for each token and head.  Its operators: quantising a step's keys and values into the cache and reading them
back (`store`); attention of a step's queries over the cache, causal (`attend`); attention of a decoder's queries over an
encoder's states, of which every query sees all (`cross`).

    listed()             the cases that stand for the range
    draw(rng)            one more case of the same range
    prepare(case, seed)  inputs, cache and tables, as a program has them before the call
    run(state)           one pass: in elementary torch operations, or through the framework where `own` is true
    exact(case, seed)    the same outputs from the definition, in 64 bits
    work(case)           bytes and operations the pass cannot do without

Definition.  A cache has pages of P tokens; a slot is page * P + place.  A row is what a token has in one head.  With lo and hi the least and the largest finite number
of the row, within +-2^126 (0 where none is finite): scale s = (hi - lo) / 15, at least max(|lo|, |hi|) / 128 and 2^-40, rounded up to seven
significant bits; zero-point z = round(lo / s); codes clamp(round(x / s) - z, 0, 15), 0 for NaN, where round takes halves away from zero.  A code stands for
(code + z) * s.  Query i of a request with n queries and length L sits at position L - n + i and sees the keys up to its own position, or all L (`cross`); a row that sees none
is zero.
"""
from __future__ import annotations

import math
import random

import torch

own = False
MAX_SCORES = 32 * 8192 * 8192    # query heads x queries x keys of the largest attention case, requests padded to one length
MAX_KEYS = 64 * 8000 * 8 * 128   # elements of keys, padded likewise
MAX_STORED = 8192 * 8 * 128      # elements of keys of the largest store


def _case(op, sequences, held, added, kv_heads=8, group=4, head_dim=128, page=64, dtype="bf16", pad=0, **name):
    """held, added: (fewest, most) tokens that the requests have in the cache before the step, and bring in it (cross: states of the encoder, queries).
    group: query heads for each key head.  pad: rows behind the last request's, as in a batch of a fixed size."""
    return dict(name, op=op, sequences=sequences, held_lo=held[0], held_hi=held[1], added_lo=added[0], added_hi=added[1],
                kv_heads=kv_heads, group=group, head_dim=head_dim, page=page, dtype=dtype, pad=pad)


def listed():
    return [
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
        # a decoder's step of 48 requests over their encoders' states, a key head for each of 20 query heads
        _case("cross", 48, (150, 1500), (1, 1), kv_heads=20, group=1, head_dim=64, dtype="f16", name="cross_step_48x20x64_f16"),
        # whole texts over their encoders' states, some longer and some shorter than those, padding rows
        _case("cross", 12, (77, 1500), (0, 448), kv_heads=4, group=4, page=32, pad=31, name="cross_texts_12x16_bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["store", "attend", "attend", "attend", "cross"])
    page = rng.choice([16, 32, 64, 128])
    dtype, head_dim = rng.choice(["f16", "bf16"]), rng.choice([64, 128, 128])
    kv_heads, pad = rng.choice([1, 2, 5, 8, 8, 10, 32, 40]), rng.choice([0, 0, 5, 77])
    sequences = _log_int(rng, 1, 64)
    if op == "store":
        most = max(1, min(_log_int(rng, 1, 8192), MAX_STORED // (sequences * kv_heads * head_dim)))
        return _case(op, sequences, (0, _log_int(rng, 1, 2000)), (rng.choice([0, 1, most]), most), kv_heads, 1, head_dim, page, dtype, pad)
    group = rng.choice([1, 2, 4, 5, 7, 8, 16]) if kv_heads <= 10 else 1
    keys = min(_log_int(rng, 1, 131072 if op == "attend" else 4096), MAX_KEYS // (sequences * kv_heads * head_dim))
    most = rng.choice([1, rng.randint(1, 8), _log_int(rng, 8, 8192 if op == "attend" else 1024)])
    most = max(1, min(most, keys if op == "attend" else most, MAX_SCORES // (2 * sequences * kv_heads * group * keys)))
    held = max(0, keys - most) if op == "attend" else keys
    return _case(op, sequences, (rng.choice([0, held // 3, held]), held), (rng.choice([0, 1, most]), most), kv_heads, group, head_dim, page, dtype, pad)


def _spread(n, lo, hi):
    """n lengths from lo to hi in a mixed order."""
    return [lo + (hi - lo) * (i * 7919 % n) // max(n - 1, 1) if n > 1 else hi for i in range(n)]


def _lengths(case):
    """Tokens in the cache before the step, the step's rows, tokens in the cache that the step's rows look at; by request."""
    held = _spread(case["sequences"], case["held_lo"], case["held_hi"])
    added = _spread(case["sequences"], case["added_lo"], case["added_hi"])[::-1]
    return held, added, held if case["op"] == "cross" else [h + a for h, a in zip(held, added)]


def _dtype(case):
    return {"f16": torch.float16, "bf16": torch.bfloat16}[case["dtype"]]


class State:
    pass


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    held, added, length = _lengths(case)
    S, P, H, D = case["sequences"], case["page"], case["kv_heads"], case["head_dim"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = State()
    s.op, s.cache, s.ws = case["op"], None, None
    s.tokens = sum(added) + case["pad"]                                  # rows of the step, padding among them
    s.max_query, s.max_length = max(added), max(length)
    starts = [0]
    for a in added:
        starts.append(starts[-1] + a)
    s.query_start, s.lengths = _ints(starts), _ints(length)
    width = (s.max_length + P - 1) // P + 3
    have = [(n + P - 1) // P for n in length]
    s.pages = sum(have) + 5
    order = torch.randperm(s.pages, generator=g, device="cuda").to(torch.int32)
    n_have = _ints(have)
    cols = torch.arange(width, device="cuda", dtype=torch.int32)[None, :]
    rank = (n_have.cumsum(0) - n_have)[:, None] + cols
    s.block_table = torch.where(cols < n_have[:, None], order[rank.clamp_(max=s.pages - 1)], -1).to(torch.int32).contiguous()

    # keys and values of the tokens that are in the cache, as rows of normal numbers leave them; what no request holds is left over from others
    s.k_codes = torch.empty((s.pages, H, P, D // 2), dtype=torch.uint8, device="cuda")
    s.v_codes = torch.empty_like(s.k_codes)
    for codes in (s.k_codes, s.v_codes):
        for p0 in range(0, s.pages, 128):
            part = codes[p0:p0 + 128]
            c = (torch.randn(part.shape + (2,), generator=g, device="cuda") * 2.8 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
            part.copy_(c[..., 0] | c[..., 1] << 4)
    unused = order[sum(have):].long()
    s.k_grid, s.v_grid = (torch.empty((s.pages, H, P), dtype=torch.int32, device="cuda") for _ in range(2))
    for grid, rubbish in ((s.k_grid, math.nan), (s.v_grid, math.inf)):
        scale = 0.36 * torch.exp(0.3 * torch.randn(grid.shape, generator=g, device="cuda"))
        scale[unused] = rubbish
        zero = torch.randint(-9, -6, grid.shape, generator=g, device="cuda", dtype=torch.int32)
        grid.copy_(zero << 16 | scale.view(torch.int32) >> 17 << 1)      # the upper half of a binary32 number, seven significant bits

    def rows(heads):
        return torch.randn((s.tokens, heads, D), generator=g, device="cuda")

    if s.op != "store":
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
    return _store(s) if s.op == "store" else _attend(s)


def _cache(s):
    from paper_2511_04002_b200 import binding as B
    if s.cache is None:                                                  # a program has one for as long as it has the cache
        s.cache = B.Cache4(s.k.dtype if s.op == "store" else s.q.dtype, s.k_codes, s.v_codes, s.k_grid, s.v_grid)
    return s.cache


def _store_plain(x, codes, grid, slots):
    P, x = codes.shape[2], x.float()
    fine = x.isfinite()
    lo = torch.where(fine, x, math.inf).amin(-1)
    hi = torch.where(fine, x, -math.inf).amax(-1)
    some = lo <= hi
    lo, hi = torch.where(some, lo, 0.0).clamp(min=-2.0 ** 126), torch.where(some, hi, 0.0).clamp(max=2.0 ** 126)
    step = (hi - lo) / torch.full_like(lo, 15.0)                         # a tensor: by a number, torch multiplies by the inverse
    step = torch.maximum(step, torch.maximum(lo.abs(), hi.abs()) / 128).clamp(min=2.0 ** -40)
    word = (step.view(torch.int32) + 0x1ffff) & ~0x1ffff                 # up to seven significant bits
    scale = word.view(torch.float32).double()

    def nearest(v):                                                      # in 64 bits: a value next to a border stays on its side of it
        return torch.where(v < 0, -torch.floor(0.5 - v), torch.floor(v + 0.5))

    zero = nearest(lo.double() / scale)
    code = (nearest(x.double() / scale[..., None]) - zero[..., None]).clamp(0, 15)
    code = torch.where(x.isnan(), 0.0, code).to(torch.uint8)
    live = (slots >= 0).nonzero()[:, 0]
    page, place = slots[live].long() // P, slots[live].long() % P
    codes[page, :, place] = (code[..., 0::2] | code[..., 1::2] << 4)[live]
    grid[page, :, place] = (zero.to(torch.int32) << 16 | word >> 16)[live]


def _values(codes, grid):
    """Numbers that codes [..., D / 2] with the words [...] stand for."""
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return (code + (grid >> 16)[..., None]).float() * (grid << 16).view(torch.float32)[..., None]


def _load_plain(codes, grid, slots, out):
    page, place = slots.long() // codes.shape[2], slots.long() % codes.shape[2]
    most = torch.finfo(out.dtype).max
    out.copy_(_values(codes[page, :, place], grid[page, :, place]).clamp(-most, most))


def _store(s):
    if own:
        cache = _cache(s)
        cache.store(s.k, s.v, s.slots)
        cache.load(s.touched, s.k_back, s.v_back)
    else:
        _store_plain(s.k, s.k_codes, s.k_grid, s.slots)
        _store_plain(s.v, s.v_codes, s.v_grid, s.slots)
        _load_plain(s.k_codes, s.k_grid, s.touched, s.k_back)
        _load_plain(s.v_codes, s.v_grid, s.touched, s.v_back)
    return {"k": s.k_back, "v": s.v_back}


def _attend(s):
    causal = s.op == "attend"
    if own:
        cache = _cache(s)
        if s.ws is None:
            s.ws = cache.workspace(s.tokens, s.q.shape[1], s.lengths.numel(), max(s.max_query, 1))
        cache.attention(s.q, s.query_start, s.lengths, s.block_table, s.out, s.ws, max(s.max_query, 1), causal=causal)
        return s.out
    S, P, L, Q = s.lengths.numel(), s.k_codes.shape[2], s.max_length, max(s.max_query, 1)
    H, D = s.k_codes.shape[1], s.q.shape[2]
    length, start = s.lengths.long(), s.query_start.long()
    at = torch.arange(L, device=s.q.device)
    held = at[None, :] < length[:, None]                                                         # [S, L]
    page = s.block_table.long()[:, at // P].clamp(min=0)
    k = torch.where(held[:, :, None, None], _values(s.k_codes[page, :, at % P], s.k_grid[page, :, at % P]), 0.0)
    v = torch.where(held[:, :, None, None], _values(s.v_codes[page, :, at % P], s.v_grid[page, :, at % P]), 0.0)
    i = torch.arange(Q, device=s.q.device)
    count = start[1:] - start[:-1]
    q = s.q[(start[:-1, None] + i).clamp(max=s.tokens - 1)].float().view(S, Q, H, -1, D)
    score = torch.einsum("sqhgd,slhd->shgql", q, k) * (1.0 / math.sqrt(D))
    seen = held[:, None, :].expand(S, Q, L)
    if causal:
        seen = seen & (at[None, None, :] <= (length - count)[:, None, None] + i[None, :, None])
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


def _exact_numbers(codes, grid):
    """[tokens, D] codes in bytes and [tokens] words as 64-bit numbers: the word's lower half is the upper half of a binary32 number, the other one signed."""
    number = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=codes.device)
    number[..., 0::2], number[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    low = grid.long() % 65536
    zero = (grid.long() - low) // 65536
    mantissa, exponent = (low % 128).double() / 128 + 1, (low // 128).double() - 127
    return (number + zero[..., None]) * (mantissa * torch.exp2(exponent))[..., None]


def exact(case, seed):
    held, added, length = _lengths(case)
    s = prepare(case, seed)
    P, D, H = case["page"], case["head_dim"], case["kv_heads"]
    table = s.block_table.cpu().tolist()
    if s.op == "store":
        out = {}
        for name, rows, codes, grid in (("k", s.k.double(), s.k_codes, s.k_grid), ("v", s.v.double(), s.v_codes, s.v_grid)):
            least, most = rows.amin(-1, keepdim=True), rows.amax(-1, keepdim=True)               # the inputs are finite
            fraction, power = torch.frexp(torch.clamp(torch.maximum((most - least) / 15, rows.abs().amax(-1, keepdim=True) / 128), min=2.0 ** -40))
            scale = torch.ldexp(torch.ceil(fraction * 128) / 128, power)
            away = lambda u: torch.sign(u) * torch.floor(u.abs() + 0.5)                          # noqa: E731
            zero = away(least / scale)
            new = (torch.clamp(away(rows / scale) - zero, 0, 15) + zero) * scale
            back, t = [], 0
            for row, h, a in zip(table, held, added):
                if a and h % P:
                    back.append(_exact_numbers(codes[row[h // P], :, :h % P], grid[row[h // P], :, :h % P]).transpose(0, 1))
                back.append(new[t:t + a])
                t += a
            limit = torch.finfo(s.k.dtype).max
            out[name] = torch.cat(back).clamp(-limit, limit)
        return out
    out = torch.full(s.q.shape, 7.0, dtype=torch.float64, device="cuda")
    t, G = 0, case["group"]
    for i, (n, a) in enumerate(zip(length, added)):
        pages = s.block_table[i, :(n + P - 1) // P].long()
        if a and not n:
            out[t:t + a] = 0.0
        for head in range(H if a and n else 0):
            k, v = (_exact_numbers(c[pages, head].reshape(-1, D // 2)[:n], f[pages, head].reshape(-1)[:n]) for c, f in ((s.k_codes, s.k_grid), (s.v_codes, s.v_grid)))
            hidden = torch.arange(n, device="cuda")[None, :] > n - a + torch.arange(a, device="cuda")[:, None] if s.op == "attend" else None
            for j in range(head * G, (head + 1) * G):
                w = s.q[t:t + a, j].double() @ k.t() / math.sqrt(D)
                out[t:t + a, j] = torch.softmax(w if hidden is None else w.masked_fill_(hidden, -math.inf), -1) @ v
        t += a
    return out


def work(case):
    """store: keys and values in, codes and words out and in again, values out; two operations to find the least and the largest, three for the code, two
    back.  attend, cross: queries, codes and words in, rows out; two operations for each product in the scores and in the sums."""
    held, added, length = _lengths(case)
    S, P, H, D = case["sequences"], case["page"], case["kv_heads"], case["head_dim"]
    n = sum(added)
    row = D // 2 + 4                                                     # bytes of a token and head in the cache
    if case["op"] == "store":
        touched = sum(h % P + a for h, a in zip(held, added) if a)
        return {"bytes": 2 * H * (2 * D * (n + touched) + row * (n + touched)) + 4 * (n + case["pad"] + touched), "flops": 2 * H * D * (5 * n + 2 * touched)}
    live = [(m, a) for m, a in zip(length, added) if a]
    keys, pages = sum(m for m, _ in live), sum((m + P - 1) // P for m, _ in live)
    seen = sum(a * m - (a * (a - 1) // 2 if case["op"] == "attend" else 0) for m, a in live)
    return {"bytes": 2 * H * row * keys + 4 * H * case["group"] * D * n + 4 * (pages + 2 * S), "flops": 4 * D * H * case["group"] * seen}
