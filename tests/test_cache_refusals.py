"""Argument errors of the paged cache's calls: returned before anything is enqueued, so no GPU is needed (pointers are numbers that nothing follows)."""
import ctypes as C

import pytest

from paper_2511_04002_b200 import binding as B

INVALID, UNSUPPORTED = 1, 2
PTR = 1 << 20


def cache(**kw):
    d = dict(dtype=0, kv_heads=4, head_dim=128, page_tokens=64, pages=100, k_codes=PTR, v_codes=PTR, k_scale=PTR, v_scale=PTR)
    d.update(kw)
    return B._CacheStruct(*[d[n] for n, _ in B._CacheStruct._fields_])


BAD_CACHES = [(dict(dtype=2), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), INVALID),
              (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=256), UNSUPPORTED), (dict(pages=0), INVALID),
              (dict(pages=2 ** 31 // 64), INVALID), (dict(k_codes=None), INVALID), (dict(v_codes=PTR + 8), INVALID), (dict(k_scale=PTR + 2), INVALID),
              (dict(v_scale=None), INVALID), (dict(kv_heads=1025), UNSUPPORTED)]


def store(c, k=PTR, ks=512, v=PTR, vs=512, tokens=3, slots=PTR):
    return B.lib().tsq_cache_store(C.byref(c), k, ks, v, vs, tokens, slots, None)


def load(c, k=PTR, ks=512, v=PTR, vs=512, tokens=3, slots=PTR):
    return B.lib().tsq_cache_load(C.byref(c), slots, tokens, k, ks, v, vs, None)


def attention(c, q=PTR, qs=1024, heads=8, tokens=3, start=PTR, lengths=PTR, requests=2, most=1, table=PTR, width=5, scale=0.1, out=PTR, outs=1024, ws=PTR,
              ws_bytes=1 << 30):
    return B.lib().tsq_cache_attention(C.byref(c), q, qs, heads, tokens, start, lengths, requests, most, table, width, scale, out, outs, ws, ws_bytes, None)


def workspace(c, tokens=3, heads=8, requests=2, most=1):
    n = C.c_size_t(0)
    return B.lib().tsq_cache_workspace(C.byref(c), tokens, heads, requests, most, C.byref(n))


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches(change, status):
    c = cache(**change)
    assert store(c) == load(c) == attention(c) == workspace(c) == status


@pytest.mark.parametrize("call", [store, load])
@pytest.mark.parametrize("change", [dict(k=None), dict(k=PTR + 8), dict(v=None), dict(ks=500), dict(ks=504), dict(vs=508), dict(tokens=-1), dict(tokens=2 ** 31),
                                    dict(slots=None), dict(slots=PTR + 1)])
def test_rows(call, change):
    assert call(cache(), **change) == INVALID


@pytest.mark.parametrize("call", [store, load])
def test_no_rows_are_nothing_to_do(call):
    assert call(cache(), tokens=0, k=None, v=None, slots=None) == 0


@pytest.mark.parametrize("change,status", [
    (dict(heads=0), INVALID), (dict(heads=6), INVALID), (dict(heads=4 * 65, qs=4 * 65 * 128), UNSUPPORTED), (dict(requests=-1), INVALID), (dict(requests=8193), UNSUPPORTED),
    (dict(most=0), INVALID), (dict(tokens=-1), INVALID), (dict(tokens=2 ** 30), UNSUPPORTED)])
def test_sizes_of_attention(change, status):
    assert attention(cache(), **change) == status and workspace(cache(), **{k: v for k, v in change.items() if k != "qs"}) == status


@pytest.mark.parametrize("change", [
    dict(q=None), dict(q=PTR + 4), dict(qs=1020), dict(qs=1016), dict(out=None), dict(outs=512), dict(start=None), dict(lengths=None), dict(table=None), dict(width=-1),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(ws=None), dict(ws=PTR + 4), dict(start=PTR + 2), dict(table=PTR + 2)])
def test_arguments_of_attention(change):
    assert attention(cache(), **change) == INVALID


@pytest.mark.parametrize("scale", [2.5e38, 3.0e38, -2.5e38, 3.4e38])
def test_a_scale_that_is_infinite_in_binary_logarithms(scale):
    assert attention(cache(), scale=scale) == INVALID


def test_no_cache_and_no_place_for_the_answer():
    L = B.lib()
    n = C.c_size_t(0)
    assert L.tsq_cache_store(None, PTR, 512, PTR, 512, 3, PTR, None) == INVALID
    assert L.tsq_cache_workspace(None, 3, 8, 2, 1, C.byref(n)) == INVALID
    assert L.tsq_cache_workspace(C.byref(cache()), 3, 8, 2, 1, None) == INVALID
    assert L.tsq_cache_workspace_init(None, 1 << 30, None) == L.tsq_cache_workspace_init(PTR + 8, 1 << 30, None) == INVALID


def test_workspace_status_wants_a_workspace_and_a_place():
    out = C.c_uint32(9)
    assert B.lib().tsq_cache_workspace_status(None, C.byref(out), None) == B.lib().tsq_cache_workspace_status(PTR, None, None) == INVALID
    assert B.lib().tsq_cache_workspace_status(PTR + 4, C.byref(out), None) == INVALID and out.value == 9


def slots(page=16, held=PTR, added=PTR, requests=3, free=PTR, n_free=4, start=PTR, lengths=PTR, table=PTR, width=5, out=PTR, tokens=9, taken=PTR):
    return B.lib().tsq_cache_slots(page, held, added, requests, free, n_free, start, lengths, table, width, out, tokens, taken, None)


@pytest.mark.parametrize("change,status", [
    (dict(page=0), INVALID), (dict(page=20), UNSUPPORTED), (dict(page=256), UNSUPPORTED), (dict(requests=-1), INVALID), (dict(requests=8193), UNSUPPORTED),
    (dict(held=None), INVALID), (dict(added=None), INVALID), (dict(free=None), INVALID), (dict(n_free=-1), INVALID), (dict(start=None), INVALID),
    (dict(lengths=None), INVALID), (dict(table=None), INVALID), (dict(width=-1), INVALID), (dict(out=None), INVALID), (dict(tokens=-1), INVALID),
    (dict(tokens=2 ** 31), INVALID), (dict(taken=None), INVALID), (dict(held=PTR + 2), INVALID), (dict(table=PTR + 1), INVALID)])
def test_slots(change, status):
    assert slots(**change) == status


@pytest.mark.parametrize("call", ["workspace_init", "workspace_status"])
def test_workspaces_on_the_host(call):
    import torch
    of = B.Cache.__new__(B.Cache)                                       # a cache's tensors need a device
    of.device = 0
    with pytest.raises(AssertionError):
        getattr(of, call)(torch.zeros(1 << 20, dtype=torch.uint8))
