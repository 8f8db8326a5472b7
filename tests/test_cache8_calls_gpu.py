"""Calls on the cache in 8 bits and with a window that other tests leave out: what a call with ranges that do not fit writes,
windows and first keys that hold every key, the same call many times."""
import math

import pytest
import torch

import cache8_ref as ref8
import decoder_ref as ref
from test_cache8_gpu import BF16, F16, F32, Held, ints, pp, tables  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("page,T", [(8, 6), (16, 300)])
@pytest.mark.parametrize("starts", [(0, 4, 7), (0, -1, 6), (1, 4, 6), (0, 7, 6), (0, 2, 5), (0, 6, 3), (-2, 3, 6), (2 ** 30, 3, 6), (0, 3, -2 ** 31)])
def test_append_with_ranges_that_do_not_fit(pp, dt, page, T, starts):
    """Recorded; a sequence whose own range fits is written as its tokens say, and nothing else is: neither the other's pages nor
    those that no sequence has."""
    H, D = 2, 32
    starts = [s * T // 6 if abs(s) < 100 else s for s in starts]
    if starts[2] == 7 * T // 6:
        starts[2] = T + 1
    need = -(-T // page) + 1
    lens = [need * page] * 2
    h = Held(pp, 2 * need + 6, H, page, D, dt, seed=3)
    table = tables(lens, page, h.c[0].shape[0])
    x = torch.randn((T, H, D), generator=torch.Generator().manual_seed(2)).to(dt)
    try:
        pp.pp_cache_append(h.cache, x.cuda(), (2 * x).cuda(), ints(starts).cuda(), table.cuda(), ints(lens).cuda())
        assert h.status() == pp.PP_CACHE_BAD_LENGTH
        for b in range(2):
            s0, s1 = starts[b], starts[b + 1]
            if 0 <= s0 <= s1 <= T:
                for i in range(2):
                    ref8.append(h.c[i], h.s[i], (1 + i) * x[s0:s1], table[b: b + 1], [0, s1 - s0], lens[b: b + 1], page)
        assert h.same()
    finally:
        h.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("H,G,D,page,lens,starts", [(1, 4, 128, 16, [300, 5, 0], None), (2, 2, 64, 32, [300, 70], [0, 100, 170]), (8, 4, 64, 16, [170], [0, 40]),
                                                    (16, 8, 128, 64, [700], [0, 60]), (1, 3, 96, 8, [90, 33], [0, 5, 9])])
def test_windowed_kernels_where_every_key_is_seen(pp, dt, codes, H, G, D, page, lens, starts):
    """A window of the longest length in a table that is wider, and first keys that are all: not the call without a window, as a
    window of the whole table is, but its numbers, to twice the tolerance against the definition."""
    T, L = len(lens) if starts is None else starts[-1], max(lens)
    need = sum(-(-v // page) for v in lens)
    table = tables(lens, page, need + 2, width=-(-L // page) + 3)
    h = Held(pp, need + 2, H, page, D, dt)
    k, v = h.values()
    if codes:
        cache = h.cache
    else:
        k, v = k.to(dt), v.to(dt)
        cache = pp.pp_cache_create(k.cuda(), v.cuda())
    q = torch.randn((T, H * G, D), generator=torch.Generator().manual_seed(4)).to(dt)
    a = (cache, q.cuda(), None if starts is None else ints(starts).cuda(), table.cuda(), ints(lens).cuda(), D ** -0.5, pp.PP_ATTN_CAUSAL)
    try:
        def call(f, *more):
            out, lse = torch.full((T, H * G, D), math.nan, device="cuda", dtype=dt), torch.full((T, H * G), math.nan, device="cuda")
            f(*a, *more, out, lse)
            return out.cpu().double(), lse.cpu().double()
        out, lse = call(pp.pp_attn_forward, None)
        _, wl, tol, tl = ref8.attend(q, k, v, table, starts, lens, D ** -0.5, True, 2 ** 31 - 1, 0, codes)
        for window, sinks in ((L, 0), (1, L), (L // 2, L - 1), (L + page, 3)):
            o, ls = call(pp.pp_attn_window, window, sinks)
            assert bool(((o - out).abs() <= 2 * tol).all()), (window, sinks)
            seen = torch.isfinite(wl)
            assert torch.equal(torch.isinf(ls), ~seen) and bool(((ls - lse)[seen].abs() <= 2 * tl[seen]).all())
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        torch.cuda.synchronize()
        if not codes:
            pp.pp_cache_destroy(cache)
        h.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("n,window", [(1, None), (1, 4096), (8, 4096), (64, None), (64, 4096), (700, None), (700, 4096)])
def test_chunks_give_the_same_bits_each_time(pp, codes, dt, n, window):
    """Rows and tiles, split along their keys or not, with and without a window: 20 calls, some without a wait in between."""
    H, G, D, page, L = 8, 4, 128, 64, 9000
    pages = -(-L // page)
    g = torch.Generator(device="cuda").manual_seed(1)
    table, lens = tables([L], page, pages).cuda(), ints([L]).cuda()
    q = torch.randn((n, H * G, D), device="cuda", generator=g).to(dt)
    h = Held(pp, pages if codes else 1, H, page, D, dt)
    if codes:
        cache = h.cache
    else:
        k, v = (torch.randn((pages, H, page, D), device="cuda", generator=g).to(dt) for _ in range(2))
        cache = pp.pp_cache_create(k, v)
    a = (cache, q, None if n == 1 else ints([0, n]).cuda(), table, lens, 0.09, pp.PP_ATTN_CAUSAL)
    try:
        outs = [torch.full((n, H * G, D), math.nan, device="cuda", dtype=dt) for _ in range(20)]
        for i, out in enumerate(outs):
            pp.pp_attn_forward(*a, None, out) if window is None else pp.pp_attn_window(*a, window, 16, out)
            if i % 3 == 0:
                torch.cuda.synchronize()
        assert pp.pp_cache_device_status(cache) == 0 and bool(torch.isfinite(outs[0].float()).all())
        assert all(torch.equal(o, outs[0]) for o in outs)
    finally:
        torch.cuda.synchronize()
        if not codes:
            pp.pp_cache_destroy(cache)
        h.close()
