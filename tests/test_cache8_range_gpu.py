"""Values, scales and page numbers at the ends of what the cache in 8 bits and attention with a window take, on the GPU
against 64 bits.

Tolerance of attention, from the arithmetic (u: half a unit in the last place of the outputs' type):
  a logit errs by d as in cache8_ref; a weight by 2 d + 2^-19 relative and, of n terms, n 2^-24.
  rows (few per key): a weight is two f16 halves, 2^-20 of it at the most and half a step of the second one, 2^-25, where the
  row's largest is 2^12 at the least: 2^-37 of that, or all of it where it is less.  Up to 2^6 times that where pages that differ
  no more than so share one product: 2^-31, and twice for two roundings.
  tiles (many rows): a weight times its page's value scale has 11 bits, and half a step of f16, 2^-25, where the row's
  largest such product is 2^8 at the least: 2^-33 of that, and twice; rows taken again have less.
Times |v| of its own key, summed, plus one rounding to the type."""
import math

import pytest
import torch

import decoder_ref as ref
from test_cache8_gpu import BF16, F16, F32, Held, ints, pp, tables  # noqa: F401

pytestmark = pytest.mark.gpu


def attend(q, k, v, table, starts, lens, scale, window, sinks, rows, key_bits=33):
    """(out, lse, tolerance of out, tolerance of lse) in float64; k, v [pages][H][page][D] in float64."""
    T, Hq, D = q.shape
    pages, H, page, _ = k.shape
    G, dt = Hq // H, q.dtype
    out, tol = torch.zeros((T, Hq, D), dtype=torch.float64), torch.full((T, Hq, D), ref.TINY[dt], dtype=torch.float64)
    lse, tl = torch.full((T, Hq), -math.inf, dtype=torch.float64), torch.zeros((T, Hq), dtype=torch.float64)
    for t, (b, n) in enumerate(ref.seen_keys(T, starts, lens, True)):
        key = torch.arange(n)
        key = key[(key >= n - window) | (key < sinks)]
        ip, io = table[b, key // page].long(), key % page
        good = (ip >= 0) & (ip < pages)
        ip, io = ip[good], io[good]
        if not len(ip):
            continue
        for h in range(H):
            kk, vv, hs = k[ip, h, io], v[ip, h, io], slice(h * G, (h + 1) * G)
            x = q[t, hs].double()
            s = scale * (x @ kk.T)
            d = scale * (x.abs() @ kk.abs().T).amax(-1, keepdim=True) * ((D + 12) * 2.0 ** -24 + 2.0 ** -key_bits)
            d = d + scale * 2.0 ** -39 * (x.abs().amax(-1, keepdim=True) * kk.abs().sum(-1)).amax(-1, keepdim=True)
            p = torch.softmax(s, -1)
            rel = 2 * d + 2.0 ** -19 + len(ip) * 2.0 ** -24 + (2.0 ** -20 if rows else 2.0 ** -11)
            out[t, hs], lse[t, hs] = p @ vv, torch.logsumexp(s, -1)
            if rows:
                lost = torch.minimum(p, 2.0 ** -30 * p.amax(-1, keepdim=True)) @ vv.abs()
            else:
                y = p * vv.abs().amax(-1)
                lost = torch.minimum(y, 2.0 ** -32 * y.amax(-1, keepdim=True)).sum(-1, keepdim=True)
            tol[t, hs] += rel * (p @ vv.abs()) + lost + ref.UNIT[dt] * out[t, hs].abs() * 1.01
            tl[t, hs] = d[:, 0] + 2.0 ** -19 + len(ip) * 2.0 ** -24 + 2.0 ** -22 * lse[t, hs].abs()
    return out, lse, tol, tl


def in_bf16(q, k, v, table, starts, lens, scale, window, sinks):
    """The same for one sequence over a cache in bf16, all keys at once on the GPU: weights of many rows have 8 bits."""
    n, Hq, D = q.shape
    _, H, page, _ = k.shape
    L, ids = lens[0], table[0].long()
    kk, vv = (x[ids].transpose(1, 2).reshape(-1, H, D)[:L].double().cuda() for x in (k, v))
    x = q.double().cuda().view(n, H, Hq // H, D)
    seen, at = torch.arange(L - n + 1, L + 1, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
    hide = ((at >= seen) | ((at < seen - window) & (at >= sinks)))[:, None, None]
    s = (torch.einsum("nhgd,shd->nhgs", x, kk) * scale).masked_fill(hide, -math.inf)
    d = torch.einsum("nhgd,shd->nhgs", x.abs(), kk.abs()).masked_fill(hide, 0).amax(-1, keepdim=True) * scale * (D + 12) * 2.0 ** -24
    p = torch.softmax(s, -1)
    out, mag = (torch.einsum("nhgs,shd->nhgd", p, y) for y in (vv, vv.abs()))
    tol = (2 * d + 2.0 ** -19 + L * 2.0 ** -24 + 2.0 ** -8) * mag + ref.UNIT[q.dtype] * out.abs() * 1.01 + ref.TINY[q.dtype]
    lse = torch.logsumexp(s, -1)
    tl = d[..., 0] + 2.0 ** -19 + L * 2.0 ** -24 + 2.0 ** -22 * lse.abs()
    return [y.reshape(n, Hq, *y.shape[3:]).cpu() for y in (out, lse, tol, tl)]


def close(got, want, tol):
    """Within tolerances, row by row: what is finite there is finite here."""
    got = got.double().cpu()
    worst = float(((got - want).abs() / tol).max())
    assert torch.isfinite(got).all() and worst <= 1, worst


def over_codes(pp, dt, H, G, D, page, L, n, window, sinks, change, rows, seed=0, status=0, q=None):
    """One call over a cache in 8 bits that `change(h, table)` has changed on the CPU."""
    need = -(-L // page)
    h = Held(pp, need + 2, H, page, D, dt, seed)
    table = tables([L], page, need + 2, seed=seed)
    change(h, table)
    for i in range(2):
        h.dc[i].copy_(h.c[i])
        h.ds[i].copy_(h.s[i])
    k, v = h.values()
    starts = None if n == 1 else [0, n]
    if q is None:
        q = torch.randn((n, H * G, D), generator=torch.Generator().manual_seed(seed + 1)).to(dt)
    out, lse = torch.full((n, H * G, D), math.nan, device="cuda", dtype=dt), torch.full((n, H * G), math.nan, device="cuda")
    try:
        pp.pp_attn_window(h.cache, q.cuda(), None if starts is None else ints(starts).cuda(), table.cuda(), ints([L]).cuda(), 0.125,
                          pp.PP_ATTN_CAUSAL, window, sinks, out, lse)
        assert h.status() == status
        want, wl, tol, tl = attend(q, k, v, table, starts, [L], 0.125, window, sinks, rows)
        close(out, want, tol)
        seen = torch.isfinite(wl)
        close(lse.cpu()[seen], wl[seen], tl[seen])
    finally:
        h.close()


# ------------------------------------------------------------------ pages of 8 and 16: several value scales in one product

@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("page", [8, 16, 32])
@pytest.mark.parametrize("power", [3, 5, 20, 40, 90])
@pytest.mark.parametrize("where", ["ahead", "left", "faint"])
def test_a_page_of_large_values_beside_small_ones(pp, dt, page, power, where):
    """Values 2^power times as large on a page that a draft's last token begins and those before it do not see; that windows have
    left but the first token's; that all see, with weights of some 2^-73.  Other pages are their neighbours in one tile."""
    D, L, n, window = 64, 13 * page + 1, 6, 1000
    if where == "left":
        n, window = 2, 8 * page  # the first token's window begins with the last key of page 4
        L = 13 * page
    if where == "faint":
        n = 1
    q = (1 + 0.1 * torch.randn((n, 4, D), generator=torch.Generator().manual_seed(2))).to(dt)

    def change(h, table):
        for i in range(2):  # (scores near 0, so that every key counts)
            h.s[i] *= 0.02 if i == 0 else 1
        id = int(table[0, {"ahead": 13, "left": 4, "faint": 5}[where]])
        h.s[1][id] *= 2.0 ** power
        if where == "faint":
            h.c[0][id], h.s[0][id] = -127, 0.05

    over_codes(pp, dt, 1, 4, D, page, L, n, window, 0, change, True, q=q)


# ------------------------------------------------------------------ values up to the largest of the type

def of_scales(powers):
    """Value scales of 2^(e - 1) to 2^e, with e from `powers` in turn along the pages, and codes from 0 on: sums of many large values."""
    def change(h, table):
        h.c[1].abs_()
        for w in range(table.shape[1]):
            id = int(table[0, w])
            h.s[1][id] = (0.5 + h.s[1][id] / h.s[1].max() / 2) * 2.0 ** powers[w % len(powers)]
    return change


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("L,n", [(40, 1), (700, 1), (9000, 1), (90, 5), (400, 40)])
@pytest.mark.parametrize("powers", [[100], [110], [120], [70, 71, 69], [120, 120, 120, 120, 120, 120, 120, 120, 0], [-60, -60, 120], [-106], [-140], [-60] * 100 + [120] * 41])
def test_values_of_any_size_by_rows(pp, dt, page, L, n, powers):
    """Outputs are averages of values up to 2^127, and sums of many such pass every type.  Short, split over CTAs, joined in two
    levels, drafts, and a chunk on few rows' kernel (one head)."""
    over_codes(pp, dt, 1, 2, 64, page, L, n, 10 ** 6, 0, of_scales(powers), True)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_values_of_any_size_that_others_see(pp, dt):
    """A draft's last token brings values near the type's largest: those before it are as if they were not there."""
    for page in (8, 16, 64):
        def change(h, table):
            h.s[1][int(table[0, 3])] = 2.0 ** 120
        over_codes(pp, dt, 1, 4, 64, page, 3 * page + 1, 5, 10 ** 6, 0, change, True)


@pytest.mark.parametrize("H,G,n,L,window,sinks", [(8, 2, 64, 500, 300, 0), (8, 4, 40, 1500, 1000, 40), (16, 1, 256, 700, 690, 3), (2, 4, 128, 9000, 8000, 0)])
@pytest.mark.parametrize("power", [0, 90, 110, 120, 127])
@pytest.mark.parametrize("rise", [0, 7, 20, 58, -58])
def test_windows_over_values_of_any_size_by_tiles(pp, H, G, n, L, window, sinks, power, rise):
    """Chunks in bf16 whose scores rise (or fall) along the keys by so many powers of two, over values near the type's largest:
    outputs are averages of them."""
    D, page, dt = 64, 64, BF16
    g = torch.Generator().manual_seed(5)
    pages = -(-L // page)
    table = tables([L], page, pages)
    k, v = torch.zeros((pages, H, page, D)), torch.zeros((pages, H, page, D))
    at = torch.arange(pages * page).view(pages, 1, page, 1) / L * rise / (D * 0.125 * 1.4427)  # logits in powers of two: rise times the place
    k[table[0].long()] = at + 0.02 * torch.randn((pages, H, page, D), generator=g)
    v[table[0].long()] = (0.5 + 0.49 * torch.rand((pages, H, page, D), generator=g)) * 2.0 ** power
    k, v, q = k.to(dt), v.to(dt), (1 + 0.1 * torch.randn((n, H * G, D), generator=g)).to(dt)
    cache = pp.pp_cache_create(k.cuda(), v.cuda())
    out, lse = torch.full((n, H * G, D), math.nan, device="cuda", dtype=dt), torch.full((n, H * G), math.nan, device="cuda")
    try:
        pp.pp_attn_window(cache, q.cuda(), ints([0, n]).cuda(), table.cuda(), ints([L]).cuda(), 0.125, pp.PP_ATTN_CAUSAL, window,
                          sinks, out, lse)
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        torch.cuda.synchronize()
        pp.pp_cache_destroy(cache)
    want, wl, tol, tl = in_bf16(q, k, v, table, [0, n], [L], 0.125, window, sinks)
    close(out, want, tol)
    close(lse, wl, tl)


# ------------------------------------------------------------------ tiles of rows over codes

TILED = [(16, 8, 64, 16, 170, 48), (16, 4, 128, 64, 700, 100), (8, 8, 128, 64, 2100, 40)]  # H, G, D, page, length, tokens; the last is split


@pytest.mark.parametrize("case", TILED)
@pytest.mark.parametrize("powers", [[-20], [-100], [-125], [-130], [-140], [100], [120], [120, -120], [-106, -106, -106, 0]])
@pytest.mark.parametrize("window", [10 ** 6, 70])
def test_values_of_any_size_by_tiles(pp, case, powers, window):
    H, G, D, page, L, n = case
    over_codes(pp, BF16, H, G, D, page, L, n, window, 0, of_scales(powers), False)


@pytest.mark.parametrize("dt", [F16, BF16])
def test_scales_below_normal_numbers_by_tiles(pp, dt):
    """The largest value scale in sight has no reciprocal in fp32."""
    for H, G, D, page, L, n in TILED:
        over_codes(pp, dt, H, G, D, page, L, n, 10 ** 6, 0, of_scales([-130]), False)
        over_codes(pp, dt, H, G, D, page, L, n, 10 ** 6, 0, of_scales([-148]), False)


def last_pages_larger(power, pages, more=None):
    """The last `pages` pages have values 2^power times those before them."""
    def change(h, table):
        for w in range(table.shape[1] - pages, table.shape[1]):
            h.s[1][int(table[0, w])] *= 2.0 ** power
        if more is not None:
            more(h, table)
    return change


@pytest.mark.parametrize("H,G,D,page,L,n,window,last", [(16, 8, 64, 16, 170, 48, 20, 2), (16, 8, 128, 64, 700, 100, 60, 1), (8, 8, 128, 64, 2100, 40, 1500, 1),
                                                        (16, 4, 80, 8, 333, 90, 10 ** 6, 3)])
@pytest.mark.parametrize("power", [40, 80, 88, 95, 120, 124])
def test_rows_that_see_small_pages_alone_by_tiles(pp, H, G, D, page, L, n, window, last, power):
    """Whatever the values are that other tokens of their tile see, down to a ratio that log2 of the scales no longer holds in the weights."""
    over_codes(pp, BF16, H, G, D, page, L, n, window, 0, last_pages_larger(power, last), False)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("H,G,D,page,L,n,window", [(16, 8, 64, 16, 170, 48, 16), (16, 8, 128, 64, 700, 100, 60), (1, 4, 64, 16, 170, 5, 16)])
def test_scales_of_zero(pp, dt, H, G, D, page, L, n, window):
    """Pages whose value scale is 0 hold zeros, whatever their codes are."""
    def change(h, table):
        for w in range(0, table.shape[1] - 1):
            if w % 4 != 1:
                h.s[1][int(table[0, w])] = 0
    over_codes(pp, dt, H, G, D, page, L, n, window, 0, last_pages_larger(100 if dt is BF16 else 4, 1, change), n * G * H < 1000)


# ------------------------------------------------------------------ entries of the table

@pytest.mark.parametrize("codes", [True, False])
@pytest.mark.parametrize("H,G,n", [(16, 8, 48), (1, 4, 5)])
@pytest.mark.parametrize("entry", [-2 ** 31, -2 ** 31 + 1, -1, 2 ** 31 - 1])
def test_entries_that_are_no_pages(pp, codes, H, G, n, entry):
    """Each is recorded and skipped by every kernel where tokens see it, and looked at by none where they do not."""
    D, page, L, dt = 64, 16, 170, F16
    h = Held(pp, 13, H, page, D, dt)
    k, v = h.values()
    pool = [x.to(dt) for x in (k, v)]
    cache = h.cache if codes else pp.pp_cache_create(pool[0].cuda(), pool[1].cuda())
    k, v = (k, v) if codes else [x.double() for x in pool]
    q = torch.randn((n, H * G, D), generator=torch.Generator().manual_seed(1)).to(dt)
    try:
        for w, window, status in ((8, 10 ** 6, pp.PP_CACHE_BAD_PAGE), (0, 10 ** 6, pp.PP_CACHE_BAD_PAGE), (10, 10 ** 6, pp.PP_CACHE_BAD_PAGE), (3, 50, 0)):
            table = tables([L], page, 13)
            table[0, w] = entry
            out, lse = torch.empty((n, H * G, D), device="cuda", dtype=dt), torch.empty((n, H * G), device="cuda")
            pp.pp_attn_window(cache, q.cuda(), ints([0, n]).cuda(), table.cuda(), ints([L]).cuda(), 0.125, pp.PP_ATTN_CAUSAL, window, 0, out, lse)
            assert pp.pp_cache_device_status(cache) == status
            want, wl, tol, tl = attend(q, k, v, table, [0, n], [L], 0.125, window, 0, False, 20)
            close(out, want, tol)
            close(lse, wl, tl)
    finally:
        torch.cuda.synchronize()
        if not codes:
            pp.pp_cache_destroy(cache)
        h.close()


@pytest.mark.parametrize("dt,H,G,D,page,L,n,window", [(F32, 2, 3, 256, 16, 500, 1, 300), (BF16, 1, 5, 256, 128, 3000, 1, 10 ** 6), (F32, 1, 16, 128, 256, 700, 3, 10 ** 6),
                                                      (BF16, 2, 8, 16, 8, 90, 2, 33), (F32, 4, 1, 48, 16, 5000, 1, 4000), (BF16, 1, 64, 128, 16, 40, 1, 10 ** 6)])
@pytest.mark.parametrize("powers", [[120], [0, 120], [90, -30, 5], [-100, 0, 60]])
def test_values_of_any_size_in_other_layouts(pp, dt, H, G, D, page, L, n, window, powers):
    over_codes(pp, dt, H, G, D, page, L, n, window, 7, of_scales(powers), True)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,most,page", [(700, 300, 16), (5, 4000, 64), (40, 900, 8)])
def test_sequences_of_large_values_beside_others(pp, dt, B, most, page):
    """Some sequences of a batch, and in some only the last pages, have values near the types' largest: CTAs go from one to the other."""
    H, G, D = 1, 2, 64
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, most, (B,), generator=g).tolist()
    need = sum(-(-v // page) for v in lens)
    h = Held(pp, need, H, page, D, dt)
    table = tables(lens, page, need)
    for b, v in enumerate(lens):
        w = -(-v // page)
        for i in range({0: 0, 1: w // 2}.get(b % 4, w), w):
            h.s[1][int(table[b, i])] *= 2.0 ** 124
    h.ds[1].copy_(h.s[1])
    k, v = h.values()
    q = torch.randn((B, H * G, D), generator=g).to(dt)
    out, lse = torch.full((B, H * G, D), math.nan, device="cuda", dtype=dt), torch.full((B, H * G), math.nan, device="cuda")
    try:
        pp.pp_attn_forward(h.cache, q.cuda(), None, table.cuda(), ints(lens).cuda(), 0.125, 0, None, out, lse)
        assert h.status() == 0
        want, wl, tol, tl = attend(q, k, v, table, None, lens, 0.125, 2 ** 31 - 1, 0, True)
        close(out, want, tol)
        seen = torch.isfinite(wl)
        close(lse.cpu()[seen], wl[seen], tl[seen])
    finally:
        h.close()
