"""The decoder operators on the GPU where they can go wrong: weights far below a row's largest, token ranges that do not
fit, statistics of NaN, mixed batches, turns at large positions, views at odd places, captured chains."""
import math
from fractions import Fraction

import pytest
import torch

import decoder_ref as ref
from test_decoder_gpu import BF16, Case, F16, F32, freqs, pp, tile_kernel_runs  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ f16 weights


def sink_case(pp, G, H, D, page, lens, tokens, gap):
    """Key 3 of each sequence draws almost all weight and holds zeros; the others' logits lie `gap` below (scale 1)."""
    c = Case(pp, F16, G, H, D, page, lens, tokens, seed=int(gap) + D, trash=False)
    g = torch.Generator().manual_seed(3)
    c.k = (0.02 * torch.randn(c.k.shape, generator=g)).to(F16)
    c.v = (1 + 0.25 * torch.randn(c.v.shape, generator=g)).to(F16)
    c.q = (0.3 * torch.randn(c.q.shape, generator=g)).to(F16)
    c.k[..., 0] = 0
    c.q[..., 0] = gap / 8
    for b in range(len(lens)):
        c.k[int(c.table[b, 0]), :, 3, 0] = 8
        c.v[int(c.table[b, 0]), :, 3] = 0
    for d, h in ((c.kd, c.k), (c.vd, c.v), (c.qd, c.q)):
        d.copy_(h)
    return c


@pytest.mark.parametrize("gap", [8.0, 14.0, 16.0, 18.0])
@pytest.mark.parametrize("G,H,D,lens,tokens", [(2, 4, 64, [4096] * 40, None), (4, 2, 128, [4096] * 70, None),
                                               (2, 1, 64, [9000], [300]), (8, 8, 64, [1500], [700]), (4, 2, 128, [5000, 900], [200, 900])])
def test_f16_weights_far_below_the_largest(pp, G, H, D, lens, tokens, gap):
    """A key that draws almost all weight and holds nothing, the others some 2^-26 of it each: what is left is their sum.
    To the bound of the reference comes what f16 loses of a weight below its smallest normal number, 2^-25 where the row's
    largest weight is at least 2^13: 2^-38 of it for every key, of values below 3."""
    c = sink_case(pp, G, H, D, 64, lens, tokens, gap)
    try:
        out, lse = c.attend(1.0)
        want, wl, tol, tl = ref.attend(c.q, c.k, c.v, c.table, c.starts, lens, 1.0, True)
        assert float(c.v.abs().max()) < 3
        assert ref.worst(out, want, tol + 2.0 ** -38 * 3 * max(lens)) <= 1
        assert ref.worst(lse, wl, tl) <= 1
        assert c.status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("tokens", [None, [400]])
def test_logits_of_any_size_stay_in_range(pp, dt, tokens):
    """Logits of 2^20 to 2^32, where neighbouring fp32 numbers are up to 2^8 apart: their own errors leave no digits to
    compare, but an output stays a mean of values."""
    for size in (4000.0, 60000.0):
        c = Case(pp, dt, 4, 2, 64, 64, [700], tokens, seed=31, trash=False)
        try:
            g = torch.Generator().manual_seed(6)
            for w in range(c.table.shape[1] - 1):  # later pages hold larger keys
                i = int(c.table[0, w])
                c.k[i] = (torch.randn(c.k[i].shape, generator=g) * (0.05 + 0.02 * w) * size).clamp(-60000, 60000).to(dt)
            c.q = (torch.randn(c.q.shape, generator=g) * size / 20).clamp(-60000, 60000).to(dt)
            c.kd.copy_(c.k)
            c.qd.copy_(c.q)
            out, lse = c.attend(1.0)
            assert torch.isfinite(out).all() and torch.isfinite(lse).all()
            assert float(out.abs().max()) <= float(c.v.abs().max()) * (1 + 2.0 ** -6)
        finally:
            c.close()


# ------------------------------------------------------------------ the device status word


def test_status_reads_lose_no_bit(pp):
    """What a side stream meets right after the word was read and cleared is there at the next reading."""
    k = torch.zeros((2, 1, 16, 64), device="cuda")
    cache = pp.pp_cache_create(k, k.clone(), torch.zeros((2, 1, 2, 64), device="cuda", dtype=torch.int8), torch.zeros((2, 1), device="cuda"))
    try:
        bad = torch.tensor([7], device="cuda", dtype=torch.int32)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        for _ in range(3000):
            pp.pp_cache_summarize(cache, bad, s)
            assert pp.pp_cache_device_status(cache) == pp.PP_CACHE_BAD_PAGE
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        pp.pp_cache_destroy(cache)


# ------------------------------------------------------------------ which kernel runs


@pytest.mark.parametrize("selected", [False, True])
def test_single_tokens_in_ranges_take_the_row_kernel(pp, tmp_path, selected):
    """One token each of many sequences, given as ranges: tiles would hold a token's rows each.  The same bits as without
    ranges."""
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 300, (64,), generator=g).tolist()
    lens[5], lens[40] = 4000, 1
    c = Case(pp, F16, 4, 8, 64, 16, lens, [1] * 64, seed=3)
    try:
        sel = None
        if selected:
            sel = torch.full((c.T, 8, 6), -1, dtype=torch.int32)
            for t, n in enumerate(lens):
                some = torch.randperm(-(-n // 16), generator=g)[:6]
                sel[t, :, : len(some)] = some.to(torch.int32)
        assert not tile_kernel_runs(c, tmp_path, None if sel is None else sel.cuda())
        out = c.check(sel=sel)
        c.sd = None
        again, _ = c.attend(sel=None if sel is None else sel.cuda())
        assert torch.equal(out, again)
        assert c.status() == 0
    finally:
        c.close()


def test_a_chunk_among_single_tokens_takes_tiles(pp, tmp_path):
    g = torch.Generator().manual_seed(2)
    lens = torch.randint(1, 300, (24,), generator=g).tolist()
    tokens = [1] * 24
    tokens[7], lens[7] = 500, 700
    c = Case(pp, BF16, 4, 2, 64, 16, lens, tokens, seed=3)
    try:
        assert tile_kernel_runs(c, tmp_path)
        c.check()
        assert c.status() == 0
    finally:
        c.close()


def test_long_lists_of_pages_take_the_row_kernel(pp, tmp_path):
    """Lists so long that a tile's entries pass 2^31: only the first ones count, one for each page that a token sees."""
    keep = 2 ** 24
    c = Case(pp, BF16, 1, 1, 64, 16, [200], [160], seed=3)
    try:
        sel = torch.full((c.T, 1, keep), -1, dtype=torch.int32, device="cuda")
        sel[:, 0, :3] = torch.tensor([1, 0, 2], dtype=torch.int32)
        assert not tile_kernel_runs(c, tmp_path, sel)
        out, _ = c.attend(sel=sel)
        want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.lens, 1 / 8.0, True, sel[:, :, :3].cpu())
        assert ref.worst(out, want, tol) <= 1
        assert c.status() == 0
    finally:
        c.close()


def test_tables_near_2_31_keys_are_refused(pp):
    k = torch.zeros((1, 1, 8, 64), device="cuda", dtype=F16)
    cache = pp.pp_cache_create(k, k.clone())
    try:
        x, n = torch.zeros((1, 1, 64), device="cuda", dtype=F16), torch.zeros(2, dtype=torch.int32, device="cuda")
        # refused before anything of the table is read
        got = pp.lib.pp_attn_forward(cache, 1, x.data_ptr(), 64, 64, 1, 1, None, n.data_ptr(), (2 ** 31 - 8) // 8, n.data_ptr(), 1.0, 0,
                                     None, 0, x.data_ptr(), None, None)
        assert got == pp.PP_ERR_UNSUPPORTED
    finally:
        pp.pp_cache_destroy(cache)


# ------------------------------------------------------------------ token ranges that do not fit


@pytest.mark.parametrize("call", ["rows", "tiles", "rows_selected", "tiles_selected", "select", "select_single"])
@pytest.mark.parametrize("kind", ["late", "short", "long", "before", "descending"])
def test_token_ranges_that_do_not_fit_are_recorded(pp, tmp_path, call, kind):
    many = call.startswith("tiles")
    tokens = [150, 60, 90] if many else [1, 1, 2] if call == "select_single" else [6, 4, 5]
    c = Case(pp, F16, 8, 1, 64, 16, [400, 300, 200], tokens, seed=4, summaries=True, trash=False)
    try:
        T, s = c.T, list(c.starts)
        s[0], s[-1] = {"late": (1, T), "short": (0, T - 1), "long": (0, T + 1), "before": (-1, T), "descending": (0, T)}[kind]
        if kind == "descending":
            s[1], s[2] = s[2], s[1]
        sel = torch.zeros((T, 1, 4), dtype=torch.int32, device="cuda") if "select" in call else None
        if call.startswith("tiles"):
            assert tile_kernel_runs(c, tmp_path, sel)

        def run():
            if call.startswith("select"):
                pp.pp_cache_select(c.cache, c.qd, c.sd, c.td, c.ld, pp.PP_ATTN_CAUSAL, 1, 2, sel)
            else:
                c.attend(sel=sel)

        run()
        assert c.status() == 0
        c.sd.copy_(torch.tensor(s))
        run()
        assert c.status() & pp.PP_CACHE_BAD_LENGTH
        if kind in ("late", "short") and not call.startswith("select"):  # ranges that fit are answered all the same
            out, _ = c.attend(sel=sel)
            want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.lens, 1 / 8.0, True, None if sel is None else sel.cpu())
            mid = slice(s[1], s[2])
            assert ref.worst(out[mid], want[mid], tol[mid]) <= 1
    finally:
        c.close()


# ------------------------------------------------------------------ statistics of NaN


@pytest.mark.parametrize("dt,lens,tokens", [(F32, [100, 60], None), (F16, [100, 60], None), (BF16, [3000, 60], None), (F32, [6000, 60], None),
                                            (BF16, [100, 60], [9, 3]), (BF16, [500, 400], [400, 300])])
def test_rows_of_nan_have_nan_statistics(pp, dt, lens, tokens):
    """A query that is NaN has an output and a log-sum of NaN; minus infinity is for rows that see no key."""
    c = Case(pp, dt, 2, 2, 64, 16, lens, tokens, seed=9)
    try:
        n0 = 1 if tokens is None else tokens[0]
        c.q[:n0, 1, 3] = math.nan
        c.qd.copy_(c.q)
        out, lse = c.attend()
        assert torch.isnan(out[:n0, 1]).all() and torch.isnan(lse[:n0, 1]).all()
        others = [0, 2, 3]
        want, wl, tol, tl = ref.attend(c.q, c.k, c.v, c.table, c.starts, lens, 1 / 8.0, True)
        assert ref.worst(out[:, others], want[:, others], tol[:, others]) <= 1
        assert ref.worst(lse[:, others], wl[:, others], tl[:, others]) <= 1
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F32, BF16])
def test_one_nan_logit_among_far_larger_ones(pp, dt):
    """A NaN in a part of a long sequence whose weights vanish beside another part's: NaN all the same."""
    c = Case(pp, dt, 2, 1, 64, 64, [20000], None, seed=9)
    try:
        c.q[:] = 1
        for key, value in ((15000, 30.0), (100, math.nan)):
            c.k[int(c.table[0, key // 64]), 0, key % 64] = value
        c.kd.copy_(c.k)
        c.qd.copy_(c.q)
        out, lse = c.attend()
        assert torch.isnan(out).all() and torch.isnan(lse).all()
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lens,tokens", [([2500], [2400]), ([3000], [150])])
def test_rows_computed_again_are_the_same_each_time(pp, dt, lens, tokens):
    """Most rows of each tile meet a NaN that they do not see, or see and get by the warp over what their own threads wrote:
    the reference's values, and the same bits twenty times over (one share per tile, and several)."""
    c = Case(pp, dt, 4, 2, 64, 16, lens, tokens, seed=12)
    try:
        for key in range(lens[0] - tokens[0] + 40, lens[0], 64):
            c.v[int(c.table[0, key // 16]), :, key % 16, 5] = math.nan
        c.vd.copy_(c.v)
        first, l1 = c.attend()
        for _ in range(20):
            again, l2 = c.attend()
            assert torch.equal(torch.nan_to_num(first, nan=99.0), torch.nan_to_num(again, nan=99.0)) and torch.equal(l1, l2)
        some = slice(0, 120)
        c.starts, n = [0, 120], lens[0] - tokens[0] + 120
        want, wl, tol, tl = ref.attend(c.q[some], c.k, c.v, c.table, c.starts, [n], 1 / 8.0, True)
        fine = torch.isfinite(want)
        got = first[some].double().cpu()
        assert torch.equal(torch.isfinite(got), fine)
        assert ref.worst(torch.where(fine, got, 0.0), torch.where(fine, want, 0.0), tol) <= 1
        assert ref.worst(l1[some], wl, tl) <= 1
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("tokens", [None, [5, 3]])
def test_infinite_values_stay_infinite(pp, dt, tokens):
    """A value that is infinite gives outputs that are, of its sign, whatever its key's weight (also the row's largest)."""
    c = Case(pp, dt, 4, 2, 64, 16, [700, 40], tokens, seed=22)
    try:
        for key, d, x in ((3, 1, math.inf), (100, 2, -math.inf), (333, 3, math.inf), (333, 4, -math.inf)):
            c.v[int(c.table[0, key // 16]), :, key % 16, d] = x
        # key 333 is the largest of the first head's logits by far, and key 5 far below them
        c.k[int(c.table[0, 333 // 16]), 0, 333 % 16] = c.q[0, 0] * 2
        c.k[int(c.table[0, 0]), 0, 5] = -c.q[0, 0]
        c.v[int(c.table[0, 0]), 0, 5, 6] = math.inf
        c.kd.copy_(c.k)
        c.vd.copy_(c.v)
        out, _ = c.attend()
        want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.lens, 1 / 8.0, True)
        got, fine = out.double().cpu(), torch.isfinite(want)
        assert torch.equal(torch.where(fine, torch.zeros_like(got), got), torch.where(fine, torch.zeros_like(want), want))
        assert ref.worst(torch.where(fine, got, 0.0), torch.where(fine, want, 0.0), tol) <= 1
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("G,D,page,lens,tokens", [(2, 64, 16, [300], [100]), (1, 128, 64, [500], [300]), (4, 96, 8, [450, 100], [420, 100]),
                                                  (8, 64, 128, [4000], [140]), (1, 64, 16, [90, 40], [3, 16]), (3, 256, 32, [120], [80])])
def test_what_is_not_finite_reaches_the_rows_that_see_it(pp, dt, G, D, page, lens, tokens):
    """NaN and infinities all over a chunk: single values, a key's whole values, the same value twice with both signs, a key
    that is NaN near the end.  Each value of each row is finite where the reference's is, and then within its bound."""
    c = Case(pp, dt, G, 2, D, page, lens, tokens, seed=21)
    try:
        def put(pool, key, d, x):
            pool[int(c.table[0, key // page]), :, key % page, d] = x

        first, n = lens[0] - tokens[0], tokens[0]
        put(c.v, first + n // 3, 5, math.nan)
        put(c.v, first + n // 3 + 1, 7, math.inf)
        put(c.v, first + n // 2, 9, -math.inf)
        put(c.v, first + n - n // 4, 9, math.inf)
        put(c.v, first + n - n // 5, slice(8, 16), math.inf)
        put(c.v, first // 2, 3, -math.inf)  # every row sees this one
        put(c.k, first + n - 1 - n // 9, 2, math.nan)
        put(c.v, first + n - 1, slice(None), math.nan)
        c.kd.copy_(c.k)
        c.vd.copy_(c.v)
        out, lse = c.attend()
        want, wl, tol, tl = ref.attend(c.q, c.k, c.v, c.table, c.starts, lens, 1 / math.sqrt(D), True)
        got, fine = out.double().cpu(), torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got == math.inf, want == math.inf)
        assert ref.worst(torch.where(fine, got, 0.0), torch.where(fine, want, 0.0), tol) <= 1
        sums = ~torch.isnan(wl)
        assert torch.equal(~torch.isnan(lse.cpu()), sums)
        assert ref.worst(torch.where(sums, lse.double().cpu(), 0.0), torch.where(sums, wl, 0.0), tl) <= 1
        assert c.status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("dt,T", [(BF16, 512), (F32, 64)])
@pytest.mark.parametrize("where", ["all rows see it", "half of them do"])
def test_a_value_that_is_not_finite_costs_little(pp, dt, T, where):
    """One NaN in a cache of 8192 keys: the call takes no more than ten times as long, and a millisecond (computing the rows
    again, each alone, took a thousand times as long)."""
    c = Case(pp, dt, 4, 4, 64, 64, [8192], [T], seed=21, trash=False)
    try:
        def best():
            ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            times = []
            for _ in range(4):
                ev[0].record()
                c.attend(lse=False)
                ev[1].record()
                torch.cuda.synchronize()
                times.append(ev[0].elapsed_time(ev[1]))
            return min(times)

        before = best()
        key = 100 if where == "all rows see it" else 8192 - T // 2
        c.vd[int(c.table[0, key // 64]), :, key % 64, 5] = math.nan
        assert best() <= 10 * before + 1
    finally:
        c.close()


# ------------------------------------------------------------------ turns


# pi to 60 places
PI = Fraction(314159265358979323846264338327950288419716939937510582097494, 10 ** 59)


@pytest.mark.parametrize("inter", [False, True])
def test_turns_at_any_position_and_frequency(pp, inter):
    """Frequencies that are no simple part of a turn, up to thousands of radians per position: the angle in exact
    arithmetic.  The turn's fraction is kept to 2^-64 per position and read to 2^-32, then rounded to fp32: 2^-25 of half a
    turn.  With both values of a pair 1 the sum of a cosine and a sine errs by at most 2 (2^-25 pi + 2^-30 + 2^-23) + 2^-23."""
    D, freq = 32, [1000.0, 1.0, 0.7300000001, 12345.678, 1e-3, 3.0e-7, 2 * math.pi, 0.1, -0.1, -777.7, 1e6 / 3, 5e9 / 7, 0.0, 1e-12, 31.4, 2.0]
    at = [0, 1, 12345, 999_999_937, 2 ** 31 - 1, -(2 ** 31), -7, 2 ** 30 + 1]
    rope = pp.pp_rope_create(D, None, freq, 1, inter)
    try:
        x = torch.ones((len(at), 1, D), device="cuda")
        out = torch.empty_like(x)
        pp.pp_qk_rotate(rope, torch.tensor([at], dtype=torch.int32, device="cuda"), -1.0, x, None, out, None, None, None)
        got = out.double().cpu()[:, 0]
        tol = 2 * (2.0 ** -25 * math.pi + 2.0 ** -30 + 2.0 ** -23) + 2.0 ** -23
        for t, p in enumerate(at):
            for j, f in enumerate(freq):
                turn = Fraction(p) * Fraction(f) / (2 * PI)
                a = float(turn - round(turn)) * 2 * math.pi
                lo, hi = (2 * j, 2 * j + 1) if inter else (j, D // 2 + j)
                assert abs(float(got[t, lo]) - (math.cos(a) - math.sin(a))) <= tol, (p, f)
                assert abs(float(got[t, hi]) - (math.cos(a) + math.sin(a))) <= tol, (p, f)
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)


# ------------------------------------------------------------------ views, fp32 sums, captured chains


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("inter", [False, True])
def test_rotations_and_stores_at_16_byte_offsets(pp, dt, inter):
    """Rows that begin 16 bytes, or one value, into a wider boundary, from a fused product: outputs and the cache."""
    T, Hq, H, D, page = 21, 4, 2, 64, 16
    step = 16 // torch.empty(0, dtype=dt).element_size()
    g = torch.Generator().manual_seed(8)
    w = torch.rand(D, generator=g) + 0.5
    pos = torch.randint(0, 900, (1, T), generator=g, dtype=torch.int32)
    slots = torch.randperm(3 * page, generator=g)[:T].to(torch.int32)
    rope = pp.pp_rope_create(D, None, freqs(D // 2), 1, inter)
    try:
        for off in (step, 2 * step, 1):
            fused = torch.randn((T, (Hq + 2 * H) * D + 2 * step), generator=g).to(dt)
            q, k, v = (fused[:, off + a * D: off + (a + n) * D].unflatten(1, (n, D)) for a, n in ((0, Hq), (Hq, H), (Hq + H, H)))
            fd = fused.cuda()
            qd, kd, vd = (fd[:, off + a * D: off + (a + n) * D].unflatten(1, (n, D)) for a, n in ((0, Hq), (Hq, H), (Hq + H, H)))
            want = [ref.rotate(x, w, 1e-6, pos, [0] * (D // 2), freqs(D // 2), inter) for x in (q, k)]
            # outputs that begin at such places too
            qo, ko = (torch.zeros(T * n * D + off, device="cuda", dtype=dt)[off:].view(T, n, D) for n in (Hq, H))
            pp.pp_qk_rotate(rope, pos.cuda(), 1e-6, qd, w.cuda(), qo, kd, w.cuda(), ko)
            for got, (y, tol) in zip((qo, ko), want):
                assert ref.worst(got, y, tol) <= 1
            kp, vp = (torch.zeros((3, H, page, D), device="cuda", dtype=dt) for _ in range(2))
            cache = pp.pp_cache_create(kp, vp)
            try:
                pp.pp_qkv_store(rope, cache, pos.cuda(), slots.cuda(), 1e-6, qd, w.cuda(), qo, kd, w.cuda(), vd)
                at = slots.long()
                assert ref.worst(qo, *want[0]) <= 1
                assert ref.worst(kp.cpu()[at // page, :, at % page], *want[1]) <= 1
                assert torch.equal(vp.cpu()[at // page, :, at % page], v)
                rest = torch.ones(3 * page, dtype=torch.bool)
                rest[at] = False
                rest = rest.nonzero()[:, 0]
                assert not kp.cpu()[rest // page, :, rest % page].any() and not vp.cpu()[rest // page, :, rest % page].any()
                assert pp.pp_cache_device_status(cache) == 0
            finally:
                pp.pp_cache_destroy(cache)
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)


@pytest.mark.parametrize("D,G,n", [(64, 1, 500), (96, 2, 700), (128, 4, 300), (256, 8, 200)])
def test_fp32_sums_are_fp32(pp, D, G, n):
    """fp32 products and sums throughout: a logit errs by d = (D + 8) 2^-24 scale sum |q k|, a weight by 2 d + 2^-19 (the
    exponential and its argument, of up to 16), n terms add n 2^-24.  No term for products of fewer bits."""
    c = Case(pp, F32, G, 1, D, 16, [n], None, seed=D, trash=False)
    try:
        out, lse = c.attend()
        ids = c.table[0, : -(-n // 16)].long()
        k, v = (x[ids, 0].reshape(-1, D)[:n].double() for x in (c.k, c.v))
        q = c.q[0].double()
        s, most = q @ k.T / math.sqrt(D), q.abs() @ k.abs().T / math.sqrt(D)
        assert float(s.abs().max()) < 16
        d = most.amax(1, keepdim=True) * (D + 8) * 2.0 ** -24
        p = torch.softmax(s, 1)
        tol = (2 * d + 2.0 ** -19 + n * 2.0 ** -24) * (p @ v.abs()) + 2.0 ** -23 * (p @ v).abs()
        assert ref.worst(out[0], p @ v, tol) <= 1
        assert ref.worst(lse[0], torch.logsumexp(s, 1), d[:, 0] + 2.0 ** -19 + n * 2.0 ** -24) <= 1
    finally:
        c.close()


def test_a_captured_chain(pp):
    """Store, summaries, selection and attention by split tiles as one graph, replayed on other tokens, positions, slots and
    lengths: the bits of the same calls one by one, and the reference's values."""
    T, G, H, D, page, W, keep = 260, 4, 2, 64, 16, 60, 12
    P = D // 2
    rope = pp.pp_rope_create(D, None, freqs(P))
    g = torch.Generator().manual_seed(5)
    pool = [torch.randn((W, H, page, D), generator=g).to(BF16) for _ in range(2)]

    class Side:
        def __init__(self):
            self.k, self.v = (x.cuda() for x in pool)
            self.codes, self.scales = torch.zeros((W, H, 2, D), dtype=torch.int8, device="cuda"), torch.zeros((W, H), device="cuda")
            self.cache = pp.pp_cache_create(self.k, self.v, self.codes, self.scales)
            self.fused = torch.zeros((T, (G + 2) * H, D), device="cuda", dtype=BF16)
            self.pos, self.slots = (torch.zeros((1, T), dtype=torch.int32, device="cuda") for _ in range(2))
            self.q, self.out = (torch.zeros((T, G * H, D), device="cuda", dtype=BF16) for _ in range(2))
            self.sel = torch.zeros((T, H, keep), dtype=torch.int32, device="cuda")
            self.lse = torch.zeros((T, G * H), device="cuda")
            self.table = torch.zeros((1, W), dtype=torch.int32, device="cuda")
            self.lens, self.starts = torch.tensor([T], dtype=torch.int32, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda")

        def run(self, s):
            f, flags = self.fused, pp.PP_ATTN_CAUSAL
            pp.pp_qkv_store(rope, self.cache, self.pos, self.slots[0], 1e-6, f[:, : G * H], None, self.q, f[:, G * H: (G + 1) * H], None,
                            f[:, (G + 1) * H:], s)
            pp.pp_cache_summarize(self.cache, self.table[0], s)
            pp.pp_cache_select(self.cache, self.q, self.starts, self.table, self.lens, flags, 1, 2, self.sel, s)
            pp.pp_attn_forward(self.cache, self.q, self.starts, self.table, self.lens, 0.125, flags, self.sel, self.out, self.lse, s)

        def load(self, x, pos, slots, table, n):
            self.fused.copy_(x)
            self.pos[0].copy_(pos)
            self.slots[0].copy_(slots)
            self.table[0].copy_(table)
            self.lens[0] = n

    a, b = Side(), Side()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    try:
        for side in (a, b):  # before the capture, every kernel once
            side.load(torch.zeros((T, (G + 2) * H, D)), torch.zeros(T), torch.arange(T), torch.arange(W), T)
            side.run(torch.cuda.current_stream())
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            a.run(s)
        for n in (W * page, 700, 301):
            x = torch.randn((T, (G + 2) * H, D), generator=g).to(BF16)
            pos = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32)
            table = torch.randperm(W, generator=g).to(torch.int32)
            key = torch.arange(n - T, n)
            slots = table[key // page] * page + (key % page).to(torch.int32)
            for side in (a, b):
                side.load(x, pos, slots, table, n)
            torch.cuda.synchronize()
            graph.replay()
            b.run(torch.cuda.current_stream())
            torch.cuda.synchronize()
            for i, j in ((a.k, b.k), (a.v, b.v), (a.codes, b.codes), (a.scales, b.scales), (a.sel, b.sel), (a.q, b.q), (a.out, b.out), (a.lse, b.lse)):
                assert torch.equal(i, j)
            codes, scales = ref.summarize(a.k.cpu())
            assert torch.equal(a.codes.cpu(), codes) and torch.equal(a.scales.cpu(), scales)
            sel = ref.select(a.q.cpu(), codes, scales, table[None], [0, T], [n], True, page, 1, 2, keep)
            assert torch.equal(a.sel.cpu(), sel)
            want, wl, tol, tl = ref.attend(a.q.cpu(), a.k.cpu(), a.v.cpu(), table[None], [0, T], [n], 0.125, True, sel)
            assert ref.worst(a.out, want, tol) <= 1 and ref.worst(a.lse, wl, tl) <= 1
        assert pp.pp_cache_device_status(a.cache) == 0 and pp.pp_cache_device_status(b.cache) == 0
    finally:
        torch.cuda.synchronize()
        for side in (a, b):
            pp.pp_cache_destroy(side.cache)
        pp.pp_rope_destroy(rope)
