"""The decoder operators on the GPU, through the binding, against their definitions in 64 bits (tests/decoder_ref.py):
rotations into tensors and into the cache, page summaries, selections, attention over all and over selected pages."""
import math
import re
import warnings

import pytest
import torch

import decoder_ref as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def pp():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import ppconv
    return ppconv


def freqs(P):
    return [10000.0 ** (-j / max(1, P)) for j in range(P)]


# ------------------------------------------------------------------ rotations

ROTATE = [
    # dtype, T, Hq, Hk, D, pairs, axes, interleaved
    (BF16, 1, 8, 8, 64, 32, 1, False),
    (BF16, 5, 4, 2, 128, 64, 3, False),
    (F16, 7, 3, 1, 80, 40, 3, True),
    (F32, 3, 5, 5, 64, 32, 3, False),
    (F32, 9, 2, 0, 96, 48, 2, True),
    (F16, 200, 12, 4, 128, 32, 3, False),   # a part of the head is not turned
    (BF16, 4, 2, 2, 80, 20, 3, False),      # pairs that do not divide into whole lanes
    (BF16, 4, 2, 2, 80, 20, 3, True),
    (F32, 2, 1, 1, 2, 1, 1, False),
    (F16, 3, 1, 2, 6, 1, 1, True),
    (BF16, 2, 1, 1, 256, 128, 8, False),
    (F32, 2, 1, 1, 256, 100, 2, True),
    (F16, 3, 2, 1, 64, 0, 1, False),        # nothing turned
    (BF16, 2500, 4, 1, 64, 32, 3, True),    # whole tokens per group of lanes
]


@pytest.mark.parametrize("dt,T,Hq,Hk,D,P,axes,inter", ROTATE)
def test_rotate(pp, dt, T, Hq, Hk, D, P, axes, inter):
    g = torch.Generator().manual_seed(T + D)
    q, k = torch.randn((T, Hq, D), generator=g).mul(3).to(dt), torch.randn((T, Hk, D), generator=g).to(dt)
    qw, kw = torch.rand(D, generator=g) + 0.5, torch.rand(D, generator=g) - 0.5
    pos = torch.randint(-50, 3000, (axes, T), generator=g, dtype=torch.int32)
    axis = [j % axes for j in range(P)]
    rope = pp.pp_rope_create(D, axis, freqs(P), axes, inter)
    try:
        qo, ko = torch.full((T, Hq, D), math.nan, device="cuda", dtype=dt), torch.full((T, Hk, D), math.nan, device="cuda", dtype=dt)
        pp.pp_qk_rotate(rope, pos.cuda(), 1e-6, q.cuda(), qw.cuda(), qo, k.cuda() if Hk else None,
                        kw.cuda() if Hk else None, ko if Hk else None, torch.cuda.current_stream())
        for got, x, w in ((qo, q, qw), (ko, k, kw)):
            want, tol = ref.rotate(x, w, 1e-6, pos, axis, freqs(P), inter)
            assert ref.worst(got, want, tol) <= 1
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)


def test_rotate_large_positions_keep_their_angle(pp):
    """2^31 - 1 and its neighbours: the turn's fraction stays exact where position * frequency in fp32 has no digits left."""
    D, P = 64, 32
    freq = [2 * math.pi * (j + 1) / 64 for j in range(P)]  # whole 64ths of a turn: the exact angle is known
    pos = torch.tensor([[2 ** 31 - 1, 2 ** 31 - 2, -2 ** 31, 123456789]], dtype=torch.int32)
    q = torch.ones((4, 1, D))
    rope = pp.pp_rope_create(D, None, freq)
    try:
        out = torch.empty((4, 1, D), device="cuda")
        pp.pp_qk_rotate(rope, pos.cuda(), -1.0, q.cuda(), None, out, None, None, None)
        for t in range(4):
            for j in range(P):
                a = 2 * math.pi * (int(pos[0, t]) * (j + 1) % 64) / 64
                # freq itself, rounded to 53 bits, moves the angle by up to 2^31 * 2^-53 * 2 pi; fp32 sines by 2^-23
                assert abs(float(out[t, 0, j]) - (math.cos(a) - math.sin(a))) < 4e-6
                assert abs(float(out[t, 0, P + j]) - (math.cos(a) + math.sin(a))) < 4e-6
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("how", ["fused", "odd_offset", "heads_first", "in_place", "no_norm", "no_weight", "zero_row", "broadcast"])
def test_rotate_views_and_options(pp, dt, how):
    T, Hq, Hk, D, P = 6, 4, 2, 64, 32
    g = torch.Generator().manual_seed(3)
    w = torch.rand(D, generator=g) + 0.5
    pos = torch.arange(T, dtype=torch.int32)[None].contiguous()
    eps = -1.0 if how == "no_norm" else 1e-6
    wq = None if how in ("no_norm", "no_weight") else w
    base = torch.randn((T, (Hq + Hk) * D + 3), generator=g).to(dt).cuda()
    if how == "zero_row":
        base[2] = 0
    off = 1 if how == "odd_offset" else 0
    q, k = base[:, off: off + Hq * D].unflatten(1, (Hq, D)), base[:, off + Hq * D: off + (Hq + Hk) * D].unflatten(1, (Hk, D))
    if how == "heads_first":
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
    if how == "in_place":
        q = q.contiguous()
    if how == "broadcast":  # one head for all: a head stride of 0
        k = k[:, :1].expand(T, Hk, D)
    hq, hk = q.cpu().clone(), k.cpu().clone()
    rope = pp.pp_rope_create(D, None, freqs(P))
    try:
        qo = q if how == "in_place" else torch.empty((T, Hq, D), device="cuda", dtype=dt)
        ko = torch.empty((T, Hk, D), device="cuda", dtype=dt)
        wd = None if wq is None else wq.cuda()
        pp.pp_qk_rotate(rope, pos.cuda(), eps, q, wd, qo, k, wd, ko)
        for got, x in ((qo, hq), (ko, hk)):
            want, tol = ref.rotate(x, wq, eps, pos, [0] * P, freqs(P), False)
            assert ref.worst(got, want, tol) <= 1
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)


def test_rotate_values_not_turned_keep_infinities_apart(pp):
    """A value beyond the pairs meets no other: an infinity there reaches nothing else when nothing is normalised."""
    D, P = 32, 8
    x = torch.ones((1, 1, D))
    x[0, 0, 20] = math.inf
    rope = pp.pp_rope_create(D, None, freqs(P))
    try:
        out = torch.empty((1, 1, D), device="cuda")
        pp.pp_qk_rotate(rope, torch.ones((1, 1), dtype=torch.int32).cuda(), -1.0, x.cuda(), None, out, None, None, None)
        got = out.cpu()[0, 0]
        assert got[20] == math.inf and torch.isfinite(got[torch.arange(D) != 20]).all() and (got[16:20] == 1).all()
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)


@pytest.mark.parametrize("dt,T,Hq,H,D,page", [(BF16, 1, 8, 8, 64, 16), (F16, 37, 6, 2, 128, 8), (F32, 100, 4, 4, 96, 32), (BF16, 300, 0, 1, 80, 64)])
def test_store(pp, dt, T, Hq, H, D, page):
    g = torch.Generator().manual_seed(T)
    P = D // 2
    fused = torch.randn((T, (Hq + 2 * H) * D), generator=g).to(dt)
    q, k, v = fused[:, : Hq * D].unflatten(1, (Hq, D)), fused[:, Hq * D: (Hq + H) * D].unflatten(1, (H, D)), fused[:, (Hq + H) * D:].unflatten(1, (H, D))
    kw = torch.rand(D, generator=g)
    pages = -(-T // page) + 3
    slots = torch.randperm(pages * page, generator=g)[:T].to(torch.int32)
    slots[T // 2] = -1  # this one is not kept
    pos = torch.randint(0, 500, (1, T), generator=g, dtype=torch.int32)
    kp, vp = torch.randn((pages, H, page, D), generator=g).to(dt), torch.randn((pages, H, page, D), generator=g).to(dt)
    kd, vd, fd = kp.cuda(), vp.cuda(), fused.cuda()
    rope, cache = pp.pp_rope_create(D, None, freqs(P)), pp.pp_cache_create(kd, vd)
    try:
        qo = torch.empty((T, Hq, D), device="cuda", dtype=dt)
        qv = fd[:, : Hq * D].unflatten(1, (Hq, D)) if Hq else None
        pp.pp_qkv_store(rope, cache, pos.cuda(), slots.cuda(), 1e-5, qv, None, qo if Hq else None,
                        fd[:, Hq * D: (Hq + H) * D].unflatten(1, (H, D)), kw.cuda(), fd[:, (Hq + H) * D:].unflatten(1, (H, D)))
        want, tol = ref.rotate(k, kw, 1e-5, pos, [0] * P, freqs(P), False)
        ek, et, ev = kp.double(), torch.zeros_like(kp, dtype=torch.float64), vp.clone()
        for t, s in enumerate(slots.tolist()):
            if s >= 0:
                ek[s // page, :, s % page], et[s // page, :, s % page], ev[s // page, :, s % page] = want[t], tol[t], v[t]
        assert ref.worst(kd, ek, et) <= 1  # untouched cells have no tolerance: bit for bit
        assert torch.equal(vd.cpu(), ev)
        if Hq:
            wq, tq = ref.rotate(q, None, 1e-5, pos, [0] * P, freqs(P), False)
            assert ref.worst(qo, wq, tq) <= 1
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        pp.pp_rope_destroy(rope)
        pp.pp_cache_destroy(cache)


# ------------------------------------------------------------------ caches

class Case:
    """A cache with sequences in it: shuffled pages; what no token sees is NaN, and tables end in ids of no page."""

    def __init__(self, pp, dt, G, H, D, page, lens, tokens=None, seed=0, extra=2, summaries=False, trash=True):
        g = torch.Generator().manual_seed(seed)
        self.pp, self.dt, self.page, self.lens = pp, dt, page, lens
        need = [-(-n // page) for n in lens]
        pages, W = sum(need) + extra, max(max(need), 1) + 1
        order = torch.randperm(pages, generator=g)
        self.table = torch.full((len(lens), W), 2 ** 31 - 1, dtype=torch.int32)
        self.k = torch.randn((pages, H, page, D), generator=g).mul(1.5).to(dt)
        self.v = torch.randn((pages, H, page, D), generator=g).to(dt)
        at = 0
        live = torch.zeros((pages, page), dtype=torch.bool)
        for b, n in enumerate(lens):
            ids = order[at: at + need[b]]
            at += need[b]
            self.table[b, : need[b]] = ids.to(torch.int32)
            for w, i in enumerate(ids.tolist()):
                live[i, : min(page, n - w * page)] = True
        if trash:
            dead = ~live[:, None, :, None].expand_as(self.k)
            self.k[dead] = math.nan
            self.v[dead] = math.inf
        self.starts = None
        T = len(lens)
        if tokens is not None:
            self.starts = [0]
            for n in tokens:
                self.starts.append(self.starts[-1] + n)
            T = self.starts[-1]
        self.T = T
        self.q = torch.randn((T, H * G, D), generator=g).to(dt)
        self.kd, self.vd, self.qd, self.td = self.k.cuda(), self.v.cuda(), self.q.cuda(), self.table.cuda()
        self.ld = torch.tensor(lens, dtype=torch.int32).cuda()
        self.sd = None if self.starts is None else torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.codes = self.scales = None
        if summaries:
            self.codes = torch.zeros((pages, H, 2, D), dtype=torch.int8, device="cuda")
            self.scales = torch.zeros((pages, H), device="cuda")
        self.cache = pp.pp_cache_create(self.kd, self.vd, self.codes, self.scales)

    def attend(self, scale=None, causal=True, sel=None, q=None, stream=None, lse=True):
        q = self.qd if q is None else q
        scale = 1 / math.sqrt(q.shape[2]) if scale is None else scale
        out = torch.full(self.q.shape, math.nan, device="cuda", dtype=self.dt)
        ls = torch.full(self.q.shape[:2], math.nan, device="cuda") if lse else None
        self.pp.pp_attn_forward(self.cache, q, self.sd, self.td, self.ld, scale, self.pp.PP_ATTN_CAUSAL if causal else 0,
                                sel, out, ls, stream)
        return out, ls

    def check(self, scale=None, causal=True, sel=None, q=None):
        s = 1 / math.sqrt(self.q.shape[2]) if scale is None else scale
        out, lse = self.attend(s, causal, None if sel is None else sel.cuda(), q)
        want, wl, tol, tl = ref.attend(self.q, self.k, self.v, self.table, self.starts, self.lens, s, causal, sel)
        assert ref.worst(out, want, tol) <= 1
        assert ref.worst(lse, wl, tl) <= 1
        return out

    def status(self):
        return self.pp.pp_cache_device_status(self.cache)

    def close(self):
        torch.cuda.synchronize()
        self.pp.pp_cache_destroy(self.cache)


ATTEND = [
    # dtype, G, H, D, page, lens, tokens per sequence (None: one each)
    (BF16, 4, 2, 128, 16, [1], None),
    (BF16, 4, 2, 64, 16, [777], None),
    (BF16, 1, 3, 64, 8, [0, 1, 7, 8, 9, 63, 64, 65], None),
    (F16, 8, 1, 128, 32, [130, 0, 511], None),
    (F32, 2, 2, 96, 16, [33, 300], None),
    (F32, 4, 1, 64, 64, [65, 1], None),
    (F16, 3, 2, 80, 64, [100, 129], None),
    (BF16, 1, 1, 256, 128, [300], None),
    (F32, 5, 1, 256, 16, [50], None),
    (BF16, 16, 1, 128, 64, [200], None),
    (F16, 20, 1, 64, 64, [200, 5], None),      # more rows than one tile of 16
    (BF16, 40, 1, 16, 256, [257], None),
    (F16, 2, 1, 24, 16, [40], None),           # a head of 24
    (F32, 1, 1, 200, 32, [70], None),
    (BF16, 2, 2, 64, 16, [5, 40, 0], [5, 3, 0]),   # a whole prompt, a chunk, an idle sequence
    (F16, 4, 2, 128, 32, [70, 33, 200], [33, 1, 130]),
    (F32, 2, 1, 64, 16, [90], [50]),
    (BF16, 8, 1, 128, 64, [300], [300]),
    (F16, 1, 2, 64, 64, [257, 64], [200, 64]),
    (BF16, 3, 1, 96, 128, [400], [77]),
    (BF16, 4, 1, 256, 64, [200], [90]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dt,G,H,D,page,lens,tokens", ATTEND)
def test_attend(pp, dt, G, H, D, page, lens, tokens, causal):
    c = Case(pp, dt, G, H, D, page, lens, tokens, seed=D + len(lens))
    try:
        c.check(causal=causal)
        assert c.status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("tokens", [None, [50, 3]])
def test_attend_large_and_negative_scale(pp, dt, tokens):
    """Logits of hundreds (one key takes all), and the other sign."""
    for scale in (20.0, -0.5, 0.0):
        c = Case(pp, dt, 2, 1, 64, 16, [100, 60], tokens, seed=5)
        try:
            c.check(scale=scale)
        finally:
            c.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("tokens", [None, [40]])
def test_attend_selected(pp, dt, tokens):
    """Any order, entries below 0 between, tokens without a page, pages beyond what a token sees."""
    c = Case(pp, dt, 4, 2, 64, 16, [333], tokens, seed=9)
    try:
        g = torch.Generator().manual_seed(1)
        keep, P = 6, -(-333 // 16)
        sel = torch.stack([torch.randperm(P, generator=g)[:keep] for _ in range(c.T * 2)]).view(c.T, 2, keep).to(torch.int32)
        sel[:, 0, 2] = -1
        sel[0, 1] = -1
        c.check(sel=sel)
        assert c.status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("tokens", [None, [70, 30]])
def test_attend_views(pp, tokens):
    """Queries as a part of a fused product, at an odd offset, heads first."""
    c = Case(pp, BF16, 4, 2, 64, 16, [150, 90], tokens, seed=2)
    try:
        T, Hq, D = c.q.shape
        base = torch.randn((T, (Hq + 4) * D + 5), device="cuda").to(BF16)
        for off in (0, 1):
            view = base[:, off: off + Hq * D].unflatten(1, (Hq, D))
            view.copy_(c.qd)
            c.check(q=view)
        c.check(q=c.qd.transpose(0, 1).contiguous().transpose(0, 1))
    finally:
        c.close()


@pytest.mark.parametrize("tokens", [None, [20, 10]])
def test_bad_entries_are_skipped_and_recorded(pp, tokens):
    c = Case(pp, F16, 2, 1, 64, 16, [100, 40], tokens, seed=4)
    try:
        for bad in (-1, c.k.shape[0], 2 ** 30):
            c.table[0, 2] = bad
            c.td.copy_(c.table)
            c.check()
            assert c.status() == pp.PP_CACHE_BAD_PAGE
            assert c.status() == 0
        # a length beyond the table, and a negative one: as the table's end, and none
        c.table[0, 2] = c.table[0, 3]
        c.table[:] = c.table.clamp(max=c.k.shape[0] - 1)
        c.td.copy_(c.table)
        c.kd.nan_to_num_(0, 0, 0)
        c.vd.nan_to_num_(0, 0, 0)
        c.k, c.v = c.kd.cpu(), c.vd.cpu()
        c.ld.copy_(torch.tensor([10 ** 9, -5]))
        c.lens = [c.table.shape[1] * 16, 0]
        c.check()
        assert c.status() == pp.PP_CACHE_BAD_LENGTH
    finally:
        c.close()


def test_bad_slots_are_skipped_and_recorded(pp):
    k = torch.zeros((2, 1, 16, 64), device="cuda")
    v = torch.zeros_like(k)
    rope, cache = pp.pp_rope_create(64, None, freqs(32)), pp.pp_cache_create(k, v)
    try:
        x = torch.ones((3, 1, 64), device="cuda")
        pos = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
        pp.pp_qkv_store(rope, cache, pos, torch.tensor([32, -2, 31], dtype=torch.int32, device="cuda"), -1.0, None, None, None, x, None, x)
        assert pp.pp_cache_device_status(cache) == pp.PP_CACHE_BAD_SLOT
        assert float(v.sum()) == 64 and bool((v[1, 0, 15] == 1).all())
    finally:
        pp.pp_rope_destroy(rope)
        pp.pp_cache_destroy(cache)


@pytest.mark.parametrize("dt,G,D,page,lens,tokens", [(BF16, 4, 128, 64, [20000], None), (F16, 4, 128, 64, [5000, 9000, 1], None),
                                                     (BF16, 2, 64, 16, [1500], [600]), (F32, 1, 64, 32, [4000, 50], None)])
def test_same_inputs_same_bits(pp, dt, G, D, page, lens, tokens):
    c = Case(pp, dt, G, 2, D, page, lens, tokens, seed=6)
    try:
        first, l1 = c.attend()
        for _ in range(4):
            again, l2 = c.attend()
            assert torch.equal(first, again) and torch.equal(l1, l2)
        c.check()
    finally:
        c.close()


def test_on_another_stream(pp):
    """Everything of a step on a side stream, in its order, without the default stream."""
    c = Case(pp, BF16, 4, 2, 64, 16, [500, 31], seed=8)
    try:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            out, _ = c.attend(stream=s)
        s.synchronize()
        want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, None, c.lens, 1 / 8.0, True)
        assert ref.worst(out, want, tol) <= 1
    finally:
        c.close()


def test_in_a_cuda_graph(pp):
    """Captured once, replayed with other lengths: what is split and how is decided on the device."""
    c = Case(pp, BF16, 4, 2, 64, 16, [900, 40], seed=8, trash=False)
    try:
        out = torch.empty(c.q.shape, device="cuda", dtype=BF16)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        args = (c.qd, None, c.td, c.ld, 0.125, pp.PP_ATTN_CAUSAL, None, out, None)
        with torch.cuda.stream(s):
            pp.pp_attn_forward(c.cache, *args, s)
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                pp.pp_attn_forward(c.cache, *args, s)
        for lens in ([900, 40], [3, 0], [512, 33]):
            c.ld.copy_(torch.tensor(lens))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, None, lens, 0.125, True)
            assert ref.worst(out, want, tol) <= 1
    finally:
        c.close()


def test_offsets_beyond_32_bits(pp):
    """Pools of 2.2 billion values each: pages at their far end."""
    H, page, D = 2, 64, 128
    pages = 2_200_000_000 // (H * page * D)
    k = torch.zeros((pages, H, page, D), device="cuda", dtype=F16)
    v = torch.zeros((pages, H, page, D), device="cuda", dtype=F16)
    codes = torch.zeros((pages, H, 2, D), dtype=torch.int8, device="cuda")
    scales = torch.zeros((pages, H), device="cuda")
    cache = pp.pp_cache_create(k, v, codes, scales)
    rope = pp.pp_rope_create(D, None, freqs(D // 2))
    try:
        g = torch.Generator().manual_seed(0)
        ids = [pages - 1, 3, pages - 2]
        T = 150
        x = torch.randn((T, H, D), generator=g).to(F16)
        u = torch.randn((T, H, D), generator=g).to(F16)
        pos = torch.zeros((1, T), dtype=torch.int32)
        slots = torch.tensor([ids[t // page] * page + t % page for t in range(T)], dtype=torch.int32)
        pp.pp_qkv_store(rope, cache, pos.cuda(), slots.cuda(), -1.0, None, None, None, x.cuda(), None, u.cuda())
        small = [torch.zeros((3, H, page, D), dtype=F16) for _ in range(2)]
        for t in range(T):
            small[0][t // page, :, t % page], small[1][t // page, :, t % page] = x[t], u[t]
        assert torch.equal(k[ids].cpu(), small[0]) and torch.equal(v[ids].cpu(), small[1])
        q = torch.randn((1, 2 * H, D), generator=g).to(F16)
        out = torch.empty_like(q, device="cuda")
        pp.pp_attn_forward(cache, q.cuda(), None, torch.tensor([ids], dtype=torch.int32, device="cuda"),
                           torch.tensor([T], dtype=torch.int32, device="cuda"), 0.1, pp.PP_ATTN_CAUSAL, None, out)
        want, _, tol, _ = ref.attend(q, *small, torch.tensor([[0, 1, 2]]), None, [T], 0.1, True)
        assert ref.worst(out, want, tol) <= 1
        pp.pp_cache_summarize(cache, torch.tensor(ids[:1], dtype=torch.int32, device="cuda"))
        wc, ws = ref.summarize(small[0][:1])
        assert torch.equal(codes[ids[:1]].cpu(), wc) and torch.equal(scales[ids[:1]].cpu(), ws)
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        pp.pp_rope_destroy(rope)
        pp.pp_cache_destroy(cache)


# ------------------------------------------------------------------ summaries and selections


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("H,D,page", [(1, 16, 8), (3, 64, 16), (2, 128, 64), (2, 80, 32), (1, 256, 256), (1, 200, 128)])
def test_summaries(pp, dt, H, D, page):
    g = torch.Generator().manual_seed(D)
    pages = 9
    k = torch.randn((pages, H, page, D), generator=g).to(dt)
    k[1] = 0
    k[2] = -k[2].abs()
    k[3, 0, 2, 1] = math.nan
    k[4, 0, 3, 0] = -math.inf
    k[5] = k[5] * (2.0 ** -120 if dt != F16 else 2.0 ** -14)
    k[6] = 1.0
    kd = k.cuda()
    codes = torch.full((pages, H, 2, D), 55, dtype=torch.int8, device="cuda")
    scales = torch.full((pages, H), 55.0, device="cuda")
    cache = pp.pp_cache_create(kd, kd.clone(), codes, scales)
    try:
        ids = torch.tensor([6, 0, 5, 3, 1, 4, 2], dtype=torch.int32)
        pp.pp_cache_summarize(cache, ids.cuda())
        wc, ws = ref.summarize(k)
        wc[7:], ws[7:] = 55, 55.0
        assert torch.equal(codes.cpu(), wc)
        assert torch.equal(torch.nan_to_num(scales.cpu(), nan=-1), torch.nan_to_num(ws, nan=-1))
        assert pp.pp_cache_device_status(cache) == 0
        pp.pp_cache_summarize(cache, torch.tensor([-1, pages], dtype=torch.int32).cuda())
        assert pp.pp_cache_device_status(cache) == pp.PP_CACHE_BAD_PAGE
        assert torch.equal(codes.cpu(), wc)
        pp.pp_cache_summarize(cache, ids[:0].cuda())
    finally:
        pp.pp_cache_destroy(cache)


SELECT = [
    # dtype, G, H, D, page, lens, tokens, first, last, keep
    (BF16, 4, 2, 128, 16, [777], None, 1, 2, 8),
    (F16, 1, 1, 64, 16, [0, 1, 16, 17, 500, 129], None, 0, 1, 4),
    (F32, 2, 3, 96, 8, [400, 333], None, 2, 2, 5),
    (BF16, 8, 1, 256, 8, [600], None, 1, 1, 33),
    (F16, 16, 1, 128, 8, [300], None, 0, 1, 1),
    (BF16, 4, 2, 64, 16, [300, 40], [41, 13], 1, 2, 6),
    (F32, 1, 1, 80, 32, [700], [9], 0, 2, 7),
    (F16, 3, 1, 64, 8, [4500], None, 1, 2, 64),
    (BF16, 2, 2, 64, 8, [2100, 17], [130, 17], 1, 2, 40),
    (BF16, 1, 1, 16, 8, [1300], None, 0, 1, 160),   # nearly everything
]


@pytest.mark.parametrize("dt,G,H,D,page,lens,tokens,first,last,keep", SELECT)
def test_select(pp, dt, G, H, D, page, lens, tokens, first, last, keep):
    c = Case(pp, dt, G, H, D, page, lens, tokens, seed=D + keep, summaries=True)
    try:
        codes, scales = ref.summarize(torch.nan_to_num(c.k, 0, 0, 0))
        c.codes.copy_(codes)
        c.scales.copy_(scales)
        sel = torch.full((c.T, H, keep), 77, dtype=torch.int32, device="cuda")
        pp.pp_cache_select(c.cache, c.qd, c.sd, c.td, c.ld, pp.PP_ATTN_CAUSAL, first, last, sel)
        want = ref.select(c.q, codes, scales, c.table, c.starts, lens, True, page, first, last, keep)
        assert torch.equal(sel.cpu(), want)
        assert c.status() == 0
        pp.pp_cache_select(c.cache, c.qd, c.sd, c.td, c.ld, 0, first, last, sel)
        assert torch.equal(sel.cpu(), ref.select(c.q, codes, scales, c.table, c.starts, lens, False, page, first, last, keep))
    finally:
        c.close()


@pytest.mark.parametrize("what", ["ties", "nan_scale", "nan_query", "zero_query", "bad_page", "negative", "infinite_scale"])
def test_select_orders(pp, what):
    """Equal scores go to the lower page; NaN ranks lowest; queries that say nothing tie everything."""
    H, G, D, page, n, keep = 1, 2, 64, 8, 400, 9
    c = Case(pp, F32, G, H, D, page, [n], None, seed=1, summaries=True, trash=False)
    try:
        codes, scales = ref.summarize(c.k)
        if what == "ties":
            codes[:] = codes[:1]
            scales[:] = 1.0
            scales[int(c.table[0, 30])] = 2.0
        elif what == "nan_scale":
            scales[c.table[0, 3:44].long()] = math.nan
        elif what == "nan_query":
            c.q[0, 1, 5] = math.nan
        elif what == "zero_query":
            c.q[:] = 0
        elif what == "bad_page":
            c.table[0, 10] = -3
            c.td.copy_(c.table)
        elif what == "negative":
            codes[:, :, 0] = -100  # every score far below zero
        elif what == "infinite_scale":
            scales[int(c.table[0, 20])] = math.inf
        c.codes.copy_(codes)
        c.scales.copy_(scales)
        c.qd.copy_(c.q)
        sel = torch.empty((1, H, keep), dtype=torch.int32, device="cuda")
        pp.pp_cache_select(c.cache, c.qd, None, c.td, c.ld, pp.PP_ATTN_CAUSAL, 1, 2, sel)
        assert torch.equal(sel.cpu(), ref.select(c.q, codes, scales, c.table, None, [n], True, page, 1, 2, keep))
        assert c.status() == (pp.PP_CACHE_BAD_PAGE if what == "bad_page" else 0)
    finally:
        c.close()


def test_select_then_attend(pp):
    """The step as a program runs it, on a prompt's chunk: summaries, selection, attention over the selected pages."""
    c = Case(pp, BF16, 4, 2, 64, 16, [600, 90], [130, 90], seed=11, summaries=True)
    try:
        full = [int(c.table[b, w]) for b, n in enumerate(c.lens) for w in range(n // 16)]
        pp.pp_cache_summarize(c.cache, torch.tensor(full, dtype=torch.int32).cuda())
        sel = torch.empty((c.T, 2, 7), dtype=torch.int32, device="cuda")
        pp.pp_cache_select(c.cache, c.qd, c.sd, c.td, c.ld, pp.PP_ATTN_CAUSAL, 1, 2, sel)
        c.check(sel=sel.cpu())
        assert c.status() == 0
    finally:
        c.close()


# ------------------------------------------------------------------ refusals that need a handle


def test_refusals(pp):
    k = torch.zeros((4, 2, 16, 64), device="cuda", dtype=BF16)
    bare, full = pp.pp_cache_create(k, k.clone()), pp.pp_cache_create(
        k, k.clone(), torch.zeros((4, 2, 2, 64), dtype=torch.int8, device="cuda"), torch.zeros((4, 2), device="cuda"))
    rope, other = pp.pp_rope_create(64, None, freqs(32)), pp.pp_rope_create(32, None, freqs(16))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q, out = torch.zeros((1, 4, 64), device="cuda", dtype=BF16), torch.empty((1, 4, 64), device="cuda", dtype=BF16)
    table, lens, sel = i32([0, 1]), i32(20), torch.zeros((1, 2, 2), dtype=torch.int32, device="cuda")
    pos = i32([0])

    def refused(code, f, *a):
        with pytest.raises(pp.PPError) as e:
            f(*a)
        assert e.value.code == code

    try:
        bad = pp.PP_ERR_INVALID_ARG
        q3 = torch.zeros((1, 3, 64), device="cuda", dtype=BF16)
        refused(bad, pp.pp_attn_forward, bare, q3, None, table, lens, 1.0, 0, None, torch.empty_like(q3))
        refused(bad, pp.pp_attn_forward, bare, q.to(F16), None, table, lens, 1.0, 0, None, out)
        refused(bad, pp.pp_attn_forward, bare, q, None, table, lens, math.nan, 0, None, out)
        refused(bad, pp.pp_attn_forward, bare, q, None, table, lens, 1.0, 8, None, out)
        refused(bad, pp.pp_attn_forward, bare, q, None, i32([0], [1]), i32(1, 1), 1.0, 0, None, out)  # T is not B
        refused(bad, pp.pp_attn_forward, bare, q, None, table.long(), lens, 1.0, 0, None, out)
        refused(bad, pp.pp_attn_forward, bare, q, None, table, lens, 1.0, 0, sel.long(), out)
        refused(bad, pp.pp_attn_forward, bare, q, None, table, lens, 1.0, 0, None, out[:, :2])
        refused(bad, pp.pp_cache_select, bare, q, None, table, lens, 0, 0, 1, sel)  # no summaries
        refused(bad, pp.pp_cache_select, full, q, None, table, lens, 0, 0, 0, sel)
        refused(bad, pp.pp_cache_select, full, q, None, table, lens, 0, -1, 1, sel)
        refused(bad, pp.pp_cache_select, full, q, None, table, lens, 0, 2, 1, sel)
        refused(pp.PP_ERR_UNSUPPORTED, pp.pp_cache_select, full, q, None, torch.zeros((1, 32769), dtype=torch.int32, device="cuda"), lens, 0, 0, 1, sel)
        refused(bad, pp.pp_cache_summarize, bare, i32(0))
        refused(bad, pp.pp_qkv_store, other, bare, pos, i32(0), 0.0, None, None, None, q[:, :2, :32], None, q[:, :2, :32])
        refused(bad, pp.pp_qkv_store, rope, bare, pos, i32(0), 0.0, None, None, None, q, None, q)  # four heads, the cache has two
        refused(bad, pp.pp_qkv_store, rope, bare, pos, i32(0), math.nan, None, None, None, q[:, :2], None, q[:, :2])
        refused(bad, pp.pp_qk_rotate, rope, pos, -1.0, q, torch.ones(64, device="cuda"), out, None, None, None)
        refused(bad, pp.pp_qk_rotate, rope, pos.long(), 0.0, q, None, out, None, None, None)
        refused(bad, pp.pp_qk_rotate, rope, pos, 0.0, q.double(), None, out, None, None, None)
        refused(bad, pp.pp_cache_create, k, k.to(F16))
        refused(bad, pp.pp_cache_create, k, k, torch.zeros((4, 2, 2, 64), dtype=torch.int8, device="cuda"), None)
        refused(pp.PP_ERR_UNSUPPORTED, pp.pp_cache_create, *[torch.zeros((1, 1, 24, 64), device="cuda")] * 2)
        refused(pp.PP_ERR_UNSUPPORTED, pp.pp_cache_create, *[torch.zeros((1, 1, 16, 60), device="cuda")] * 2)
        # nothing to do is no error
        none = torch.empty((0, 4, 64), device="cuda", dtype=BF16)
        pp.pp_attn_forward(bare, none, None, torch.zeros((0, 2), dtype=torch.int32, device="cuda"), i32(), 1.0, 0, None, none)
        pp.pp_qk_rotate(rope, torch.zeros((1, 0), dtype=torch.int32, device="cuda"), 0.0, none, None, none, None, None, None)
        assert pp.pp_cache_device_status(bare) == 0
    finally:
        for c in (bare, full):
            pp.pp_cache_destroy(c)
        for r in (rope, other):
            pp.pp_rope_destroy(r)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("where", ["value", "key"])
def test_what_a_later_token_sees_reaches_no_earlier_one(pp, dt, where):
    """NaN and infinity at a key of the chunk's own tokens: those before it stay as they were, bit for bit finite."""
    c = Case(pp, dt, 2, 1, 64, 16, [90], [40], seed=12)
    try:
        pool = c.v if where == "value" else c.k
        for key, bad in ((70, math.nan), (81, math.inf)):
            pool[int(c.table[0, key // 16]), 0, key % 16, 5] = bad
        c.kd.copy_(c.k)
        c.vd.copy_(c.v)
        out, lse = c.attend()
        want, wl, tol, tl = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.lens, 1 / 8.0, True)
        clean = 70 - 50  # tokens 50 .. 89 are the chunk; the first 20 see neither
        assert ref.worst(out[:clean], want[:clean], tol[:clean]) <= 1
        assert ref.worst(lse[:clean], wl[:clean], tl[:clean]) <= 1
        got = out[clean:].double().cpu()
        assert torch.equal(torch.isfinite(got), torch.isfinite(want[clean:]))
    finally:
        c.close()


def test_many_parts_of_one_unit(pp):
    """One long sequence with one cache head: hundreds of parts, joined in two levels; and unequal neighbours."""
    for dt, lens in ((BF16, [120_000]), (F32, [60_000]), (F16, [90_000, 0, 3, 70_000])):
        c = Case(pp, dt, 4, 1, 64, 64, lens, seed=13)
        try:
            c.check()
            assert c.status() == 0
        finally:
            c.close()


# ------------------------------------------------------------------ many tokens: tiles of 128 rows

TILES = [
    # dtype, G, H, D, page, lens, tokens: enough rows that the tile kernel takes them
    (BF16, 8, 1, 128, 64, [400], [330]),
    (F16, 8, 1, 128, 64, [331, 0, 70], [331, 0, 5]),
    (BF16, 2, 2, 64, 16, [900], [700]),
    (F16, 3, 2, 80, 32, [520, 77], [500, 40]),     # 42 tokens to a tile, heads that end inside a column
    (BF16, 1, 2, 128, 128, [1350], [1300]),
    (F16, 1, 2, 64, 8, [1300, 20], [1300, 1]),
    (BF16, 64, 1, 16, 8, [90], [50]),
    (F16, 4, 4, 96, 256, [300], [170]),
    (BF16, 5, 1, 24, 64, [640], [600]),
]


def kernels_of(c, tmp_path, sel=None):
    """The names of the attention kernels that this call launches, from a captured graph's dump."""
    g = torch.cuda.CUDAGraph(keep_graph=True)
    g.enable_debug_mode()
    with torch.cuda.graph(g):
        c.attend(sel=sel, stream=torch.cuda.current_stream())
    dot = tmp_path / "graph.dot"
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        g.debug_dump(str(dot))
    names = re.findall(r"attn_\w*kernel", dot.read_text())
    assert names
    return names


def tile_kernel_runs(c, tmp_path, sel=None):
    return any("attn_tile_kernel" in n for n in kernels_of(c, tmp_path, sel))


@pytest.mark.parametrize("dt,G,H,D,page,lens,tokens", TILES)
def test_tiles(pp, tmp_path, dt, G, H, D, page, lens, tokens):
    c = Case(pp, dt, G, H, D, page, lens, tokens, seed=D + G)
    try:
        assert tile_kernel_runs(c, tmp_path)
        c.check()
        c.check(causal=False)
        c.check(scale=-0.3)
        c.check(scale=0.0)
        assert c.status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("dt,G,H,D,page,lens,tokens", TILES)
@pytest.mark.parametrize("keep", [1, 7])
def test_tiles_selected(pp, tmp_path, dt, G, H, D, page, lens, tokens, keep):
    """Neighbours that select different pages, tokens without any, entries of no page."""
    c = Case(pp, dt, G, H, D, page, lens, tokens, seed=D + G + keep)
    try:
        g = torch.Generator().manual_seed(2)
        sel = torch.full((c.T, H, keep), -1, dtype=torch.int32)
        for t, (b, n) in enumerate(ref.seen_keys(c.T, c.starts, lens, True)):
            P = -(-n // page)
            for h in range(H):
                some = torch.randperm(P, generator=g)[:keep]
                sel[t, h, : len(some)] = some.to(torch.int32)
        sel[3] = -1
        sel[5, 0, 0] = -7
        assert tile_kernel_runs(c, tmp_path, sel.cuda())
        c.check(sel=sel)
        assert c.status() == 0
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F16, BF16])
def test_tiles_large_logits(pp, dt):
    """Maxima that grow by hundreds from block to block, so that the sums are rescaled, and ones that never do."""
    c = Case(pp, dt, 4, 2, 64, 64, [700], [400], seed=21)
    try:
        for w in range(c.table.shape[1] - 1):  # later pages hold larger keys
            i = int(c.table[0, w])
            c.k[i] = (c.k[i].float() * (0.1 + 0.4 * w)).to(dt)
        c.kd.copy_(c.k)
        for scale in (0.125, 2.0, 20.0):
            c.check(scale=scale)
    finally:
        c.close()


@pytest.mark.parametrize("selected", [False, True])
@pytest.mark.parametrize("where", ["value", "key"])
def test_tiles_keep_tokens_apart(pp, where, selected):
    """NaN and infinity at a key that some of a tile's tokens see: the others stay as they were."""
    c = Case(pp, BF16, 4, 2, 64, 16, [500], [400], seed=12)
    try:
        pool = c.v if where == "value" else c.k
        for key, bad in ((170, math.nan), (230, math.inf)):
            pool[int(c.table[0, key // 16]), 0, key % 16, 5] = bad
        c.kd.copy_(c.k)
        c.vd.copy_(c.v)
        sel = None
        if selected:
            g = torch.Generator().manual_seed(4)
            sel = torch.stack([torch.randperm(100 // 16, generator=g)[:3] for _ in range(c.T * 2)]).view(c.T, 2, 3).to(torch.int32)
            sel[::3, :, 1] = 170 // 16
        out, lse = c.attend(sel=None if sel is None else sel.cuda())
        want, wl, tol, tl = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.lens, 1 / 8.0, True, sel)
        fine = torch.isfinite(want)
        got = out.double().cpu()
        assert torch.equal(torch.isfinite(got), fine)
        assert ref.worst(torch.where(fine, got, 0.0), torch.where(fine, want, 0.0), tol) <= 1
    finally:
        c.close()


def test_tiles_bad_pages(pp):
    c = Case(pp, F16, 4, 2, 64, 16, [500, 40], [300, 40], seed=4)
    try:
        for bad in (-1, c.k.shape[0], 2 ** 30):
            c.table[0, 2] = bad
            c.td.copy_(c.table)
            c.check()
            assert c.status() == pp.PP_CACHE_BAD_PAGE
        c.sd.copy_(torch.tensor([0, 400, 340]))  # token ranges that do not fit
        c.attend()
        assert c.status() & pp.PP_CACHE_BAD_LENGTH
    finally:
        c.close()


def test_tiles_over_windows_of_pages(pp, tmp_path):
    """More pages than the masks of one window hold."""
    c = Case(pp, BF16, 1, 2, 64, 8, [9000], [1300], seed=4)
    try:
        g = torch.Generator().manual_seed(2)
        sel = torch.stack([torch.randperm(7700 // 8, generator=g)[:5] for _ in range(c.T * 2)]).view(c.T, 2, 5).to(torch.int32)
        assert tile_kernel_runs(c, tmp_path, sel.cuda())
        c.check(sel=sel)
    finally:
        c.close()


def test_tiles_same_bits(pp):
    c = Case(pp, BF16, 4, 2, 128, 64, [3000, 500], [500, 100], seed=6)
    try:
        first, l1 = c.attend()
        for _ in range(4):
            again, l2 = c.attend()
            assert torch.equal(first, again) and torch.equal(l1, l2)
        c.check()
    finally:
        c.close()


@pytest.mark.parametrize("dt,G,H,D,page,lens,tokens", [(BF16, 4, 2, 128, 64, [7000], [300]), (F16, 8, 1, 64, 16, [3000, 500, 40], [300, 1, 40]),
                                                      (BF16, 3, 2, 80, 128, [9000, 2500], [150, 200])])
def test_tiles_split(pp, tmp_path, dt, G, H, D, page, lens, tokens):
    """Few tiles over many blocks: shares of them in CTAs of their own, joined; a selection; values that are not finite."""
    c = Case(pp, dt, G, H, D, page, lens, tokens, seed=D + G)
    try:
        assert any("join" in n for n in kernels_of(c, tmp_path))
        c.check()
        c.check(causal=False, scale=-0.3)
        g = torch.Generator().manual_seed(2)
        keep = 2048 // page
        sel = torch.full((c.T, H, keep), -1, dtype=torch.int32)
        for t, (b, n) in enumerate(ref.seen_keys(c.T, c.starts, lens, True)):
            some = torch.randperm(-(-n // page), generator=g)[:keep]
            sel[t, :, : len(some)] = some.to(torch.int32)
        c.check(sel=sel)
        again, _ = c.attend(sel=sel.cuda())
        assert torch.equal(again, c.attend(sel=sel.cuda())[0])
        key = lens[0] - tokens[0] // 2
        c.v[int(c.table[0, key // page]), 0, key % page, 5] = math.nan
        c.k[int(c.table[0, key // page]), 0, key % page, 3] = math.inf
        c.kd.copy_(c.k)
        c.vd.copy_(c.v)
        for scale in (0.125, -0.125):
            out, _ = c.attend(scale=scale)
            want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, lens, scale, True)
            fine, got = torch.isfinite(want), out.double().cpu()
            assert torch.equal(torch.isfinite(got), fine)
            assert ref.worst(torch.where(fine, got, 0.0), torch.where(fine, want, 0.0), tol) <= 1
        assert c.status() == 0
    finally:
        c.close()


def test_not_finite_at_a_negative_scale(pp):
    """Rows computed again for a value that others see: with the sign of the scale."""
    for tokens in ([400], [40]):
        c = Case(pp, BF16, 4, 2, 64, 16, [500], tokens, seed=12)
        try:
            c.v[int(c.table[0, 480 // 16]), 0, 480 % 16, 5] = math.nan
            c.vd.copy_(c.v)
            for scale in (-0.2, 0.0):
                out, _ = c.attend(scale=scale)
                want, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.lens, scale, True)
                fine, got = torch.isfinite(want), out.double().cpu()
                assert torch.equal(torch.isfinite(got), fine)
                assert ref.worst(torch.where(fine, got, 0.0), torch.where(fine, want, 0.0), tol) <= 1
        finally:
            c.close()


@pytest.mark.parametrize("tokens", [None, [40]])
@pytest.mark.parametrize("G,D", [(8, 128), (16, 64), (3, 256)])
def test_select_sums_near_their_largest(pp, G, D, tokens):
    """Integers of 23 and 24 bits whose last one decides: every code and every query near its largest."""
    page, n, keep = 8, 900, 12
    c = Case(pp, F32, G, 1, D, page, [n], tokens, seed=3, summaries=True, trash=False)
    try:
        g = torch.Generator().manual_seed(7)
        pages = c.k.shape[0]
        codes = torch.randint(125, 128, (pages, 1, 2, D), generator=g).to(torch.int8)
        codes[:, :, 1] = torch.randint(-127, -120, (pages, 1, D), generator=g).to(torch.int8)
        scales = torch.ones((pages, 1))
        c.q = 1.0 - 0.02 * torch.rand(c.q.shape, generator=g)
        c.q[:, 0, 0] = 1.0
        c.codes.copy_(codes)
        c.scales.copy_(scales)
        c.qd.copy_(c.q)
        sel = torch.empty((c.T, 1, keep), dtype=torch.int32, device="cuda")
        pp.pp_cache_select(c.cache, c.qd, c.sd, c.td, c.ld, pp.PP_ATTN_CAUSAL, 1, 2, sel)
        assert torch.equal(sel.cpu(), ref.select(c.q, codes, scales, c.table, c.starts, [n], True, page, 1, 2, keep))
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("tokens", [None, [30, 10]])
def test_select_views(pp, dt, tokens):
    """Queries in a fused product: on 32-byte boundaries, on 16-byte ones, on those of one value, heads first."""
    page, D, G, H, keep = 8, 64, 2, 2, 6
    c = Case(pp, dt, G, H, D, page, [300, 200], tokens, seed=5, summaries=True, trash=False)
    try:
        codes, scales = ref.summarize(c.k)
        c.codes.copy_(codes)
        c.scales.copy_(scales)
        want = ref.select(c.q, codes, scales, c.table, c.starts, c.lens, True, page, 1, 2, keep)
        step = 16 // c.q.element_size()
        base = torch.randn((c.T, (H * G + 2) * D + 2 * step), device="cuda").to(dt)
        views = [c.qd.transpose(0, 1).contiguous().transpose(0, 1)]
        for off in (0, step, 1):
            views.append(base[:, off: off + H * G * D].unflatten(1, (H * G, D)))
            views[-1].copy_(c.qd)
            sel = torch.empty((c.T, H, keep), dtype=torch.int32, device="cuda")
            for q in views[-1:] + views[:1]:
                pp.pp_cache_select(c.cache, q, c.sd, c.td, c.ld, pp.PP_ATTN_CAUSAL, 1, 2, sel)
                assert torch.equal(sel.cpu(), want)
        # heads of an odd distance
        wide = torch.randn((c.T, H * G, D + step), device="cuda").to(dt)[:, :, :D]
        wide.copy_(c.qd)
        pp.pp_cache_select(c.cache, wide, c.sd, c.td, c.ld, pp.PP_ATTN_CAUSAL, 1, 2, sel)
        assert torch.equal(sel.cpu(), want)
    finally:
        c.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
def test_rotate_and_attend_at_16_byte_offsets(pp, dt):
    """Rows that begin 16 bytes, or one value, into a wider boundary: stores, tiles and rows."""
    step = 16 // torch.empty(0, dtype=dt).element_size()
    for off in (step, 1):
        for tokens in (None, [90], [700]):
            c = Case(pp, dt, 4, 2, 64, 16, [720], tokens, seed=2)
            try:
                T, Hq, D = c.q.shape
                view = torch.zeros((T, Hq * D + 2 * step), device="cuda", dtype=dt)[:, off: off + Hq * D].unflatten(1, (Hq, D))
                view.copy_(c.qd)
                c.check(q=view)
            finally:
                c.close()
