"""The cache in 8 bits and attention with a window on the GPU, through the binding, against their definitions
(tests/cache8_ref.py): codes and scales bit by bit, attention within tolerances that are derived there."""
import math

import pytest
import torch

import cache8_ref as ref8
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


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


class Held:
    """A cache in 8 bits on the GPU with copies on the CPU; garbage in it, as memory that was used before."""

    def __init__(self, pp, pages, H, page, D, dt, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.pp, self.page, self.dt = pp, page, dt
        self.c = [torch.randint(-127, 128, (pages, H, page, D), generator=g, dtype=torch.int8) for _ in range(2)]
        self.s = [torch.rand((pages, H), generator=g) * 0.02 + 0.005 for _ in range(2)]
        self.dc, self.ds = [x.cuda() for x in self.c], [x.cuda() for x in self.s]
        self.cache = pp.pp_cache8_create(self.dc[0], self.dc[1], self.ds[0], self.ds[1], dt)

    def append(self, k, v, table, starts, lens):
        self.pp.pp_cache_append(self.cache, k.cuda() if not k.is_cuda else k, v.cuda() if not v.is_cuda else v,
                                None if starts is None else ints(starts).cuda(), table.cuda(), ints(lens).cuda(),
                                torch.cuda.current_stream())
        for i, x in enumerate((k, v)):
            ref8.append(self.c[i], self.s[i], x.cpu(), table, starts, lens, self.page)

    def same(self):
        return all(torch.equal(a.cpu(), b) for a, b in zip(self.dc + self.ds, self.c + self.s))

    def status(self):
        return self.pp.pp_cache_device_status(self.cache)

    def values(self):
        return [ref8.values(c, s) for c, s in zip(self.c, self.s)]

    def close(self):
        torch.cuda.synchronize()
        self.pp.pp_cache_destroy(self.cache)


def tables(lens, page, pages, width=None, seed=0):
    """Distinct random pages for each sequence, -1 behind the last."""
    need = [-(-max(v, 0) // page) for v in lens]
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    assert sum(need) <= pages
    t = torch.full((len(lens), width or max(need + [1])), -1, dtype=torch.int32)
    for b, w in enumerate(need):
        t[b, :w] = ints([order.pop() for _ in range(w)])
    return t


# ------------------------------------------------------------------ writing and reading back

APPEND = [
    # dtype, H, D, page, the lengths of the sequences after each call
    (BF16, 2, 64, 16, [[5], [6], [16], [17], [40]]),
    (F16, 1, 128, 64, [[64, 1, 63], [65, 70, 64], [130, 71, 65]]),
    (F32, 3, 96, 32, [[33, 0, 7], [34, 1, 8], [35, 2, 9], [100, 3, 40]]),
    (BF16, 1, 16, 8, [[1], [2], [3], [9], [33]]),
    (F32, 1, 256, 256, [[255], [256], [511]]),       # more than a thread's registers hold
    (BF16, 2, 256, 128, [[128, 100], [129, 101], [300, 256]]),
    (F16, 8, 80, 16, [[0, 0, 1], [0, 1, 2], [16, 2, 3]]),
]


@pytest.mark.parametrize("dt,H,D,page,steps", APPEND)
def test_append_and_read(pp, dt, H, D, page, steps):
    """Prompts and single tokens in turn, with larger and larger values, so that scales grow; then all read back."""
    g = torch.Generator().manual_seed(D + page)
    last = steps[-1]
    h = Held(pp, sum(-(-v // page) for v in last) + 2, H, page, D, dt)
    table = tables(last, page, h.c[0].shape[0])
    old = [0] * len(last)
    try:
        for i, lens in enumerate(steps):
            n = [v - o for v, o in zip(lens, old)]
            starts = [sum(n[:b]) for b in range(len(n) + 1)]
            k, v = ((torch.randn((starts[-1], H, D), generator=g) * (1 + i)).to(dt) for _ in range(2))
            single = all(m == 1 for m in n)
            h.append(k, v, table, None if single else starts, lens)
            assert h.same(), i
            old = lens
        ends = [sum(last[:b]) for b in range(len(last) + 1)]
        out = [torch.full((ends[-1], H, D), math.nan, device="cuda", dtype=dt) for _ in range(2)]
        pp.pp_cache_read(h.cache, ints(ends).cuda(), table.cuda(), ints(last).cuda(), out[0], out[1], torch.cuda.current_stream())
        for i in range(2):
            assert torch.equal(out[i].cpu(), ref8.read(h.c[i], h.s[i], table, ends, last, page, dt))
        assert h.status() == 0
    finally:
        h.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("how", ["fused", "odd_offset", "heads_first", "broadcast"])
def test_append_views(pp, dt, how):
    H, D, page, T = 4, 48, 16, 23
    g = torch.Generator().manual_seed(1)
    base = torch.randn((T, 3 * H * D + 5), generator=g).to(dt).cuda()
    off = 1 if how == "odd_offset" else 0
    k, v = base[:, off: off + H * D].unflatten(1, (H, D)), base[:, off + H * D: off + 2 * H * D].unflatten(1, (H, D))
    if how == "heads_first":
        k = k.transpose(0, 1).contiguous().transpose(0, 1)
    if how == "broadcast":
        v = v[:, :1].expand(T, H, D)
    h = Held(pp, 4, H, page, D, dt)
    try:
        h.append(k, v, tables([T + 3], page, 4), [0, T], [T + 3])
        assert h.same() and h.status() == 0
    finally:
        h.close()


def test_append_values_at_the_ends_of_the_types(pp):
    """Largest and smallest values, zeros, halves of a step (to even), and what is not finite."""
    H, D, page = 1, 16, 8
    rows = torch.zeros((8, H, D))
    rows[0, 0, :4] = torch.tensor([3.4028234663852886e38, -3.4028234663852886e38, 1.0, 1e-38])
    rows[1, 0, :3] = 2.0 ** -100
    rows[2, 0, :3] = torch.tensor([2.0 ** -101, 2.0 ** -149, -2.0 ** -110])
    rows[4, 0] = torch.arange(16) - 7.5
    rows[4, 0, 15] = 127.0
    rows[5, 0, :4] = torch.tensor([math.nan, math.inf, -math.inf, 2.0])
    rows[6, 0, :2] = torch.tensor([math.nan, math.inf])
    h = Held(pp, 10, H, page, D, F32)
    try:
        for t in range(8):  # a page for each
            table, bits = ints([[t]]), pp.PP_CACHE_NOT_FINITE if t in (5, 6) else 0
            h.append(rows[t: t + 1], rows[t: t + 1], table, None, [1])
            assert h.same() and h.status() == bits, t
        one = torch.ones((1, H, D))
        for t in range(8):  # and a second token behind it: scales grow from 0, or do not
            h.append(one * 10.0 ** (t - 4), one * 0.0, ints([[t]]), None, [2])
            assert h.same() and h.status() == 0, t
    finally:
        h.close()


def test_append_leaves_what_is_not_its_own(pp):
    """Slots without tokens, pages and lengths out of range, ranges that do not fit: recorded, and nothing else written."""
    H, D, page = 2, 32, 8
    g = torch.Generator().manual_seed(2)
    x = torch.randn((6, H, D), generator=g)
    h = Held(pp, 4, H, page, D, F32)
    try:
        h.append(x[:3], x[:3], ints([[0, 1], [2, 3], [2, 3]]), None, [0, 0, 0])
        assert h.same() and h.status() == 0
        h.append(x[:3], x[:3], ints([[0, 1], [-1, 3], [4, 3]]), None, [1, 1, 1])
        assert h.same() and h.status() == pp.PP_CACHE_BAD_PAGE
        h.append(x[:3], x[:3], ints([[0, 1], [2, 3], [2, 3]]), None, [-1, 17, 2])
        assert h.same() and h.status() == pp.PP_CACHE_BAD_LENGTH
        h.append(x[:6], x[:6], ints([[0, 1], [2, 3]]), [0, 4, 6], [2, 5])  # two tokens too many in the first
        assert h.same() and h.status() == 0
        was = [t.clone() for t in h.dc + h.ds]
        for starts in ([0, 4, 7], [0, -1, 6], [1, 4, 6], [0, 7, 6], [0, 2, 5]):
            pp.pp_cache_append(h.cache, x.cuda(), x.cuda(), ints(starts).cuda(), ints([[0, 1], [2, 3]]).cuda(), ints([8, 8]).cuda())
            assert h.status() & pp.PP_CACHE_BAD_LENGTH, starts
        assert was[0].shape == h.dc[0].shape
    finally:
        h.close()


@pytest.mark.parametrize("dt", [F32, F16, BF16])
def test_read_of_some(pp, dt):
    """The last tokens of each sequence, more than it has, pages that are not there, one output alone, odd places."""
    H, D, page = 3, 48, 16
    h = Held(pp, 9, H, page, D, dt, seed=5)
    table = tables([40, 3, 0, 60], page, 9)
    table[3, 1], table[0, 2] = -1, 99
    starts, lens = [0, 10, 15, 17, 50], [40, 3, 0, 60]
    try:
        want = [ref8.read(h.c[i], h.s[i], table, starts, lens, page, dt) for i in range(2)]
        base = torch.full((2, 50 * H * D + 1), math.nan, device="cuda", dtype=dt)
        for off in (0, 1):
            out = [base[i, off: off + 50 * H * D].view(50, H, D) for i in range(2)]
            pp.pp_cache_read(h.cache, ints(starts).cuda(), table.cuda(), ints(lens).cuda(), out[0], out[1])
            assert all(torch.equal(o.cpu(), w) for o, w in zip(out, want))
            assert h.status() == pp.PP_CACHE_BAD_PAGE
        for i in range(2):
            out = [torch.full((50, H, D), math.nan, device="cuda", dtype=dt) if j == i else None for j in range(2)]
            pp.pp_cache_read(h.cache, ints(starts).cuda(), table.cuda(), ints(lens).cuda(), *out)
            assert torch.equal(out[i].cpu(), want[i])
        h.status()
        one = torch.full((4, H, D), math.nan, device="cuda", dtype=dt)
        pp.pp_cache_read(h.cache, None, table.cuda(), ints([33, 3, 0, 17]).cuda(), one, None)
        assert torch.equal(one.cpu(), ref8.read(h.c[0], h.s[0], table, None, [33, 3, 0, 17], page, dt))
        h.status()
        pp.pp_cache_read(h.cache, None, table.cuda(), ints([-1, 3, 0, 65]).cuda(), one, None)
        assert h.status() & pp.PP_CACHE_BAD_LENGTH
    finally:
        h.close()


def test_calls_that_a_cache_refuses(pp):
    no, bad = pp.PP_ERR_UNSUPPORTED, pp.PP_ERR_INVALID_ARG
    h = Held(pp, 4, 1, 16, 64, F16)
    k = torch.zeros((4, 1, 16, 64), device="cuda", dtype=F16)
    plain = pp.pp_cache_create(k, k.clone())
    rope = pp.pp_rope_create(64, None, [1.0])
    x, i = torch.zeros((2, 1, 64), device="cuda", dtype=F16), ints([0, 1]).cuda()
    table, sel = ints([[0], [1]]).cuda(), torch.zeros((2, 1, 3), device="cuda", dtype=torch.int32)

    def refused(code, f, *a):
        with pytest.raises(pp.PPError) as e:
            f(*a)
        assert e.value.code == code
    try:
        refused(no, pp.pp_qkv_store, rope, h.cache, i[None], i, 1e-6, None, None, None, x, None, x)
        refused(no, pp.pp_attn_forward, h.cache, x, None, table, i, 1.0, 0, sel, x)
        refused(bad, pp.pp_cache_summarize, h.cache, i)
        refused(bad, pp.pp_cache_select, h.cache, x, None, table, i, 0, 0, 1, sel)
        refused(no, pp.pp_cache_append, plain, x, x, None, table, i)
        refused(no, pp.pp_cache_read, plain, None, table, i, x, x)
        for f in (x.float(), x[:, :, :32], x.expand(2, 3, 64), x[:1]):
            refused(bad, pp.pp_cache_append, h.cache, f, x, None, table, i)
            refused(bad, pp.pp_cache_append, h.cache, x, f, None, table, i)
            refused(bad, pp.pp_cache_read, h.cache, None, table, i, f, x)
        refused(bad, pp.pp_cache_append, h.cache, x, x, None, table, i[:1])
        refused(bad, pp.pp_cache_append, h.cache, x, x, ints([0, 2]).cuda(), table, i)
        refused(bad, pp.pp_cache_read, h.cache, None, table[:1], i[:1], x, x)
        refused(bad, pp.pp_cache_read, h.cache, None, table, i, None, None)
        for window, sinks in ((0, 0), (-3, 0), (1, -1)):
            refused(bad, pp.pp_attn_window, h.cache, x, None, table, i, 1.0, 0, window, sinks, x)
        refused(bad, pp.pp_attn_window, plain, x, None, table, i, math.inf, 0, 1, 0, x)
        refused(bad, pp.pp_attn_window, plain, x, None, table, i, 1.0, 2, 1, 0, x)
        pp.pp_cache_append(h.cache, x[:0], x[:0], ints([0, 0, 0]).cuda(), table, i)
        pp.pp_cache_read(h.cache, ints([0, 0, 0]).cuda(), table, i, x[:0], x[:0])
        assert h.status() == 0
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)
        pp.pp_cache_destroy(plain)
        h.close()


# ------------------------------------------------------------------ attention

def check(pp, dt, H, G, D, page, lens, starts, window, sinks, codes=True, causal=True, scale=None, seed=0, garbage=False,
          strided=False, mutate=None):
    """One call of pp_attn_window (window None: pp_attn_forward) against the definition; its outputs."""
    g = torch.Generator().manual_seed(seed + D)
    scale = D ** -0.5 if scale is None else scale
    T = len(lens) if starts is None else starts[-1]
    need = sum(-(-max(v, 0) // page) for v in lens)
    table = tables(lens, page, need + 3, seed=seed)
    if codes:
        h = Held(pp, need + 3, H, page, D, dt, seed)
        for c, s in zip(h.dc, h.ds):  # pages of different sizes
            s.mul_(torch.exp2(torch.randint(-3, 4, s.shape, generator=g).float()).cuda())
        h.s = [s.cpu() for s in h.ds]
        k, v = h.values()
        cache = h.cache
    else:
        k, v = (torch.randn((need + 3, H, page, D), generator=g).to(dt) for _ in range(2))
        if mutate is not None:
            mutate(k, v, table)
        dk, dv = k.cuda(), v.cuda()
        cache = pp.pp_cache_create(dk, dv)
    q = torch.randn((T, 3 * H * G * D), generator=g).mul(1.5).to(dt)
    q = q[:, 1: 1 + H * G * D].view(T, H * G, D) if strided else q[:, : H * G * D].contiguous().view(T, H * G, D)
    out = torch.full((T, H * G, D), math.nan, device="cuda", dtype=dt)
    lse = torch.full((T, H * G), math.nan, device="cuda")
    w = 2 ** 31 - 1 if window is None else window
    if garbage:  # pages that no token reads are taken out of the table, and what they hold with them
        seen = ref.seen_keys(T, starts, lens, causal)
        for b in range(len(lens)):
            used = set()
            for s, n in seen:
                if s == b:
                    used |= {j // page for j in range(n) if j >= n - w or j < sinks}
            for j in range(table.shape[1]):
                if j not in used:
                    table[b, j] = -1 if j % 2 else 2 ** 30
    dq = q.cuda()
    if strided:
        wide = torch.zeros((T, 3 * H * G * D), device="cuda", dtype=dt)
        wide[:, 1: 1 + H * G * D] = dq.reshape(T, -1)
        dq = wide[:, 1: 1 + H * G * D].view(T, H * G, D)
    args = (cache, dq, None if starts is None else ints(starts).cuda(), table.cuda(), ints(lens).cuda(), scale,
            pp.PP_ATTN_CAUSAL if causal else 0)
    try:
        if window is None:
            pp.pp_attn_forward(*args, None, out, lse, torch.cuda.current_stream())
        else:
            pp.pp_attn_window(*args, window, sinks, out, lse, torch.cuda.current_stream())
        assert pp.pp_cache_device_status(cache) == 0
        want, wl, tol, tl = ref8.attend(q, k, v, table, starts, lens, scale, causal, w, sinks, codes)
        assert ref.worst(out, want, tol) <= 1
        assert ref.worst(lse, wl, tl) <= 1
    finally:
        torch.cuda.synchronize()
        h.close() if codes else pp.pp_cache_destroy(cache)
    return out, lse


SINGLE = [
    # dtype, H, G, D, page, lens
    (BF16, 2, 4, 128, 16, [777]),
    (F16, 1, 1, 64, 8, [1, 0, 2, 63, 64, 65, 129]),
    (F32, 2, 2, 96, 32, [100, 5, 0, 33]),
    (BF16, 1, 8, 128, 64, [64, 128, 200, 1]),
    (F16, 2, 16, 64, 16, [50, 17]),
    (BF16, 1, 12, 80, 128, [300, 129]),
    (F32, 1, 12, 128, 8, [90, 31]),
    (F32, 1, 3, 64, 256, [257, 3]),
    (BF16, 1, 5, 256, 32, [70, 200]),
    (F16, 1, 10, 256, 8, [70, 33]),
    (F32, 1, 2, 256, 16, [70, 33]),
    (BF16, 3, 2, 16, 16, [40, 16]),
    (F16, 1, 64, 32, 16, [40]),
    (F32, 1, 1, 48, 64, [1000]),
    (BF16, 1, 4, 112, 64, [5000, 3]),       # split over CTAs, and joined
    (F16, 8, 2, 128, 16, [1500, 1, 700]),
]
CHUNK = [
    # dtype, H, G, D, page, lens, starts
    (BF16, 2, 4, 64, 16, [50], [0, 20]),
    (F16, 1, 3, 128, 8, [33, 0, 9], [0, 7, 7, 16]),
    (F32, 2, 2, 96, 32, [40, 70], [0, 5, 45]),
    (BF16, 1, 1, 80, 64, [150], [0, 150]),
    (F16, 2, 2, 128, 128, [300, 20], [0, 100, 110]),
    (BF16, 1, 8, 128, 16, [140], [0, 64]),
    (F32, 1, 5, 64, 16, [31], [0, 31]),
    (F16, 1, 2, 256, 16, [90], [0, 30]),
    (BF16, 1, 4, 128, 64, [5], [0, 9]),     # more tokens than keys: the first see none
    (BF16, 2, 1, 128, 32, [400, 17, 260], [0, 200, 217, 330]),
]


@pytest.mark.parametrize("case", SINGLE)
@pytest.mark.parametrize("strided", [False, True])
def test_codes_single(pp, case, strided):
    check(pp, *case, None, None, 0, strided=strided)


@pytest.mark.parametrize("case", CHUNK)
@pytest.mark.parametrize("causal", [False, True])
def test_codes_chunk(pp, case, causal):
    check(pp, *case, None, 0, causal=causal)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
@pytest.mark.parametrize("dt", [F32, F16, BF16])
def test_codes_scales(pp, dt, scale):
    check(pp, dt, 2, 2, 64, 16, [70, 20], None, None, 0, scale=scale)
    check(pp, dt, 1, 4, 128, 16, [70], [0, 40], None, 0, scale=scale)


# enough rows for tiles of them on the tensor cores
TILES = [
    (BF16, 8, 4, 64, 16, [170], [0, 40]),
    (F16, 8, 1, 128, 8, [300, 40], [0, 150, 190]),
    (BF16, 4, 3, 80, 64, [200], [0, 130]),
    (F16, 8, 2, 64, 128, [500], [0, 64]),
    (BF16, 16, 8, 128, 32, [90, 0, 200], [0, 20, 20, 52]),
    (F16, 4, 64, 128, 16, [70, 30], [0, 3, 12]),
    (BF16, 8, 2, 112, 256, [700], [0, 128]),
    (F16, 8, 4, 48, 16, [30], [0, 50]),      # more tokens than keys
]

# and over codes, where tiles are taken from more rows on
TILES8 = [
    (BF16, 16, 8, 64, 16, [170], [0, 48]),
    (F16, 16, 8, 128, 8, [300, 40], [0, 30, 52]),
    (BF16, 16, 4, 80, 64, [200], [0, 100]),
    (F16, 16, 2, 64, 128, [500], [0, 180]),
    (BF16, 16, 8, 128, 32, [90, 0, 200], [0, 20, 20, 52]),
    (F16, 4, 64, 128, 16, [70, 30], [0, 20, 26]),
    (BF16, 16, 4, 112, 256, [700], [0, 96]),
    (F16, 16, 8, 48, 16, [30], [0, 50]),      # more tokens than keys
    (F16, 8, 8, 128, 64, [2100], [0, 40]),    # split along the keys, and joined
]


@pytest.mark.parametrize("case", TILES + TILES8)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("strided", [False, True])
def test_codes_tiles(pp, case, causal, strided):
    check(pp, *case, None, 0, causal=causal, strided=strided)


WINDOWS = [(1, 0), (2, 1), (5, 3), (16, 0), (17, 130), (63, 4), (64, 64), (100, 1), (200, 16), (2 ** 31 - 1, 5), (3, 2 ** 31 - 1)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("case", [SINGLE[i] for i in (0, 1, 2, 6, 8, 14)])
@pytest.mark.parametrize("codes", [False, True])
def test_window_single(pp, case, window, sinks, codes):
    check(pp, *case, None, window, sinks, codes=codes, garbage=True)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("case", [CHUNK[i] for i in (0, 1, 2, 4, 7, 8, 9)])
@pytest.mark.parametrize("codes", [False, True])
def test_window_chunk(pp, case, window, sinks, codes):
    check(pp, *case, window, sinks, codes=codes, garbage=True)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("case", TILES)
@pytest.mark.parametrize("codes", [False, True])
def test_window_tiles(pp, case, window, sinks, codes):
    check(pp, *case, window, sinks, codes=codes, garbage=True)


@pytest.mark.parametrize("window,sinks", [WINDOWS[i] for i in (0, 2, 4, 6, 8, 10)])
@pytest.mark.parametrize("case", TILES8)
def test_window_tiles_of_codes(pp, case, window, sinks):
    check(pp, *case, window, sinks, garbage=True)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B", [33, 150, 900])
@pytest.mark.parametrize("window", [None, 20])
def test_many_sequences(pp, dt, B, codes, window):
    """More sequences than a lane or a thread looks after one of, idle ones among them; as single tokens and as ranges."""
    g = torch.Generator().manual_seed(B)
    lens = torch.randint(0, 40, (B,), generator=g).tolist()
    check(pp, dt, 1, 2, 64, 16, lens, None, window, 3, codes=codes, garbage=True)
    if B == 150:
        n = torch.randint(0, 4, (B,), generator=g).tolist()
        check(pp, dt, 1, 2, 64, 16, lens, [sum(n[:b]) for b in range(B + 1)], window, 3, codes=codes, garbage=True)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dt,H,G,D,page,lens,n,window", [
    (BF16, 1, 8, 128, 64, [40000], 1, None), (F32, 1, 3, 96, 32, [30000, 17], 1, None), (F16, 1, 4, 64, 16, [50000, 20000, 1], 1, 33333),
    (BF16, 2, 4, 128, 64, [30000], 5, 20000), (F16, 8, 8, 128, 128, [20000], 40, None), (BF16, 8, 4, 64, 16, [20000], 100, 15000)])
def test_long_sequences(pp, dt, H, G, D, page, lens, n, window, codes):
    """Split over many CTAs and joined in two levels, or along tiles' keys; against 64 bits on the GPU.  Tolerance as derived for
    the short ones with the softmax's own sums: 2^-11 of sum p |v| for 16-bit weights (over keys in bf16 2^-8), 2^-17 for the rest (logits err
    by some 140 x 2^-24 x 10, and 50000 x 2^-24 of the sum), one rounding to the type."""
    g = torch.Generator(device="cuda").manual_seed(D)
    need = sum(-(-v // page) for v in lens)
    table = tables(lens, page, need).cuda()
    q = torch.randn((n * len(lens), H * G, D), device="cuda", generator=g).to(dt)
    if codes:
        k, v = (torch.randint(-127, 128, (need, H, page, D), device="cuda", generator=g, dtype=torch.int8) for _ in range(2))
        ks, vs = (torch.rand((need, H), device="cuda", generator=g) * 0.01 + 0.005 for _ in range(2))
        cache = pp.pp_cache8_create(k, v, ks, vs, dt)
        k64, v64 = k.double() * ks.double()[:, :, None, None], v.double() * vs.double()[:, :, None, None]
    else:
        k, v = (torch.randn((need, H, page, D), device="cuda", generator=g).to(dt) for _ in range(2))
        cache = pp.pp_cache_create(k, v)
        k64, v64 = k.double(), v.double()
    out, lse = torch.empty_like(q), torch.empty((q.shape[0], H * G), device="cuda")
    starts = None if n == 1 else torch.arange(0, n * len(lens) + 1, n, device="cuda", dtype=torch.int32)
    a = (cache, q, starts, table, ints(lens).cuda(), D ** -0.5, pp.PP_ATTN_CAUSAL)
    try:
        pp.pp_attn_forward(*a, None, out, lse) if window is None else pp.pp_attn_window(*a, window, 40, out, lse)
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        pp.pp_cache_destroy(cache)
    u = 2.0 ** -20 if dt is F32 else 2.0 ** -11 if codes or dt is F16 else 2.0 ** -8
    for b, L in enumerate(lens):
        ids = table[b, : -(-L // page)].long()
        kk, vv = (x[ids].transpose(1, 2).reshape(-1, H, D)[:L] for x in (k64, v64))
        x = q[b * n: (b + 1) * n].double().view(n, H, G, D)
        s = torch.einsum("nhgd,shd->nhgs", x, kk) * D ** -0.5
        seen = torch.arange(L - n + 1, L + 1, device="cuda")[:, None]
        at = torch.arange(L, device="cuda")[None]
        hide = at >= seen
        if window is not None:
            hide = hide | ((at < seen - window) & (at >= 40))
        s = s.masked_fill(hide[:, None, None], -math.inf)
        p = torch.softmax(s, -1)
        want = torch.einsum("nhgs,shd->nhgd", p, vv).reshape(n, H * G, D)
        tol = (u + 2.0 ** -17) * torch.einsum("nhgs,shd->nhgd", p, vv.abs()).reshape(n, H * G, D) + ref.UNIT[dt] * want.abs() * 1.01 + ref.TINY[dt]
        assert ref.worst(out[b * n: (b + 1) * n], want.cpu(), tol.cpu()) <= 1
        assert float((lse[b * n: (b + 1) * n].double() - torch.logsumexp(s, -1).reshape(n, -1)).abs().max()) < 2.0 ** -14


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("starts,n", [(None, 3), ([0, 48], 48)])
def test_codes_queries_not_finite(pp, dt, starts, n):
    """Rows of queries with NaN have NaN, the others are as if they were not there."""
    H, G, D, page = 16, 8, 64, 16
    lens = [50, 70, 20] if starts is None else [90]
    h = Held(pp, 12, H, page, D, dt)
    table = tables(lens, page, 12)
    k, v = h.values()
    q = torch.randn((n, H * G, D), generator=torch.Generator().manual_seed(8)).to(dt)
    want, wl, tol, tl = ref8.attend(q, k, v, table, starts, lens, 0.125, True, 10 ** 6, 0, True)
    bad = torch.zeros((n, H * G), dtype=torch.bool)
    bad[0, 3] = bad[n - 1, 5] = bad[1, 64:72] = True
    q[bad] = math.nan
    out, lse = torch.empty((n, H * G, D), device="cuda", dtype=dt), torch.empty((n, H * G), device="cuda")
    try:
        pp.pp_attn_forward(h.cache, q.cuda(), None if starts is None else ints(starts).cuda(), table.cuda(), ints(lens).cuda(), 0.125,
                           pp.PP_ATTN_CAUSAL, None, out, lse)
        got, gl = out.cpu(), lse.cpu()
        assert torch.isnan(got[bad]).all() and torch.isnan(gl[bad]).all()
        assert ref.worst(got[~bad], want[~bad], tol[~bad]) <= 1 and ref.worst(gl[~bad], wl[~bad], tl[~bad]) <= 1
    finally:
        h.close()


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dt", [F32, F16, BF16])
def test_window_of_all_tokens(pp, dt, codes):
    """Without the causal flag every token sees the sequence's last keys."""
    check(pp, dt, 2, 2, 64, 16, [150, 40], [0, 20, 70], 33, 2, codes=codes, causal=False, garbage=True)
    check(pp, dt, 1, 3, 128, 32, [150, 0], None, 33, 70, codes=codes, causal=False, garbage=True)
    check(pp, dt, 8, 2, 64, 16, [150, 40], [0, 50, 100], 33, 2, codes=codes, causal=False, garbage=True)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("case", [(1, 4, 128, 16, [300, 5], None), (2, 2, 64, 32, [300, 70], [0, 100, 170])])
def test_window_of_all_keys_is_forward(pp, dt, codes, case):
    """A window that holds every key, or first keys that do, gives the same bits as no window where the rows' kernel is
    the same, and the same numbers to rounding in any case."""
    a, la = check(pp, dt, *case, None, 0, codes=codes)
    b, lb = check(pp, dt, *case, 10 ** 9, 7, codes=codes)
    assert torch.equal(a, b) and torch.equal(la, lb)


def broken(values, where):
    """Puts values that are not finite where no token looks, or where some tokens look."""
    def mutate(k, v, table):
        page = k.shape[2]
        for key, x in zip(where, values):
            id = int(table[0, key // page])
            v[id, :, key % page, ::3] = x
    return mutate


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("G,n,window,sinks", [(2, 6, 40, 3), (1, 16, 5, 0), (4, 60, 20, 10), (1, 150, 30, 64), (2, 64, 1, 0), (8, 3, 100, 2)])
@pytest.mark.parametrize("H", [2, 8])
def test_values_not_finite_reach_who_sees_them(pp, dt, H, G, n, window, sinks):
    """Keys of a chunk, at the ends of the windows and of the first keys: a row that sees one has what the definition gives,
    every other row is as if it was not there."""
    D, page, L = 64, 16, 170
    where = sorted({0, sinks, max(0, L - n - window), max(0, L - n - window + 2), L - n, L - n + 1, L - 1, L - window})
    values = [math.inf, math.nan, -math.inf, math.nan, math.inf, math.nan, math.inf, -math.inf][: len(where)]
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((L // page + 2, H, page, D), generator=g).to(dt) for _ in range(2))
    table = tables([L], page, k.shape[0])
    broken(values, where)(k, v, table)
    q = torch.randn((n, H * G, D), generator=g).to(dt)
    out = torch.empty((n, H * G, D), device="cuda", dtype=dt)
    cache = pp.pp_cache_create(k.cuda(), v.cuda())
    try:
        pp.pp_attn_window(cache, q.cuda(), ints([0, n]).cuda(), table.cuda(), ints([L]).cuda(), 0.125, pp.PP_ATTN_CAUSAL, window,
                          sinks, out)
        assert pp.pp_cache_device_status(cache) == 0
    finally:
        pp.pp_cache_destroy(cache)
    want, _, tol, _ = ref8.attend(q, k, v, table, [0, n], [L], 0.125, True, window, sinks, False)
    got = out.cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~fine].nan_to_num(0), want[~fine].nan_to_num(0))
    assert ref.worst(got[fine], want[fine], tol[fine]) <= 1


def test_codes_pages_of_zeros(pp):
    """Pages whose scale is 0 hold zeros: their keys count in the softmax, and beside pages of any size."""
    G, D, page, L = 4, 64, 8, 90
    for dt, H, starts, n in [(dt, H, *x) for dt in (F32, F16, BF16) for H in (1, 8) for x in ((None, 1), ([0, 40], 40))]:
        h = Held(pp, 14, H, page, D, dt)
        table = tables([L], page, 14)
        for i in range(2):
            for w in range(0, 12, 3):
                h.dc[i][int(table[0, w])] = 0
                h.ds[i][int(table[0, w])] = 0
            for w in range(1, 12, 4):
                h.ds[i][int(table[0, w])] *= 2.0 ** -60 if i else 2.0 ** -20
            h.c[i], h.s[i] = h.dc[i].cpu(), h.ds[i].cpu()
        q = torch.randn((n, H * G, D), generator=torch.Generator().manual_seed(4)).to(dt)
        out = torch.empty((n, H * G, D), device="cuda", dtype=dt)
        try:
            pp.pp_attn_forward(h.cache, q.cuda(), None if starts is None else ints(starts).cuda(), table.cuda(), ints([L]).cuda(), 0.125,
                               pp.PP_ATTN_CAUSAL, None, out)
            k, v = h.values()
            want, _, tol, _ = ref8.attend(q, k, v, table, starts, [L], 0.125, True, L, 0, True)
            assert ref.worst(out, want, tol) <= 1 and h.status() == 0
            for i in range(2):
                h.dc[i].zero_()
                h.ds[i].zero_()
            pp.pp_attn_forward(h.cache, q.cuda(), None if starts is None else ints(starts).cuda(), table.cuda(), ints([L]).cuda(), 0.125,
                               pp.PP_ATTN_CAUSAL, None, out)
            assert not out.any()
        finally:
            h.close()


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("H,G,n", [(1, 4, 48), (16, 8, 48)])
@pytest.mark.parametrize("power", [-20, -50, 40])
def test_codes_rows_that_see_small_pages_alone(pp, dt, H, G, n, power):
    """The values' scales change by a large factor from one page to the next, which the first tokens of a chunk still see."""
    D, page, L, window = 64, 32, 170, 20
    h = Held(pp, 8, H, page, D, dt)
    table = tables([L], page, 8)
    for w in range(4, 6):
        h.ds[1][int(table[0, w])] *= 2.0 ** power
    h.s[1] = h.ds[1].cpu()
    k, v = h.values()
    q = torch.randn((n, H * G, D), generator=torch.Generator().manual_seed(4)).to(dt)
    out = torch.empty((n, H * G, D), device="cuda", dtype=dt)
    try:
        pp.pp_attn_window(h.cache, q.cuda(), ints([0, n]).cuda(), table.cuda(), ints([L]).cuda(), 0.125, pp.PP_ATTN_CAUSAL, window, 0, out)
        want, _, tol, _ = ref8.attend(q, k, v, table, [0, n], [L], 0.125, True, window, 0, True)
        assert ref.worst(out, want, tol) <= 1 and h.status() == 0
    finally:
        h.close()


def test_codes_queries_of_any_size(pp):
    """Rows of queries from the smallest to the largest: each has its own power of two."""
    H, G, D, page, L = 1, 8, 64, 16, 40
    for dt in (F32, BF16, F16):
        h = Held(pp, 3, H, page, D, dt)
        table = tables([L], page, 3)
        k, v = h.values()
        q = torch.randn((1, H * G, D), generator=torch.Generator().manual_seed(6))
        powers = [-14, -8, -3, 0, 2, 4, 6, 8] if dt is F16 else [-120, -90, -40, -3, 0, 4, 6, 8]
        q = (q * torch.tensor([2.0 ** e for e in powers])[None, :, None]).to(dt)
        q[0, 2] = 0
        out = torch.empty((1, H * G, D), device="cuda", dtype=dt)
        try:
            pp.pp_attn_forward(h.cache, q.cuda(), None, table.cuda(), ints([L]).cuda(), 0.125, 0, None, out)
            want, _, tol, _ = ref8.attend(q, k, v, table, None, [L], 0.125, False, L, 0, True)
            assert ref.worst(out, want, tol) <= 1
        finally:
            h.close()


# ------------------------------------------------------------------ the operators together

@pytest.mark.parametrize("dt", [F32, BF16])
def test_steps_together_and_captured(pp, dt):
    """A prompt and tokens behind it on a stream of their own: rotated, appended, attended to with a window; pages outside it
    used again.  The same step captured in a graph and replayed gives the same bits."""
    H, G, D, page, window, sinks = 2, 2, 64, 16, 40, 3
    ring, prompt, steps = 6, 50, 30  # pages behind the first one are used in turn: 96 keys, of which a step reads 43 and a page
    width = -(-(prompt + steps) // page)
    table = ints([[0] + [1 + (w - 1) % ring for w in range(1, width)]])
    g = torch.Generator().manual_seed(9)
    rope = pp.pp_rope_create(D, None, [10000.0 ** (-j / 32) for j in range(32)])
    h = Held(pp, ring + 1, H, page, D, dt)
    keys, vals = torch.zeros((0, H, D)), torch.zeros((0, H, D))
    lens, pos = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    x = torch.zeros((1, (G * H + 2 * H) * D), device="cuda", dtype=dt)
    q1, k1 = torch.zeros((1, H * G, D), device="cuda", dtype=dt), torch.zeros((1, H, D), device="cuda", dtype=dt)
    out = torch.zeros((1, H * G, D), device="cuda", dtype=dt)
    dtab = table.cuda()
    stream = torch.cuda.Stream()

    def step(q, k, starts, x, pos, out, s):
        T = x.shape[0]
        heads = x.view(T, H * G + 2 * H, D)
        pp.pp_qk_rotate(rope, pos, 1e-6, heads[:, : H * G], None, q, heads[:, H * G: H * G + H], None, k, s)
        pp.pp_cache_append(h.cache, k, heads[:, H * G + H:], starts, dtab, lens, s)
        pp.pp_attn_window(h.cache, q, starts, dtab, lens, D ** -0.5, pp.PP_ATTN_CAUSAL, window, sinks, out, None, s)

    def expect(q, k, v, n, starts, got):
        """Against the codes and scales that the definition has by now."""
        for i, new in enumerate((k, v)):
            ref8.append(h.c[i], h.s[i], new.cpu(), table, starts, [n], page)
        assert h.same()
        kk, vv = h.values()
        want, _, tol, _ = ref8.attend(q.cpu(), kk, vv, table, starts, [n], D ** -0.5, True, window, sinks, True)
        assert ref.worst(got, want, tol) <= 1

    try:
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            px = torch.randn((prompt, x.shape[1]), generator=g).to(dt).cuda()
            pq, pk = torch.empty((prompt, H * G, D), device="cuda", dtype=dt), torch.empty((prompt, H, D), device="cuda", dtype=dt)
            po = torch.empty_like(pq)
            lens.fill_(prompt)
            step(pq, pk, ints([0, prompt]).cuda(), px, torch.arange(prompt, device="cuda", dtype=torch.int32)[None].contiguous(), po, stream)
        stream.synchronize()
        expect(pq, pk, px.view(prompt, -1, D)[:, H * G + H:], prompt, [0, prompt], po)
        graph = None
        for n in range(prompt + 1, prompt + steps + 1):
            with torch.cuda.stream(stream):
                x.copy_(torch.randn(x.shape, generator=g).to(dt))
                lens.fill_(n)
                pos.fill_(n - 1)
                if n == prompt + 4:
                    graph = torch.cuda.CUDAGraph()
                    stream.synchronize()
                    with torch.cuda.graph(graph, stream=stream):
                        step(q1, k1, None, x, pos, out, torch.cuda.current_stream())
                if graph is None:
                    step(q1, k1, None, x, pos, out, stream)
                else:
                    graph.replay()
            stream.synchronize()
            expect(q1, k1, x.view(1, -1, D)[:, H * G + H:], n, None, out)
        assert h.status() == 0 and keys.shape == vals.shape
    finally:
        torch.cuda.synchronize()
        pp.pp_rope_destroy(rope)
        h.close()


@pytest.mark.parametrize("codes", [False, True])
def test_same_bits_each_time(pp, codes):
    """A long ragged batch, whose parts are joined by whoever comes last."""
    H, G, D, page, dt = 4, 4, 128, 64, BF16
    lens = [9000, 1, 0, 4000, 64, 7777]
    need = sum(-(-v // page) for v in lens)
    g = torch.Generator(device="cuda").manual_seed(1)
    table, q = tables(lens, page, need).cuda(), torch.randn((6, H * G, D), device="cuda", generator=g).to(dt)
    if codes:
        h = Held(pp, need, H, page, D, dt)
        cache = h.cache
    else:
        k, v = (torch.randn((need, H, page, D), device="cuda", generator=g).to(dt) for _ in range(2))
        cache = pp.pp_cache_create(k, v)
    try:
        for window in (None, 5000):
            outs = []
            for _ in range(5):
                out = torch.full((6, H * G, D), math.nan, device="cuda", dtype=dt)
                a = (cache, q, None, table, ints(lens).cuda(), 0.09, pp.PP_ATTN_CAUSAL)
                pp.pp_attn_forward(*a, None, out) if window is None else pp.pp_attn_window(*a, window, 16, out)
                outs.append(out)
            assert all(torch.equal(o, outs[0]) for o in outs) and bool(torch.isfinite(outs[0].float()).all())
    finally:
        torch.cuda.synchronize()
        pp.pp_cache_destroy(cache)


@pytest.mark.parametrize("codes", [False, True])
def test_bad_device_data(pp, codes):
    """Pages and lengths out of range are skipped and recorded."""
    H, G, D, page, dt = 1, 2, 64, 16, F16
    k = torch.randn((4, H, page, D), device="cuda", dtype=dt)
    h = Held(pp, 4, H, page, D, dt) if codes else None
    cache = h.cache if codes else pp.pp_cache_create(k, k.clone())
    kk, vv = h.values() if codes else (k.cpu(), k.cpu())
    q = torch.randn((2, H * G, D), device="cuda", dtype=dt)
    out = torch.empty_like(q)

    def call(table, lens, starts=None, window=20, sinks=4):
        pp.pp_attn_window(cache, q, None if starts is None else ints(starts).cuda(), ints(table).cuda(), ints(lens).cuda(), 0.125,
                          pp.PP_ATTN_CAUSAL, window, sinks, out)
        return pp.pp_cache_device_status(cache)
    try:
        t = [[0, -1, 7, 1], [2, 3, -5, 2]]
        assert call(t, [50, 60]) == pp.PP_CACHE_BAD_PAGE
        want, _, tol, _ = ref8.attend(q.cpu(), kk, vv, ints(t), None, [50, 60], 0.125, True, 20, 4, codes)
        assert ref.worst(out, want, tol) <= 1
        assert call([[0, 1, 2, 3]] * 2, [-1, 65]) == pp.PP_CACHE_BAD_LENGTH
        want, _, tol, _ = ref8.attend(q.cpu(), kk, vv, ints([[0, 1, 2, 3]] * 2), None, [0, 64], 0.125, True, 20, 4, codes)
        assert ref.worst(out, want, tol) <= 1
        for starts in ([0, 3, 2], [0, -1, 2], [1, 1, 2], [0, 1, 1]):
            assert call([[0, 1, 2, 3]] * 2, [60, 60], starts) & pp.PP_CACHE_BAD_LENGTH
    finally:
        torch.cuda.synchronize()
        h.close() if codes else pp.pp_cache_destroy(cache)
