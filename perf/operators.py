"""What is measured: the operators that follow a vision trunk in a program that answers about its frames.

The trunk's maps become tokens on a (time, row, column) grid; a decoder keeps their keys and values in a paged
cache and attends to them.  A case is one step of such a program on one of its layers.

Kinds of cases (``"kind"``):
  rotate   queries and keys of T tokens, normalised per head and rotated (``pp_qk_rotate``).
  store    the same, the keys and the values written to their slots of the paged cache (``pp_qkv_store``).
  attend   one new token of each of B sequences over its cached keys (``pp_attn_forward``).
  sparse   n new tokens of each of B sequences: pages selected by a cheap score (``pp_cache_select``), attention
           over the selected ones; ``"fresh"``: the pages that the chunk filled are summarised first
           (``pp_cache_summarize``).

Layouts: pools [pages][Hkv][page][D]; queries, keys and values are views of one fused [T][(Hq + 2 Hkv) D] product;
outputs [T][Hq][D].  ``L`` is the longest sequence; ``ragged`` spreads the lengths from an idle slot (0) to L.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
THETA = 10000.0


def _rows(name, kind, dtype, T, Hq, Hkv, D, page, side, pairs=0, interleaved=False):
    """``side``: tokens of a video, side x side per frame; 0: text tokens, one position on every axis."""
    c = dict(kind=kind, dtype=dtype, T=T, Hq=Hq, Hkv=Hkv, D=D, page=page, side=side, pairs=pairs or D // 2, interleaved=interleaved)
    return dict(c, name=name) if name else c


def _attend(name, dtype, B, L, Hq, Hkv, D, page, ragged):
    c = dict(kind="attend", dtype=dtype, B=B, n=1, L=L, Hq=Hq, Hkv=Hkv, D=D, page=page, ragged=ragged)
    return dict(c, name=name) if name else c


def _sparse(name, dtype, B, n, L, Hq, Hkv, D, page, keep, first=1, last=2, ragged=False):
    c = dict(kind="sparse", dtype=dtype, B=B, n=n, L=L, Hq=Hq, Hkv=Hkv, D=D, page=page, keep=keep, first=first, last=last,
             ragged=ragged, fresh=n > 1)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The next token of one answer, a small decoder (512 channels, as the VGG-16 trunk's maps): latency decides.
        _rows("store_1_bf16", "store", "bf16", 1, 8, 8, 64, 16, 0),
        # One step of 64 answers at once, queries of 32 heads over 8 key heads.
        _rows("store_64_bf16", "store", "bf16", 64, 32, 8, 128, 64, 0),
        # 16 frames of 14 x 14 trunk positions, in the library's own fp32, not cached.
        _rows("rotate_video_f32", "rotate", "f32", 3136, 8, 8, 64, 16, 14),
        # A long prompt: 16384 tokens with their keys and values into the cache.
        _rows("store_16384_f16", "store", "f16", 16384, 32, 8, 128, 64, 32),
        # One short answer: 777 cached tokens, latency again.
        _attend("attend_1x777_bf16", "bf16", 1, 777, 8, 2, 128, 16, False),
        # fp32 decoder, heads of 96, pages of 16.
        _attend("attend_16x2500_f32", "f32", 16, 2500, 8, 4, 96, 16, True),
        # A server's batch: 48 sequences from idle to 8192 tokens.
        _attend("attend_48x8192_bf16", "bf16", 48, 8192, 32, 8, 128, 64, True),
        # Long videos: 8 sequences of 65536 tokens.
        _attend("attend_8x65536_f16", "f16", 8, 65536, 32, 8, 128, 64, False),
        # One answer about a long video: 32 of 625 pages read.
        _sparse("sparse_1x40000_bf16", "bf16", 1, 1, 40000, 32, 8, 128, 64, 32),
        # The batched form of the same.
        _sparse("sparse_32x32768_bf16", "bf16", 32, 1, 32768, 32, 8, 128, 64, 32, ragged=True),
        # Odd chunks of three prompts, heads of 64, small pages.
        _sparse("sparse_3x333_f16", "f16", 3, 333, 5001, 8, 4, 64, 32, 20),
        # A prompt's chunk of 2048 tokens behind 30720 cached ones.
        _sparse("sparse_2048x32768_bf16", "bf16", 1, 2048, 32768, 32, 8, 128, 64, 32),
    ]


# ------------------------------------------------------------------ drawn cases


def _log(rng: random.Random, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _fits(c):
    """No drawn case costs more than the largest listed one of its kind."""
    H, D, e = c["Hq"] + 2 * c["Hkv"], c["D"], BYTES[c["dtype"]]
    sizes = [H * D, c["Hq"] * D, c["Hkv"] * D, c.get("T", 0), c.get("L", 0), c.get("keep", 0) * c["page"]]
    if 3072 in sizes:
        return False
    if c["kind"] in ("rotate", "store"):
        return c["T"] * H * D * e <= 16384 * 48 * 128 * 2
    if c["kind"] == "attend":
        return c["B"] * c["L"] * c["Hkv"] * D * e <= 8 * 65536 * 8 * 128 * 2
    return c["n"] < c["L"] and c["B"] * c["n"] * c["Hq"] * c["L"] * D <= 2048 * 32 * 32768 * 128 and c["B"] * c["L"] * c["Hkv"] * D * e <= 2 ** 31


def draw(rng: random.Random):
    """1 .. 16384 tokens to rotate and store; 1 .. 128 sequences of 1 .. 131072 cached tokens; selection for 1 .. 2048
    tokens of 1 .. 48 sequences; heads of 64 .. 128 (attention also 256), groups of 1 .. 8, pages of 16 .. 128."""
    while True:
        kind = rng.choice(["rotate", "store", "attend", "attend", "sparse", "sparse"])
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
        D = rng.choice([64, 80, 96, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        page = rng.choice([16, 32, 64, 128])
        if kind in ("rotate", "store"):
            side = rng.choice([0, 7, 14, 28])
            T = _log(rng, 1, 16384)
            pairs = rng.choice([D // 2, D // 2, D // 4])
            c = _rows(None, kind, dtype, T, Hq, Hkv, D, page, side, pairs, rng.random() < 0.3)
        elif kind == "attend":
            if rng.random() < 0.15:
                D = 256
            c = _attend(None, dtype, _log(rng, 1, 128), _log(rng, 1, 131072), Hq, Hkv, D, page, rng.random() < 0.5)
        else:
            if rng.random() < 0.5:
                B, n = _log(rng, 1, 48), 1
            else:
                B, n = rng.choice([1, 1, 2, 3]), _log(rng, 2, 2048)
            c = _sparse(None, rng.choice(["bf16", "f16", "bf16", "f16", "f32"]), B, n, _log(rng, 64, 65536), Hq, Hkv, D, page,
                        rng.randint(4, 40), rng.randint(0, 2), rng.randint(1, 2), rng.random() < 0.5 and n == 1)
        if _fits(c):
            return c


# ------------------------------------------------------------------ inputs (from the seed alone)


def _lens(c):
    """The sequences' lengths (cached tokens, the new ones among them): of the case alone, so that its work is known."""
    if not c["ragged"] or c["B"] == 1:
        return [c["L"]] * c["B"]
    r = random.Random(c["B"] * 1000003 + c["L"])
    lens = [0, c["L"]] + [r.randint(1, c["L"]) for _ in range(c["B"] - 2)]
    r.shuffle(lens)
    return lens


def _freq(c):
    """(axis of each pair, its frequency): a quarter of the pairs follows time, the rest rows and columns."""
    P = c["pairs"]
    t = P // 4
    h = (P - t) // 2
    return [0] * t + [1] * h + [2] * (P - t - h), [THETA ** (-j / P) for j in range(P)]


class _State:
    pass


def _inputs(c, seed):
    s = _State()
    s.case = c
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPE[c["dtype"]]
    Hq, Hkv, D, page = c["Hq"], c["Hkv"], c["D"], c["page"]

    def normal(*shape, std=1.0, type=dt):
        # in pieces of the first axis where the whole in 32 bits would be large
        x = torch.empty(shape, device="cuda", dtype=type)
        step = max(1, (1 << 28) // max(1, x[0].numel()))
        for i in range(0, shape[0], step):
            x[i: i + step] = torch.randn(x[i: i + step].shape, device="cuda", generator=g) * std
        return x

    if c["kind"] in ("rotate", "store"):
        T = c["T"]
        fused = normal(T, (Hq + 2 * Hkv) * D, std=2.0)
        s.q = fused[:, : Hq * D].view(T, Hq, D)
        s.k = fused[:, Hq * D: (Hq + Hkv) * D].view(T, Hkv, D)
        s.v = fused[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        s.qw = 1.0 + normal(D, std=0.2, type=torch.float32)
        s.kw = 1.0 + normal(D, std=0.2, type=torch.float32)
        i = torch.arange(T, device="cuda", dtype=torch.int32)
        if c["side"]:
            a = c["side"]
            s.pos = torch.stack([i // (a * a), i // a % a, i % a])
        elif T <= 128:  # a step: each token is another sequence's next
            at = torch.randint(0, 200 if c["dtype"] == "f32" else 30000, (T,), device="cuda", generator=g, dtype=torch.int32)
            s.pos = torch.stack([at, at, at])
        else:
            at = i % 256 if c["dtype"] == "f32" else i
            s.pos = torch.stack([at, at, at])
        s.axis, s.freq = _freq(c)
        s.qo = torch.empty((T, Hq, D), device="cuda", dtype=dt)
        if c["kind"] == "rotate":
            s.ko = torch.empty((T, Hkv, D), device="cuda", dtype=dt)
            return s
        pages = -(-T // page) + 2
        order = torch.randperm(pages, device="cuda", generator=g)
        if T <= 128:  # each token in a page of its own sequence where there are pages enough
            s.slots = torch.randperm(pages * page, device="cuda", generator=g)[:T].to(torch.int32)
        else:
            s.slots = (order[(i // page).long()] * page + i % page).to(torch.int32)
        s.kp, s.vp = normal(pages, Hkv, page, D), normal(pages, Hkv, page, D)
        return s

    B, n = c["B"], c["n"]
    lens = _lens(c)
    need = [-(-v // page) for v in lens]
    W = max(need)
    pages = sum(need) + 1
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros((B, W), dtype=torch.int32)
    at, host = 0, order.cpu()
    for b, w in enumerate(need):
        table[b, :w] = host[at: at + w]
        at += w
    s.table = table.cuda()
    s.lens = torch.tensor(lens, device="cuda", dtype=torch.int32)
    s.starts = torch.arange(0, (B + 1) * n, n, device="cuda", dtype=torch.int32)
    s.scale = 1.0 / math.sqrt(D)
    s.kp, s.vp = normal(pages, Hkv, page, D), normal(pages, Hkv, page, D)
    s.out = torch.empty((B * n, Hq, D), device="cuda", dtype=dt)
    if c["kind"] == "attend":
        s.q = normal(B, Hq, D, std=1.5)
        return s
    # a page's keys belong together (one patch, one sentence), and neighbouring queries look for similar things
    s.kp += normal(pages, Hkv, 1, D, std=0.7)
    rough = torch.randn((B, -(-n // 32) + 1, Hkv, 1, D), device="cuda", generator=g)
    f = torch.arange(n, device="cuda") / 32.0
    lo, w = f.long(), (f - f.floor())[None, :, None, None, None]
    base = rough[:, lo] * (1 - w) + rough[:, lo + 1] * w
    s.q = (base + 0.6 * torch.randn((B, n, Hkv, Hq // Hkv, D), device="cuda", generator=g)).reshape(B * n, Hq, D).to(dt)
    s.codes = torch.zeros((pages, Hkv, 2, D), device="cuda", dtype=torch.int8)
    s.scales = torch.zeros((pages, Hkv), device="cuda")
    every = torch.arange(pages, device="cuda", dtype=torch.int32)
    _summarize(s, every)  # what earlier steps left
    if c["fresh"]:  # the full pages that hold the chunk's keys
        new = [host[sum(need[:b]) + p] for b, v in enumerate(lens) for p in range((v - n) // page, v // page)]
        s.fresh = torch.tensor([int(p) for p in new], device="cuda", dtype=torch.int32)
        s.codes[s.fresh.long()] = 0
        s.scales[s.fresh.long()] = 0
    s.sel = torch.empty((B * n, Hkv, c["keep"]), device="cuda", dtype=torch.int32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2004_11250_gb300 import ppconv as pp
        s.pp, s.stream = pp, torch.cuda.current_stream()
        s.rope = s.cache = None
        if case["kind"] in ("rotate", "store"):
            s.rope = pp.pp_rope_create(case["D"], s.axis, s.freq, 3, case["interleaved"])
        if case["kind"] != "rotate":
            s.cache = pp.pp_cache_create(s.kp, s.vp, getattr(s, "codes", None), getattr(s, "scales", None))
        s.close = _Close(pp, s.rope, s.cache)
    return s


class _Close:
    """The program's own teardown."""

    def __init__(self, pp, rope, cache):
        self.pp, self.rope, self.cache = pp, rope, cache

    def __del__(self):
        torch.cuda.synchronize()
        if self.rope is not None:
            self.pp.pp_rope_destroy(self.rope)
        if self.cache is not None:
            self.pp.pp_cache_destroy(self.cache)


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    pp, c = s.pp, s.case
    if c["kind"] == "rotate":
        pp.pp_qk_rotate(s.rope, s.pos, EPS, s.q, s.qw, s.qo, s.k, s.kw, s.ko, s.stream)
        return {"q": s.qo, "k": s.ko}
    if c["kind"] == "store":
        pp.pp_qkv_store(s.rope, s.cache, s.pos, s.slots, EPS, s.q, s.qw, s.qo, s.k, s.kw, s.v, s.stream)
        return {"q": s.qo, "k": s.kp, "v": s.vp}
    if c["kind"] == "attend":
        pp.pp_attn_forward(s.cache, s.q, None, s.table, s.lens, s.scale, pp.PP_ATTN_CAUSAL, None, s.out, None, s.stream)
        return {"out": s.out}
    r = {}
    if c["fresh"]:
        pp.pp_cache_summarize(s.cache, s.fresh, s.stream)
        r["pages"] = s.codes * s.scales[:, :, None, None]
    starts = s.starts if c["n"] > 1 else None
    pp.pp_cache_select(s.cache, s.q, starts, s.table, s.lens, pp.PP_ATTN_CAUSAL, c["first"], c["last"], s.sel, s.stream)
    pp.pp_attn_forward(s.cache, s.q, starts, s.table, s.lens, s.scale, pp.PP_ATTN_CAUSAL, s.sel, s.out, None, s.stream)
    return {**r, "sel": s.sel, "out": s.out}


# ------------------------------------------------------------------ the plain form


def _rotated(s, x, w):
    c = s.case
    P = c["pairs"]
    y = x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w
    axis = torch.tensor(s.axis, device=x.device)
    angle = s.pos[axis].t().float() * torch.tensor(s.freq, device=x.device, dtype=torch.float32)
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if c["interleaved"]:
        a, b = y[..., 0: 2 * P: 2], y[..., 1: 2 * P: 2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :P], y[..., P: 2 * P]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., 2 * P:]], -1).to(x.dtype)


def _summarize(s, pages):
    k = s.kp[pages.long()].float()
    mx, mn = k.amax(2), k.amin(2)
    a = torch.maximum(mx.abs(), mn.abs()).amax(-1, keepdim=True)
    r = torch.full_like(a, 127.0) / a
    s.codes[pages.long()] = torch.stack([torch.ceil(mx * r).clamp(-127, 127), torch.floor(mn * r).clamp(-127, 127)], 2).to(torch.int8)
    s.scales[pages.long()] = a[..., 0] * (1.0 / 127.0)


def _select(s):
    c = s.case
    B, n, H, D, page, keep = c["B"], c["n"], c["Hkv"], c["D"], c["page"], c["keep"]
    G, W = c["Hq"] // H, s.table.shape[1]
    q = s.q.view(B, n, H, G, D).float()
    a = q.abs().amax((-1, -2), keepdim=True)
    most = float(min(127, 2 ** 24 // (127 * D * G)))
    code = torch.round(q * (torch.full_like(a, most) / a))
    code = torch.cat([code.clamp(min=0).sum(3), code.clamp(max=0).sum(3)], -1).transpose(1, 2)  # [B][H][n][2 D]
    t = s.table.long()
    score = torch.matmul(code, s.codes[t].float().permute(0, 2, 3, 4, 1).reshape(B, H, 2 * D, W))
    score = (score * s.scales[t].transpose(1, 2)[:, :, None]).transpose(1, 2)  # [B][n][H][W]
    seen = s.lens[:, None] - n + 1 + torch.arange(n, device=q.device)[None]  # visible keys of each token
    P = ((seen.clamp(min=0) + page - 1) // page)[:, :, None, None]
    w = torch.arange(W, device=q.device)
    score = torch.where((w < c["first"]) | (w >= P - c["last"]), math.inf, score)
    score = torch.where(w < P, score, -math.inf)
    most = min(keep, W)
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :most]
    best = torch.sort(torch.where(torch.arange(most, device=q.device) < P, best, W), dim=-1)[0]
    best = torch.where(best < W, best, -1).to(torch.int32)
    return torch.nn.functional.pad(best, (0, keep - most), value=-1).reshape(B * n, H, keep)


def _over_pages(s, sel):
    c = s.case
    B, n, H, D, page = c["B"], c["n"], c["Hkv"], c["D"], c["page"]
    G, W = c["Hq"] // H, s.table.shape[1]
    t = s.table.long()
    k = s.kp[t].float().transpose(1, 2).reshape(B, H, W * page, D)
    v = s.vp[t].float().transpose(1, 2).reshape(B, H, W * page, D)
    q = s.q.view(B, n, H, G, D).float().transpose(1, 2).reshape(B, H, n * G, D)
    score = torch.matmul(q, k.transpose(-1, -2)).view(B, H, n, G, W * page) * s.scale
    seen = s.lens[:, None] - n + 1 + torch.arange(n, device=q.device)[None]
    see = (torch.arange(W * page, device=q.device) < seen[..., None])[:, None]  # [B][1][n][keys]
    if sel is not None:
        on = torch.zeros((B, n, H, W + 1), device=q.device, dtype=torch.bool)
        at = sel.view(B, n, H, -1).long()
        on.scatter_(-1, torch.where(at < 0, W, at), True)
        see = see & on[..., :W].transpose(1, 2).repeat_interleave(page, -1)
    score = score.masked_fill(~see[:, :, :, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most > -math.inf, most, 0.0))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total > 0, total, 1.0)).view(B, H, n * G, W * page)
    o = torch.matmul(p, v)
    return o.view(B, H, n, G, D).transpose(1, 2).reshape(B * n, H * G, D).to(s.q.dtype)


def _plain(s):
    c = s.case
    if c["kind"] in ("rotate", "store"):
        q, k = _rotated(s, s.q, s.qw), _rotated(s, s.k, s.kw)
        if c["kind"] == "rotate":
            return {"q": q, "k": k}
        at = s.slots.long()
        s.kp[at // c["page"], :, at % c["page"]] = k
        s.vp[at // c["page"], :, at % c["page"]] = s.v
        return {"q": q, "k": s.kp, "v": s.vp}
    if c["kind"] == "attend":
        return {"out": _over_pages(s, None)}
    r = {}
    if c["fresh"]:
        _summarize(s, s.fresh)
        r["pages"] = s.codes * s.scales[:, :, None, None]
    sel = _select(s)
    return {**r, "sel": sel, "out": _over_pages(s, sel)}


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    e, D, Hq, Hkv = BYTES[c["dtype"]], c["D"], c["Hq"], c["Hkv"]
    if c["kind"] in ("rotate", "store"):
        heads = Hq + Hkv + (Hkv if c["kind"] == "store" else 0)
        return {"bytes": c["T"] * (2.0 * heads * D * e + 12 + (4 if c["kind"] == "store" else 0)), "flops": 10.0 * c["T"] * (Hq + Hkv) * D}
    T, page = c["B"] * c["n"], c["page"]
    io = 2.0 * T * Hq * D * e
    if c["kind"] == "attend":
        keys = sum(_lens(c))
        return {"bytes": io + 2.0 * keys * Hkv * D * e + 4.0 * -(-keys // page), "flops": 4.0 * keys * Hq * D}
    keys = pairs = scored = pages = 0
    for v in _lens(c):
        reach = 0
        for i in range(c["n"]):
            seen = max(0, v - c["n"] + i + 1)
            full = -(-seen // page)
            got = min(seen, c["keep"] * page - (full * page - seen if full > c["keep"] else 0))
            pairs += got
            scored += full
            reach += got
        keys += min(v, reach)  # each key that some token can select is read once
        pages += -(-v // page)
    made = c["n"] * c["B"] if c["fresh"] else 0
    size = io + 2.0 * keys * Hkv * D * e + pages * (Hkv * (2.0 * D + 4) + 4) + 4.0 * T * Hkv * c["keep"] + made * Hkv * D * (e + 2.0 / page)
    return {"bytes": size, "flops": 4.0 * pairs * Hq * D + 4.0 * scored * Hkv * D}


# ------------------------------------------------------------------ in 64 bits, apart from the plain form


def _exact_rows(s, x, w):
    c, P = s.case, s.case["pairs"]
    z = x.double()
    z = z / torch.sqrt((z * z).sum(-1, keepdim=True) / c["D"] + EPS) * w.double()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device),
                       torch.stack([s.pos[a].double() * f for a, f in zip(s.axis, s.freq)], 1))[:, None]
    out = z.clone()
    lo, hi = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if c["interleaved"] else (slice(0, P), slice(P, 2 * P))
    y = torch.complex(z[..., lo], z[..., hi]) * turn
    out[..., lo], out[..., hi] = y.real, y.imag
    return out


def _exact_page(s, p):
    """(codes as the values they stand for) of one page: the definition's own 32-bit steps."""
    k = s.kp[p].float()
    mx, mn = k.max(1)[0], k.min(1)[0]
    a = torch.stack([mx, -mn]).abs().amax((0, 2))[:, None]
    r = torch.full_like(a, 127.0) / a
    return torch.stack([(mx * r).ceil().clamp(-127, 127), (mn * r).floor().clamp(-127, 127)], 1), a[:, 0] * (1.0 / 127.0)


def exact(case, seed):
    """The operators' definitions in 64 bits, sequence by sequence.  Page summaries and selections are whole numbers
    whose definition is in 32 bits: they come out of its steps, the attention of 64-bit sums."""
    c = case
    s = _inputs(c, seed)
    D, page, H = c["D"], c["page"], c["Hkv"]
    G = c["Hq"] // H
    if c["kind"] in ("rotate", "store"):
        q, k = _exact_rows(s, s.q, s.qw), _exact_rows(s, s.k, s.kw)
        if c["kind"] == "rotate":
            return {"q": q, "k": k}
        kp, vp = s.kp.double(), s.vp.double()
        flat = s.slots.long()
        kp[flat // page, :, flat % page] = k
        vp[flat // page, :, flat % page] = s.v.double()
        return {"q": q, "k": kp, "v": vp}
    n, lens = c["n"], _lens(c)
    if c["B"] * n * c["Hq"] * c["L"] * D > 4e11:
        return None
    out = torch.zeros((c["B"] * n, c["Hq"], D), device="cuda", dtype=torch.float64)
    r = {}
    sel = None
    if c["kind"] == "sparse":
        if c["fresh"]:
            for p in s.fresh.tolist():
                s.codes[p], s.scales[p] = _exact_page(s, p)
            r["pages"] = s.codes.double() * s.scales.double()[:, :, None, None]
        sel = torch.full((c["B"] * n, H, c["keep"]), -1, device="cuda", dtype=torch.int32)
        top = min(127, 2 ** 24 // (127 * D * G))
    for b, v in enumerate(lens):
        if not v:
            continue
        ids = s.table[b, : -(-v // page)].long()
        for h in range(H):
            k = s.kp[ids, h].reshape(-1, D)[:v].double()
            u = s.vp[ids, h].reshape(-1, D)[:v].double()
            x = s.q[b * n: (b + 1) * n, h * G: (h + 1) * G]
            logits = torch.einsum("ngd,kd->ngk", x.double(), k) * s.scale
            seen = torch.arange(v - n + 1, v + 1, device="cuda")
            hide = torch.arange(v, device="cuda")[None] >= seen[:, None]
            if sel is not None:
                f = x.float()
                big = f.abs().amax((1, 2), keepdim=True)
                f = torch.round(f * (torch.full_like(big, float(top)) / big)).double()
                up, down = torch.relu(f).sum(1), -torch.relu(-f).sum(1)
                whole = up @ s.codes[ids, h, 0].double().T + down @ s.codes[ids, h, 1].double().T
                score = (whole.float() * s.scales[ids, h]).double()
                full = ((seen + page - 1) // page)[:, None]
                at = torch.arange(len(ids), device="cuda")[None]
                score[(at < c["first"]) | (at >= full - c["last"])] = 1e300
                score[(at >= full).expand_as(score)] = -1e300
                m = min(c["keep"], len(ids))
                # larger scores first, then lower pages: one stable ascending sort
                best = torch.argsort(-score, dim=1, stable=True)[:, :m]
                on = torch.zeros_like(score, dtype=torch.bool).scatter_(1, best, True) & (at < full)
                rank = torch.cumsum(on, 1) - 1
                row, col = torch.nonzero(on, as_tuple=True)
                sel[b * n + row, h, rank[row, col]] = col.to(torch.int32)
                hide = hide | ~on.repeat_interleave(page, 1)[:, :v]
            logits = logits.masked_fill(hide[:, None], -math.inf)
            out[b * n: (b + 1) * n, h * G: (h + 1) * G] = torch.einsum("ngk,kd->ngd", torch.softmax(logits, -1), u)
    return {**r, "sel": sel, "out": out} if sel is not None else {"out": out}
