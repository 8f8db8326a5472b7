"""What is measured: a cache of keys and values held in 8 bits, and attention with a sliding window, behind a vision trunk.

A program that watches long videos keeps many sequences' keys and values.  In 8 bits, with a scale for each page and head,
twice as many fit and a step reads half the bytes; with a window and a few first tokens that stay visible, what a step
reads does not grow with the video.  A case is one step of such a program on one of its layers.

Kinds of cases (``"kind"``):
  append   n new tokens of each of B sequences quantised into their pages (``pp_cache_append``), and all sequences read
           back (``pp_cache_read``), as a program does that hands them on.
  read     B sequences of up to L tokens read back (``pp_cache_read``).
  attend   n new tokens of each of B sequences over the keys of an 8-bit cache (``pp_attn_forward``).
  window   the same with a window of ``window`` keys and ``sinks`` first ones (``pp_attn_window``), over a cache of
           ``bits`` 8, or of the tokens' own type (0).

A page's scale of one head is a 127th of the largest value written since its first token; codes are whole numbers.  Layouts:
pools [pages][H][page][D], scales [pages][H]; queries and values are views of one fused [T][(Hq + 2 H) D] product, keys come
rotated and dense; outputs [T][heads][D].  ``ragged`` spreads the lengths from an idle slot (0) to L.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _case(name, kind, dtype, B, n, L, Hq, H, D, page, ragged=False, window=0, sinks=0, bits=8):
    c = dict(kind=kind, dtype=dtype, B=B, n=n, L=L, Hq=Hq, H=H, D=D, page=page, ragged=ragged, window=window, sinks=sinks, bits=bits)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The next token of one answer, a small decoder: latency decides.
        _case("append_1x777_bf16", "append", "bf16", 1, 1, 777, 8, 2, 128, 16),
        # One step of 64 short answers at once, most into pages begun before.
        _case("append_64x512_bf16", "append", "bf16", 64, 1, 512, 32, 8, 128, 64, True),
        # Odd chunks of three prompts in the library's own fp32, heads of 96.
        _case("append_3x333_f32", "append", "f32", 3, 333, 1001, 8, 4, 96, 32),
        # A long prompt.
        _case("append_16384_f16", "append", "f16", 1, 16384, 16384, 32, 8, 128, 64),
        # Eight sequences handed to a program that holds 16 bits.
        _case("read_8x8192_bf16", "read", "bf16", 8, 1, 8192, 32, 8, 128, 64),
        # One short answer over 777 cached tokens: latency again.
        _case("attend_1x777_bf16", "attend", "bf16", 1, 1, 777, 8, 2, 128, 16),
        # A server's batch: 48 sequences from idle to 8192 tokens.
        _case("attend_48x8192_bf16", "attend", "bf16", 48, 1, 8192, 32, 8, 128, 64, True),
        # Long videos: 8 sequences of 65536 tokens.
        _case("attend_8x65536_f16", "attend", "f16", 8, 1, 65536, 32, 8, 128, 64),
        # A chunk of 2048 tokens behind a long cache.
        _case("attend_2048x32768_bf16", "attend", "bf16", 1, 2048, 32768, 32, 8, 128, 64),
        # fp32 decoder, heads of 96, a window that most of the sequences have outgrown.
        _case("window_16x2500_f32", "window", "f32", 16, 1, 2500, 8, 4, 96, 16, True, 1000, 4),
        # 32 endless videos: 4096 keys and 16 first ones of each, the cache in 16 bits.
        _case("window_32x32768_bf16", "window", "bf16", 32, 1, 32768, 32, 8, 128, 64, False, 4096, 16, 0),
        # A chunk of frames of one of them.
        _case("window_2048x32768_f16", "window", "f16", 1, 2048, 32768, 32, 8, 128, 64, False, 4096, 64, 0),
    ]


# ------------------------------------------------------------------ drawn cases


def _log(rng: random.Random, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 6.8e12 + w["flops"] / 1.8e15


def _fits(c):
    """No drawn case costs more than the largest listed one of its kind, or needs more memory in its plain form."""
    B, n, L = c["B"], c["n"], c["L"]
    return (n <= L and _cost(c) <= max(_cost(x) for x in listed() if x["kind"] == c["kind"])
            and B * L * c["H"] * c["D"] <= 8 * 65536 * 8 * 128 and B * n * c["Hq"] * L <= 2048 * 32 * 32768)


def draw(rng: random.Random):
    """1 .. 16384 new tokens of 1 .. 128 sequences, 1 .. 131072 cached ones; attention for single tokens of 1 .. 128
    sequences, for 2 .. 8 tokens of some (drafts of an answer), and for chunks of up to 2048 in 16 bits; heads of 64 .. 128
    (single tokens also 256), groups of 1 .. 8, pages of 16 .. 128, windows of 1 .. 8192 keys with 0 .. 128 first ones."""
    while True:
        kind = rng.choice(["append", "append", "read", "attend", "attend", "window", "window"])
        H = rng.choice([1, 2, 4, 8])
        Hq = H * rng.choice([1, 2, 3, 4, 8])
        D = rng.choice([64, 80, 96, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        page = rng.choice([16, 32, 64, 128])
        if kind == "read":
            c = _case(None, kind, dtype, _log(rng, 1, 64), 1, _log(rng, 1, 65536), Hq, H, D, page, rng.random() < 0.5)
        elif kind == "append":
            if rng.random() < 0.5:
                B, n, ragged = _log(rng, 1, 128), 1, rng.random() < 0.5
            else:
                B, n, ragged = rng.choice([1, 1, 2, 3, 8]), _log(rng, 2, 16384), False
            c = _case(None, kind, dtype, B, n, n + _log(rng, 1, 2048) - 1, Hq, H, D, page, ragged)
        else:
            ragged = False
            way = rng.choice(["single", "single", "draft", "chunk"])
            if way == "single":
                if rng.random() < 0.15:
                    D = 256
                B, n, ragged = _log(rng, 1, 128), 1, rng.random() < 0.5
            elif way == "draft":
                B, n = _log(rng, 1, 32), rng.randint(2, 8)
            else:
                B, n, dtype = rng.choice([1, 1, 2, 3]), _log(rng, 16, 2048), rng.choice(["bf16", "f16"])
            window, sinks, bits = 0, 0, 8
            if kind == "window":
                window, sinks, bits = _log(rng, 1, 8192), rng.choice([0, 1, 4, 16, 64, rng.randint(0, 128)]), rng.choice([0, 8])
            c = _case(None, kind, dtype, B, n, _log(rng, max(n, 16), 131072), Hq, H, D, page, ragged, window, sinks, bits)
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


class _State:
    pass


def _inputs(c, seed):
    s = _State()
    s.case = c
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPE[c["dtype"]]
    B, n, Hq, H, D, page = c["B"], c["n"], c["Hq"], c["H"], c["D"], c["page"]
    lens = _lens(c)
    need = [-(-v // page) for v in lens]
    W = max(max(need), 1)
    pages = sum(need) + 1
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.zeros((B, W), dtype=torch.int32)
    at, host = 0, order.cpu()
    for b, w in enumerate(need):
        table[b, :w] = host[at: at + w]
        at += w
    s.spare = int(host[at])  # a page that no sequence has
    s.table = table.cuda()
    s.lens = torch.tensor(lens, device="cuda", dtype=torch.int32)
    s.starts = torch.arange(0, (B + 1) * n, n, device="cuda", dtype=torch.int32)
    s.scale = 1.0 / math.sqrt(D)

    # what earlier steps left: pages of keys and of values, of somewhat different sizes from page to page
    def pool(std):
        full = torch.empty((pages, H, page, D), device="cuda", dtype=dt if c["bits"] == 0 else torch.int8)
        scales = torch.empty((pages, H), device="cuda")
        step = max(1, (1 << 28) // (H * page * D))
        for i in range(0, pages, step):
            m = min(step, pages - i)
            x = torch.randn((m, H, page, D), device="cuda", generator=g)
            x *= std * (0.6 + 0.8 * torch.rand((m, H, 1, 1), device="cuda", generator=g))
            if c["bits"] == 0:
                full[i: i + m] = x
            else:
                scales[i: i + m] = x.abs().amax((2, 3)) * (1.0 / 127.0)
                full[i: i + m] = torch.round(x / scales[i: i + m, :, None, None]).clamp(-127, 127)
        return full, scales

    s.k, s.ks = pool(1.0)
    s.v, s.vs = pool(0.5)
    if c["kind"] in ("append", "read"):
        total = sum(lens)
        s.ends = torch.tensor([sum(lens[:b]) for b in range(B + 1)], device="cuda", dtype=torch.int32)
        s.ko = torch.empty((total, H, D), device="cuda", dtype=dt)
        s.vo = torch.empty((total, H, D), device="cuda", dtype=dt)
    if c["kind"] == "append":
        s.new_k = torch.randn((B * n, H, D), device="cuda", generator=g).to(dt)
        fused = (0.5 * torch.randn((B * n, (Hq + 2 * H) * D), device="cuda", generator=g)).to(dt)
        s.new_v = fused[:, (Hq + H) * D:].view(B * n, H, D)
    elif c["kind"] != "read":
        s.q = (1.5 * torch.randn((B * n, (Hq + 2 * H) * D), device="cuda", generator=g)).to(dt)[:, : Hq * D].view(B * n, Hq, D)
        s.out = torch.empty((B * n, Hq, D), device="cuda", dtype=dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2004_11250_gb300 import ppconv as pp
        s.pp, s.stream = pp, torch.cuda.current_stream()
        s.cache = pp.pp_cache_create(s.k, s.v) if case["bits"] == 0 else pp.pp_cache8_create(s.k, s.v, s.ks, s.vs, DTYPE[case["dtype"]])
        s.close = _Close(pp, s.cache)
    return s


class _Close:
    """The program's own teardown."""

    def __init__(self, pp, cache):
        self.pp, self.cache = pp, cache

    def __del__(self):
        torch.cuda.synchronize()
        self.pp.pp_cache_destroy(self.cache)


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ the framework's calls


def _own(s):
    pp, c = s.pp, s.case
    starts = s.starts if c["n"] > 1 else None
    if c["kind"] == "append":
        pp.pp_cache_append(s.cache, s.new_k, s.new_v, starts, s.table, s.lens, s.stream)
    if c["kind"] in ("append", "read"):
        pp.pp_cache_read(s.cache, s.ends, s.table, s.lens, s.ko, s.vo, s.stream)
        return {"k": s.ko, "v": s.vo}
    if c["kind"] == "attend":
        pp.pp_attn_forward(s.cache, s.q, starts, s.table, s.lens, s.scale, pp.PP_ATTN_CAUSAL, None, s.out, None, s.stream)
    else:
        pp.pp_attn_window(s.cache, s.q, starts, s.table, s.lens, s.scale, pp.PP_ATTN_CAUSAL, c["window"], c["sinks"], s.out, None,
                          s.stream)
    return {"out": s.out}


# ------------------------------------------------------------------ the plain form


def _append(s, codes, scales, x):
    """New tokens x into a pool: the largest value of each page's new ones, the page's scale, its older codes, its new ones."""
    c = s.case
    B, n, H, page = c["B"], c["n"], c["H"], c["page"]
    at = (s.lens.long()[:, None] - n + torch.arange(n, device=x.device)[None]).reshape(-1)
    b = torch.arange(B, device=x.device).repeat_interleave(n)
    p = torch.where(at >= 0, s.table[b, at.clamp(min=0) // page].long(), s.spare)  # an idle slot's token goes nowhere
    o = at.clamp(min=0) % page
    x = x.float()
    top = torch.zeros_like(scales).scatter_reduce(0, p[:, None].expand(-1, H), x.abs().amax(-1), "amax")
    top = torch.where(top >= 2.0 ** -100, top, 0.0)
    first = torch.full_like(scales[:, 0], page).scatter_reduce(0, p, o.float(), "amin")[:, None]
    old = torch.where(first == 0, 0.0, scales)
    new = torch.where(first < page, torch.maximum(old, top * (1.0 / 127.0)), scales)
    f = torch.where((first < page) & (new > 0), old / new, 1.0)
    older = torch.arange(page, device=x.device) < first
    codes.copy_(torch.where(older[:, None, :, None], torch.round(codes.float() * f[:, :, None, None]), codes.float()))
    r = torch.where(new > 0, torch.ones_like(new) / new, 0.0)
    codes[p, :, o] = torch.round(x * r[p][:, :, None]).clamp(-127, 127).to(torch.int8)
    scales.copy_(new)


def _read(s, codes, scales):
    c = s.case
    t = torch.arange(s.ko.shape[0], device=codes.device, dtype=torch.int32)
    b = torch.bucketize(t, s.ends[1:], right=True)
    at = (t - s.ends[b]).long()
    p = s.table[b, at // c["page"]].long()
    return (codes[p, :, at % c["page"]].float() * scales[p][:, :, None]).to(DTYPE[c["dtype"]])


def _attend(s):
    c = s.case
    B, n, H, D, page = c["B"], c["n"], c["H"], c["D"], c["page"]
    G, W = c["Hq"] // H, s.table.shape[1]
    t = s.table.long()
    k, v = s.k[t].float(), s.v[t].float()
    if c["bits"]:
        k, v = k * s.ks[t][:, :, :, None, None], v * s.vs[t][:, :, :, None, None]
    k, v = k.transpose(1, 2).reshape(B, H, W * page, D), v.transpose(1, 2).reshape(B, H, W * page, D)
    q = s.q.view(B, n, H, G, D).float().transpose(1, 2).reshape(B, H, n * G, D)
    score = torch.matmul(q, k.transpose(-1, -2)).view(B, H, n, G, W * page) * s.scale
    seen = (s.lens[:, None] - n + 1 + torch.arange(n, device=q.device)[None])[:, None, :, None, None]
    at = torch.arange(W * page, device=q.device)
    see = at < seen
    if c["window"]:
        see = see & ((at >= seen - c["window"]) | (at < c["sinks"]))
    score = score.masked_fill(~see, -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(most > -math.inf, most, 0.0))
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total > 0, total, 1.0)).view(B, H, n * G, W * page)
    o = torch.matmul(p, v)
    return o.view(B, H, n, G, D).transpose(1, 2).reshape(B * n, H * G, D).to(s.q.dtype)


def _plain(s):
    c = s.case
    if c["kind"] == "append":
        _append(s, s.k, s.ks, s.new_k)
        _append(s, s.v, s.vs, s.new_v)
    if c["kind"] in ("append", "read"):
        return {"k": _read(s, s.k, s.ks), "v": _read(s, s.v, s.vs)}
    return {"out": _attend(s)}


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    e, D, Hq, H, n, page = BYTES[c["dtype"]], c["D"], c["Hq"], c["H"], c["n"], c["page"]
    lens = _lens(c)
    held = sum(lens)
    used = sum(-(-v // page) for v in lens)
    if c["kind"] in ("append", "read"):
        new = sum(min(v, n) for v in lens) if c["kind"] == "append" else 0
        size = 2.0 * H * D * (new * (e + 1.0) + held * (e + 1.0)) + used * (8.0 * H + 4.0) + 4.0 * c["B"]
        return {"bytes": size, "flops": 2.0 * H * D * (3.0 * new + held)}
    w, k = c["window"], c["sinks"]
    keys = pairs = pages = 0
    for v in lens:
        low = max(0, v - n + 1 - w) if w else 0  # the first key that some token's window has
        keys += v - low + min(k, low)
        pages += -(-v // page) - low // page + -(-min(k, low) // page)
        if not w:
            pairs += sum(max(0, v - n + i + 1) for i in range(n))
        else:
            for i in range(n):
                seen = max(0, v - n + i + 1)
                pairs += min(seen, w) + min(k, max(0, seen - w))
    size = 2.0 * c["B"] * n * Hq * D * e + 2.0 * keys * H * D * (1 if c["bits"] else e) + pages * (4.0 + (8.0 * H if c["bits"] else 0))
    return {"bytes": size, "flops": 4.0 * pairs * Hq * D}


# ------------------------------------------------------------------ in 64 bits, apart from the plain form


def _exact_append(c, lens, table, codes, scales, x):
    """Page by page.  Codes and scales are defined by 32-bit steps, which come here as numpy's."""
    import numpy as np
    x = x.float().cpu().numpy()
    table = table.cpu().numpy()
    for b, v in enumerate(lens):
        lo = v - c["n"]
        for w in range(max(0, lo) // c["page"], -(-v // c["page"]) if v else 0):
            p, from_, to = int(table[b, w]), max(lo, w * c["page"]), min(v, (w + 1) * c["page"])
            rows = x[b * c["n"] + from_ - lo: b * c["n"] + to - lo].transpose(1, 0, 2)  # [H][rows][D]
            a = np.abs(rows).max((1, 2))
            a[a < 2.0 ** -100] = 0
            at = from_ - w * c["page"]
            had = scales[p].cpu().numpy() if at else np.zeros_like(a)
            now = np.maximum(had, a * np.float32(1.0 / 127.0))
            inv = np.divide(np.float32(1), now, out=np.zeros_like(now), where=now > 0)
            if at:
                f = np.divide(had, now, out=np.ones_like(now), where=now > 0)
                if (f != 1).any():
                    was = codes[p, :, :at].cpu().numpy().astype(np.float32)
                    codes[p, :, :at] = torch.from_numpy(np.rint(was * f[:, None, None]).astype(np.int8)).to(codes.device)
            new = np.clip(np.rint(rows * inv[:, None, None]), -127, 127).astype(np.int8)
            codes[p, :, at: at + to - from_] = torch.from_numpy(new).to(codes.device)
            scales[p] = torch.from_numpy(now).to(scales.device)


def exact(case, seed):
    """The operators' definitions in 64 bits, sequence by sequence."""
    c = case
    s = _inputs(c, seed)
    n, lens, page, H, D = c["n"], _lens(c), c["page"], c["H"], c["D"]
    G = c["Hq"] // H
    if c["kind"] in ("append", "read"):
        if c["kind"] == "append":
            _exact_append(c, lens, s.table, s.k, s.ks, s.new_k)
            _exact_append(c, lens, s.table, s.v, s.vs, s.new_v)

        def back(codes, scales):
            got = []
            for b, v in enumerate(lens):
                ids = s.table[b, : -(-v // page)].long()
                x = codes[ids].double() * scales[ids].double()[:, :, None, None]
                got.append(x.transpose(1, 2).reshape(-1, H, D)[:v])
            return torch.cat(got)

        return {"k": back(s.k, s.ks), "v": back(s.v, s.vs)}
    if c["B"] * n * c["Hq"] * c["L"] * D > 4e11:
        return None
    out = torch.zeros((c["B"] * n, c["Hq"], D), device="cuda", dtype=torch.float64)
    for b, v in enumerate(lens):
        if not v:
            continue
        ids = s.table[b, : -(-v // page)].long()
        seen = torch.arange(v - n + 1, v + 1, device="cuda")[:, None]
        at = torch.arange(v, device="cuda")[None]
        if c["window"] and n == 1:  # one token: its keys alone
            low = max(0, v - c["window"])
            at = torch.cat([at[:, : min(c["sinks"], low)], at[:, low:]], 1)
        hide = at >= seen
        if c["window"]:
            hide = hide | ((at < seen - c["window"]) & (at >= c["sinks"]))
        for h in range(H):
            k, u = s.k[ids, h], s.v[ids, h]
            k, u = k.reshape(-1, D)[at[0]].double(), u.reshape(-1, D)[at[0]].double()
            if c["bits"]:
                k = k * s.ks[ids, h].double().repeat_interleave(page)[at[0]][:, None]
                u = u * s.vs[ids, h].double().repeat_interleave(page)[at[0]][:, None]
            x = s.q[b * n: (b + 1) * n, h * G: (h + 1) * G].double()
            for i in range(G):
                logits = (x[:, i] @ k.T * s.scale).masked_fill(hide, -math.inf)
                out[b * n: (b + 1) * n, h * G + i] = torch.softmax(logits, -1) @ u
    return {"out": out}
