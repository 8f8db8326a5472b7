"""The cache in 8 bits and attention with a window by their definitions, over CPU tensors in plain loops: codes and scales in
the 32-bit steps that define them, attention in 64 bits.

Tolerances of attention (u: half a unit in the last place as in decoder_ref), from the arithmetic:
  a logit errs by d = (D + 12) 2^-24 of scale sum |q k| (sums of products in fp32, the page's and the row's scale); fp32
  queries over codes come as three f16 parts, which leave 2^-33 of each and 2^-39 of the row's largest, over fp32 keys as in
  decoder_ref (2^-20).
  a weight errs by 2 d + 2^-19 relative, by its rounding before its product with v (over codes f16's: 2^-11 of it; else u of
  the type; fp32 queries, which take two halves, and fp32 values: 2^-20), and over codes and in f16 by half a step of f16 where
  it has left the range that is normal: 2^-25 where the largest weight is 2^10 at the least (f16) or 2^8 (codes), times the
  largest scale, and twice that for two roundings: 2^-34 or 2^-32 max p max |v| for each key.
  n terms add n 2^-24.  Together times sum p |v|, plus one rounding to the type.
"""
import math

import torch

import decoder_ref as ref

TINY = 2.0 ** -100


def append(codes, scales, x, table, starts, lens, page):
    """One call's new tokens x [T][H][D] into codes [pages][H][page][D] and scales [pages][H], in place."""
    pages, H = scales.shape
    inv = torch.tensor(1.0 / 127.0, dtype=torch.float32)
    x = torch.where(torch.isfinite(x.float()), x.float(), 0.0)
    for b, v in enumerate(lens):
        s0, s1 = (starts[b], starts[b + 1]) if starts is not None else (b, b + 1)
        if v < 0 or v > table.shape[1] * page:
            continue
        n = s1 - s0
        for w in range(-(-v // page)):
            lo, hi = max(v - n, w * page, 0), min(v, (w + 1) * page)
            id = int(table[b, w]) if lo < hi else -1
            if not 0 <= id < pages:
                continue
            rows = x[s0 + lo - (v - n): s0 + hi - (v - n)].transpose(0, 1)  # [H][rows][D]
            at = lo - w * page
            for h in range(H):
                a = rows[h].abs().max()
                top = a * inv if float(a) >= TINY else torch.zeros(())
                had = scales[id, h].clone() if at else torch.zeros(())
                now = torch.maximum(had, top)
                if at and float(now) > float(had):
                    codes[id, h, :at] = torch.round(codes[id, h, :at].float() * (had / now)).clamp(-127, 127).to(torch.int8)
                r = torch.ones(()) / now if float(now) > 0 else torch.zeros(())
                codes[id, h, at: at + hi - lo] = torch.round(rows[h] * r).clamp(-127, 127).to(torch.int8)
                scales[id, h] = now


def read(codes, scales, table, starts, lens, page, dt):
    """[T][H][D] of type dt."""
    pages, H, _, D = codes.shape
    T = starts[-1] if starts is not None else len(lens)
    out = torch.zeros((T, H, D), dtype=dt)
    for t, (b, n) in enumerate(ref.seen_keys(T, starts, lens, True)):
        if n > 0:
            id = int(table[b, (n - 1) // page])
            if 0 <= id < pages:
                out[t] = (codes[id, :, (n - 1) % page].float() * scales[id][:, None]).to(dt)
    return out


def values(codes, scales):
    """What a pool's codes stand for, in 64 bits."""
    return codes.double() * scales.double()[:, :, None, None]


def attend(q, k, v, table, starts, lens, scale, causal, window, sinks, codes):
    """(out, lse, tolerance of out, tolerance of lse) in float64; k, v: pools of values; codes: they stood in 8 bits."""
    T, Hq, D = q.shape
    pages, H, page, _ = k.shape
    G, dt = Hq // H, q.dtype
    wide = dt == torch.float32
    u = 2.0 ** -20 if wide else ref.UNIT[torch.float16] if codes else ref.UNIT[dt]
    step = 2.0 ** -32 if codes else 2.0 ** -34 if dt == torch.float16 else 0.0
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    tol = torch.full((T, Hq, D), ref.TINY[dt], dtype=torch.float64)
    tl = torch.zeros((T, Hq), dtype=torch.float64)
    for t, (b, n) in enumerate(ref.seen_keys(T, starts, lens, causal)):
        key = torch.arange(n)
        key = key[(key >= n - window) | (key < sinks)]
        ip, io = table[b, key // page].long(), key % page
        good = (ip >= 0) & (ip < pages)
        ip, io = ip[good], io[good]
        if not len(ip):
            continue
        for h in range(H):
            kk, vv = k[ip, h, io].double(), v[ip, h, io].double()
            hs = slice(h * G, (h + 1) * G)
            x = q[t, hs].double()
            s = scale * (x @ kk.T)
            d = abs(scale) * (x.abs() @ kk.abs().T).amax(-1, keepdim=True) * ((D + 12) * 2.0 ** -24 + (2.0 ** -20 if wide and not codes else 0))
            if wide and codes:
                d = d + abs(scale) * 2.0 ** -33 * (x.abs() @ kk.abs().T + 2.0 ** -6 * x.abs().amax(-1, keepdim=True) * kk.abs().sum(-1)).amax(-1, keepdim=True)
            p = torch.softmax(s, -1)
            rel = 2 * d + 2.0 ** -19 + len(ip) * 2.0 ** -24 + u
            out[t, hs], lse[t, hs] = p @ vv, torch.logsumexp(s, -1)
            tol[t, hs] += rel * (p @ vv.abs()) + ref.UNIT[dt] * out[t, hs].abs() * 1.01
            tol[t, hs] += step * len(ip) * p.amax(-1, keepdim=True) * vv[torch.isfinite(vv)].abs().max()
            tl[t, hs] = d[:, 0] + 2.0 ** -19 + len(ip) * 2.0 ** -24 + 2.0 ** -22 * lse[t, hs].abs()
    return out, lse, tol, tl
