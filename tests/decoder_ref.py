"""The decoder operators in 64 bits (and, for page summaries and selections, in the 32-bit steps that define them),
token by token in plain loops over CPU tensors: what the GPU tests compare with, and how far outputs may be off.

Tolerances, from the arithmetic (u: half a unit in the last place, relative: 2^-24 in fp32, 2^-11 in f16, 2^-8 in bf16;
products of two f16 or bf16 values are exact in fp32):
  rotation   the mean of D squares, its root, two products and the rotation in fp32: (D + 24) 2^-24 of |a| + |b| of the
             pair, one rounding to the type.
  attention  a logit errs by d = (D + 8) 2^-24 (plus 2^-20 for fp32 inputs, whose products the tensor cores sum as three
             tf32 ones) of scale sum |q k|; a weight by 2 d + 2^-20 relative; a weight may be rounded to the inputs' type
             before its product with v (u; fp32: 2^-20); n terms add n 2^-24.  Together times sum p |v|, plus one
             rounding to the type.
"""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}


def seen_keys(T, starts, lens, causal):
    """[(sequence, visible keys)] of every token."""
    out = []
    for b, n in enumerate(lens):
        s0, s1 = (starts[b], starts[b + 1]) if starts is not None else (b, b + 1)
        for i in range(s1 - s0):
            out.append((b, max(0, n - (s1 - s0) + i + 1) if causal else n))
    assert len(out) == T
    return out


def rotate(x, w, eps, pos, axis, freq, interleaved):
    """(result, tolerance) in float64 of x [T][H][D] before and after its rounding to x's type."""
    T, H, D = x.shape
    P = len(freq)
    z = x.double()
    if eps >= 0:
        z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
        if w is not None:
            z = z * w.double()
    y, mag = z.clone(), z.abs().clone()
    for j in range(P):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, P + j)
        # a turn's fraction with whole numbers, so that large positions stay exact
        ang = [math.fmod(int(p) * float(freq[j]), 2 * math.pi) for p in pos[axis[j]].tolist()]
        c = torch.tensor([math.cos(v) for v in ang], dtype=torch.float64)[:, None]
        s = torch.tensor([math.sin(v) for v in ang], dtype=torch.float64)[:, None]
        y[..., a] = z[..., a] * c - z[..., b] * s
        y[..., b] = z[..., b] * c + z[..., a] * s
        mag[..., a] = mag[..., b] = z[..., a].abs() + z[..., b].abs()
    tol = (D + 24) * 2.0 ** -24 * mag + UNIT[x.dtype] * y.abs() * 1.01 + TINY[x.dtype]
    return y, tol


def summarize(k):
    """(codes [pages][H][2][D], scales [pages][H]) of pools k [pages][H][page][D]: every step one fp32 operation."""
    f = k.float()
    mx, mn = f.amax(2), f.amin(2)
    a = torch.maximum(mx.abs(), mn.abs()).amax(-1)
    odd = ~torch.isfinite(f).all(-1).all(-1)
    zero = odd | ~(a >= 2.0 ** -100)
    r = torch.where(zero, torch.zeros_like(a), torch.full_like(a, 127.0) / torch.where(zero, torch.ones_like(a), a))
    up = torch.ceil(torch.nan_to_num(mx) * r[..., None]).clamp(max=127)
    down = torch.floor(torch.nan_to_num(mn) * r[..., None]).clamp(min=-127)
    codes = torch.stack([up, down], 2)
    codes[zero] = 0
    scales = a * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    scales = torch.where(odd, torch.full_like(a, math.nan), scales)
    return codes.to(torch.int8), scales


def select(q, codes, scales, table, starts, lens, causal, page, first, last, keep):
    """sel [T][H][keep] from the definition; whole numbers in Python's own."""
    T, Hq, D = q.shape
    pages, H = scales.shape
    G = Hq // H
    Q = min(127, 2 ** 24 // (127 * D * G))
    sel = torch.full((T, H, keep), -1, dtype=torch.int32)
    for t, (b, n) in enumerate(seen_keys(T, starts, lens, causal)):
        P = -(-n // page)
        for h in range(H):
            f = q[t, h * G: (h + 1) * G].float()
            a = f.abs().max()
            if torch.isfinite(f).all() and a >= 2.0 ** -100:
                c = torch.round(f * (torch.full_like(a, float(Q)) / a)).to(torch.int64)
            else:
                c = torch.zeros_like(f, dtype=torch.int64)
            up, down = c.clamp(min=0).sum(0), c.clamp(max=0).sum(0)
            rank = []
            for w in range(P):
                if w < first or w >= P - last:
                    v = math.inf
                else:
                    i = int(table[b, w])
                    v = -math.inf
                    if 0 <= i < pages:
                        dot = int((up * codes[i, h, 0].long()).sum() + (down * codes[i, h, 1].long()).sum())
                        v = float(torch.tensor(float(dot), dtype=torch.float32) * scales[i, h])
                        v = -math.inf if math.isnan(v) else v
                rank.append((-v, w))
            best = sorted(w for _, w in sorted(rank)[:keep])
            sel[t, h, : len(best)] = torch.tensor(best, dtype=torch.int32)
    return sel


def attend(q, k, v, table, starts, lens, scale, causal, sel=None):
    """(out, lse, tolerance of out, tolerance of lse) in float64."""
    T, Hq, D = q.shape
    pages, H, page, _ = k.shape
    G = Hq // H
    dt = q.dtype
    out = torch.zeros((T, Hq, D), dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    tol = torch.full((T, Hq, D), TINY[dt], dtype=torch.float64)
    tl = torch.zeros((T, Hq), dtype=torch.float64)
    wide = dt == torch.float32
    for t, (b, n) in enumerate(seen_keys(T, starts, lens, causal)):
        P = -(-n // page)
        for h in range(H):
            some = torch.arange(P) if sel is None else sel[t, h][(sel[t, h] >= 0) & (sel[t, h] < P)].long()
            key = (some[:, None] * page + torch.arange(page)).flatten()
            key = key[key < n]
            ip, io = table[b, key // page].long(), key % page
            good = (ip >= 0) & (ip < pages)
            ip, io = ip[good], io[good]
            if not len(ip):
                continue
            kk, vv = k[ip, h, io].double(), v[ip, h, io].double()
            x = q[t, h * G: (h + 1) * G].double()
            s = scale * (x @ kk.T)
            d = abs(scale) * (x.abs() @ kk.abs().T).amax(-1, keepdim=True) * ((D + 8) * 2.0 ** -24 + (2.0 ** -20 if wide else 0))
            p = torch.softmax(s, -1)
            o = p @ vv
            hs = slice(h * G, (h + 1) * G)
            rel = 2 * d + 2.0 ** -19 + len(ip) * 2.0 ** -24 + (2.0 ** -20 if wide else UNIT[dt])
            out[t, hs], lse[t, hs] = o, torch.logsumexp(s, -1)
            tol[t, hs] += rel * (p @ vv.abs()) + UNIT[dt] * o.abs() * 1.01
            tl[t, hs] = d[:, 0] + 2.0 ** -19 + len(ip) * 2.0 ** -24 + 2.0 ** -22 * lse[t, hs].abs()
    return out, lse, tol, tl


def worst(got, want, tol):
    """The largest error over its tolerance (0/0 is 0); infinities have to be equal."""
    got, want = got.double().cpu(), want.double()
    same = got == want
    r = torch.where(same, torch.zeros_like(want), (got - want).abs() / tol)
    return float(torch.nan_to_num(r, nan=math.inf).max()) if r.numel() else 0.0
