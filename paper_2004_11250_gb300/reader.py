"""A frame reader: a pruned trunk, and a small decoder that keeps what it has seen in a paged cache and answers.

The trunk (a ``synth.Net`` through ``runner.DeviceNet``) turns a frame into a map of C channels; every place of the map
is a token at position (frame, row, column).  A decoder layer projects its tokens, normalises and rotates queries and
keys into the cache (``pp_qkv_store``), summarises the pages that this filled (``pp_cache_summarize``), selects the
pages worth reading for each token (``pp_cache_select``) and attends to them (``pp_attn_forward``).  Answers continue
after the frames, a token at a time, on all three axes alike.  The projections are plain matrix products of torch;
weights are random, as there is no trained model here.

    python -m paper_2004_11250_gb300.reader --frames 32 --tokens 16
"""
from __future__ import annotations

import math
from typing import List, Optional

import torch

from . import ppconv as pp
from . import runner, synth


class Layer:
    """One decoder layer's weights and its cache: x + attention(x) Wo."""

    def __init__(self, width: int, Hq: int, H: int, D: int, pages: int, page: int, dtype, gen):
        def normal(*shape):
            return torch.randn(shape, device="cuda", generator=gen) / math.sqrt(shape[0])

        self.wqkv = normal(width, (Hq + 2 * H) * D).to(dtype)
        self.wo = (0.5 * normal(Hq * D, width)).to(dtype)
        self.qw = 1 + 0.1 * torch.randn(D, device="cuda", generator=gen)
        self.kw = 1 + 0.1 * torch.randn(D, device="cuda", generator=gen)
        self.k = torch.zeros((pages, H, page, D), device="cuda", dtype=dtype)
        self.v = torch.zeros_like(self.k)
        self.codes = torch.zeros((pages, H, 2, D), device="cuda", dtype=torch.int8)
        self.scales = torch.zeros((pages, H), device="cuda")
        self.cache = pp.pp_cache_create(self.k, self.v, self.codes, self.scales)


class FrameReader:
    """Reads frames and answers about them (one sequence).

    keep: pages that a token reads at most, the first and the last two among them; None: all, without a selection.
    """

    EPS = 1e-6

    def __init__(self, trunk: Optional[synth.Net] = None, layers: int = 2, Hq: int = 8, H: int = 2, D: int = 64,
                 page: int = 16, max_tokens: int = 4096, keep: Optional[int] = 16, dtype=torch.bfloat16, seed: int = 0):
        spec = trunk if trunk is not None else synth.cfg1_vgg16()
        self.net = runner.DeviceNet(spec)
        _, self.C, self.rows, self.cols = self.net.out_shape
        self.Hq, self.H, self.D, self.page, self.keep, self.dtype = Hq, H, D, page, keep, dtype
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        pages = -(-max_tokens // page)
        self.layers: List[Layer] = [Layer(self.C, Hq, H, D, pages, page, dtype, gen) for _ in range(layers)]
        # a quarter of the pairs follows the frame's number, the rest its rows and columns
        P = D // 2
        axis = [0] * (P // 4) + [1] * ((P - P // 4) // 2)
        axis += [2] * (P - len(axis))
        self.freq = [10000.0 ** (-j / P) for j in range(P)]
        self.axis = axis
        self.rope = pp.pp_rope_create(D, axis, self.freq, 3)
        self.table = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32)[None].contiguous()
        self.map = torch.empty(self.net.out_shape, device="cuda")
        self.seen = 0    # tokens in the cache
        self.frames = 0
        torch.cuda.synchronize()  # what was made here is ready for any stream

    def features(self, frame: torch.Tensor) -> torch.Tensor:
        """The tokens of a frame [1][3][H][W] on the GPU: [rows * cols][C], each of mean square 1."""
        self.net.run(frame, self.map)
        x = self.map.reshape(self.C, -1).t()
        return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + self.EPS)).to(self.dtype)

    def step(self, x: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        """The decoder over T new tokens x [T][C] at positions pos [3][T] (int32): its outputs [T][C]."""
        T, n = x.shape[0], self.seen
        if n + T > self.table.shape[1] * self.page:
            raise ValueError("the cache is full")
        s = torch.cuda.current_stream()
        at = torch.arange(n, n + T, device="cuda")
        slots = (self.table[0][at // self.page] * self.page + at % self.page).to(torch.int32)
        filled = self.table[0, n // self.page: (n + T) // self.page].contiguous()
        lens = torch.full((1,), n + T, device="cuda", dtype=torch.int32)
        starts = None if T == 1 else torch.tensor([0, T], dtype=torch.int32).cuda()
        sel = None if self.keep is None else torch.empty((T, self.H, self.keep), device="cuda", dtype=torch.int32)
        q = torch.empty((T, self.Hq, self.D), device="cuda", dtype=self.dtype)
        out = torch.empty_like(q)
        for L in self.layers:
            fused = x @ L.wqkv
            heads = fused.view(T, self.Hq + 2 * self.H, self.D)
            new_q, new_k, new_v = heads[:, : self.Hq], heads[:, self.Hq: self.Hq + self.H], heads[:, self.Hq + self.H:]
            pp.pp_qkv_store(self.rope, L.cache, pos, slots, self.EPS, new_q, L.qw, q, new_k, L.kw, new_v, s)
            if sel is not None:
                pp.pp_cache_summarize(L.cache, filled, s)
                pp.pp_cache_select(L.cache, q, starts, self.table, lens, pp.PP_ATTN_CAUSAL, 1, 2, sel, s)
            pp.pp_attn_forward(L.cache, q, starts, self.table, lens, 1 / math.sqrt(self.D), pp.PP_ATTN_CAUSAL, sel, out, None, s)
            x = x + out.view(T, -1) @ L.wo
        self.seen = n + T
        return x

    def watch(self, frame: torch.Tensor) -> torch.Tensor:
        """Takes a frame in: the decoder's outputs for its tokens."""
        i = torch.arange(self.rows * self.cols, device="cuda", dtype=torch.int32)
        pos = torch.stack([torch.full_like(i, self.frames), i // self.cols, i % self.cols])
        y = self.step(self.features(frame), pos)
        self.frames += 1
        return y

    def answer(self, tokens: int, start: Optional[torch.Tensor] = None) -> torch.Tensor:
        """`tokens` outputs [tokens][C], each the next one's input; start [1][C]: the first input (default: ones)."""
        x = torch.ones((1, self.C), device="cuda", dtype=self.dtype) if start is None else start
        got = []
        for i in range(tokens):
            at = max(self.frames, self.rows, self.cols) + i  # beyond every position of the frames
            x = self.step(x, torch.full((3, 1), at, device="cuda", dtype=torch.int32))
            got.append(x)
        return torch.cat(got) if got else x[:0]

    def status(self) -> int:
        """What the calls on the layers' caches met (PP_CACHE_* bits; synchronous)."""
        bits = 0
        for L in self.layers:
            bits |= pp.pp_cache_device_status(L.cache)
        return bits

    def close(self):
        torch.cuda.synchronize()
        for L in self.layers:
            pp.pp_cache_destroy(L.cache)
        self.layers = []
        if self.rope is not None:
            pp.pp_rope_destroy(self.rope)
            self.rope = None
        self.net.close()


def main(argv=None):
    import argparse
    a = argparse.ArgumentParser(description="read synthetic frames with a pruned VGG-16 trunk and answer about them")
    a.add_argument("--frames", type=int, default=32)
    a.add_argument("--tokens", type=int, default=16)
    a.add_argument("--keep", type=int, default=16, help="pages that a token reads at most; 0: all")
    o = a.parse_args(argv)
    if o.frames < 1 or o.tokens < 0 or not (o.keep == 0 or o.keep >= 3):
        a.error("at least 1 frame, 0 tokens, and 3 pages (the first and the last two)")
    r = FrameReader(max_tokens=196 * o.frames + o.tokens, keep=o.keep or None)  # maps of 14 x 14
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    with torch.cuda.stream(torch.cuda.Stream()):
        r.watch(torch.rand((1, 3, 224, 224), device="cuda", generator=gen))
        ev[0].record()
        for _ in range(o.frames - 1):
            r.watch(torch.rand((1, 3, 224, 224), device="cuda", generator=gen))
        ev[1].record()
        y = r.answer(o.tokens)
        ev[2].record()
        torch.cuda.current_stream().synchronize()
    answer = "" if not o.tokens else (f", {ev[1].elapsed_time(ev[2]) / o.tokens:.3f} ms an answer token, "
                                      f"mean |output| {float(y.float().abs().mean()):.4f}")
    print(f"{r.frames} frames, {r.seen} tokens in the cache: {ev[0].elapsed_time(ev[1]) / max(1, o.frames - 1):.3f} ms a frame{answer}, "
          f"status {r.status()}")
    r.close()


if __name__ == "__main__":
    main()
