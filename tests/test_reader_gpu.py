"""The frame reader, which runs trunk, rotations, cache, selection and attention together: its decoder against plain
matrix products in 64 bits on the trunk's own features, and its selection at work."""
import math

import numpy as np
import pytest
import torch

from paper_2004_11250_gb300 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def reader():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import reader
    return reader


def small_trunk():
    rng = np.random.default_rng(5)
    ops = [synth.Op(synth.small_random_layer(rng, 32, 3, keep=1.0), relu=True, pool=True),
           synth.Op(synth.small_random_layer(rng, 64, 32, keep=0.5), relu=True, pool=True)]
    return synth.Net("small", rng.uniform(0, 1, (1, 3, 20, 28)).astype(np.float32), ops)


def decoder64(r, x, pos):
    """All tokens at once in 64 bits: x [T][C] the decoder's inputs, pos [3][T]."""
    T, G = x.shape[0], r.Hq // r.H
    x = x.double().cpu()
    turn = torch.stack([pos[a].double().cpu() * f for a, f in zip(r.axis, r.freq)], 1)
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]

    def rotated(v, w):
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + r.EPS) * w.double().cpu()
        z = torch.complex(v[..., : r.D // 2], v[..., r.D // 2:]) * turn
        return torch.cat([z.real, z.imag], -1)

    outs = []
    for L in r.layers:
        heads = (x @ L.wqkv.double().cpu()).view(T, r.Hq + 2 * r.H, r.D)
        q, k = rotated(heads[:, : r.Hq], L.qw), rotated(heads[:, r.Hq: r.Hq + r.H], L.kw)
        v = heads[:, r.Hq + r.H:]
        s = torch.einsum("thgd,shd->hgts", q.view(T, r.H, G, r.D), k) / math.sqrt(r.D)
        s = s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -math.inf)
        x = x + torch.einsum("hgts,shd->thgd", torch.softmax(s, -1), v).reshape(T, -1) @ L.wo.double().cpu()
        outs.append(x)
    return outs[-1]


@pytest.mark.parametrize("keep", [None, 32])
def test_reader_matches_64_bits(reader, keep):
    """fp32, all pages read (35 tokens a frame, pages of 16: 12 pages): within 1e-4 of the largest output, ten times what
    two layers of fp32 products of up to 256 terms (2^-24 each, summed) can add up to."""
    r = reader.FrameReader(small_trunk(), keep=keep, dtype=torch.float32, max_tokens=256)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        frames = [torch.rand((1, 3, 20, 28), device="cuda", generator=g) for _ in range(5)]
        feats = [r.features(f).clone() for f in frames]
        got = torch.cat([r.watch(f) for f in frames])
        n = r.rows * r.cols
        assert r.seen == 5 * n
        i = torch.arange(5 * n)
        pos = torch.stack([i // n, i % n // r.cols, i % r.cols])
        want = decoder64(r, torch.cat(feats), pos)
        assert float((got.double().cpu() - want).abs().max() / want.abs().max()) < 1e-4
        # an answer goes on after the frames: its inputs are its own outputs
        ans = r.answer(3)
        x = torch.cat([torch.cat(feats), torch.ones((1, r.C), device="cuda"), ans[:2]])
        at = max(5, r.rows, r.cols)
        pos = torch.cat([pos, torch.tensor([[at, at + 1, at + 2]] * 3)], 1)
        want = decoder64(r, x, pos)[-3:]
        assert float((ans.double().cpu() - want).abs().max() / want.abs().max()) < 1e-4
        assert r.status() == 0
    finally:
        r.close()


def test_reader_selects(reader):
    """More pages than a token reads: other outputs than with all of them, the same again on the same frames."""
    def run(keep):
        r = reader.FrameReader(small_trunk(), keep=keep, max_tokens=1024)
        try:
            g = torch.Generator(device="cuda")
            g.manual_seed(4)
            for _ in range(20):
                r.watch(torch.rand((1, 3, 20, 28), device="cuda", generator=g))
            y = r.answer(4)
            assert torch.isfinite(y).all() and r.status() == 0
            return y
        finally:
            r.close()

    few, again, all_of_them = run(4), run(4), run(None)
    assert torch.equal(few, again)
    assert not torch.equal(few, all_of_them)


def test_reader_command(reader, capsys):
    reader.main(["--frames", "3", "--tokens", "2"])
    assert "3 frames, 590 tokens in the cache" in capsys.readouterr().out
