"""The frame reader with a window and with a cache in 8 bits: against plain products in 64 bits, with pages used again."""
import math

import pytest
import torch

from test_reader_gpu import small_trunk


@pytest.fixture(scope="module")
def reader():
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import reader
    return reader


def decoder64(r, x, pos):
    """All tokens at once in 64 bits, each reading the last r.window tokens and the first r.sinks."""
    T, G = x.shape[0], r.Hq // r.H
    x = x.double().cpu()
    turn = torch.stack([pos[a].double() * f for a, f in zip(r.axis, r.freq)], 1)
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]
    i, j = torch.arange(T)[:, None], torch.arange(T)[None]
    hide = j > i
    if r.window is not None:
        hide = hide | ((j <= i - r.window) & (j >= r.sinks))

    def rotated(v, w):
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + r.EPS) * w.double().cpu()
        z = torch.complex(v[..., : r.D // 2], v[..., r.D // 2:]) * turn
        return torch.cat([z.real, z.imag], -1)

    for L in r.layers:
        heads = (x @ L.wqkv.double().cpu()).view(T, r.Hq + 2 * r.H, r.D)
        q, k, v = rotated(heads[:, : r.Hq], L.qw), rotated(heads[:, r.Hq: r.Hq + r.H], L.kw), heads[:, r.Hq + r.H:]
        s = torch.einsum("thgd,shd->hgts", q.view(T, r.H, G, r.D), k) / math.sqrt(r.D)
        p = torch.softmax(s.masked_fill(hide, -math.inf), -1)
        x = x + torch.einsum("hgts,shd->thgd", p, v).reshape(T, -1) @ L.wo.double().cpu()
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("bits,window,sinks", [(16, 50, 3), (16, 20, 0), (8, None, 0), (8, 50, 3), (16, 1000, 5)])
def test_reader_matches_64_bits(reader, bits, window, sinks):
    """fp32: within 1e-4 of the largest output, as without a window.  In 8 bits a key or value is within a step of its page's scale
    (half for its own rounding, half for growths of the scale), 1/127 of the page's largest, so scores of |q| = |k| = 1 a head
    err by some 1/127 / 2 and outputs of two layers by a few of them: 0.1 of the largest."""
    r = reader.FrameReader(small_trunk(), keep=None, dtype=torch.float32, max_tokens=512, bits=bits, window=window, sinks=sinks)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        frames = [torch.rand((1, 3, 20, 28), device="cuda", generator=g) for _ in range(9)]
        feats = [r.features(f).clone() for f in frames]
        got = torch.cat([r.watch(f) for f in frames])
        n = r.rows * r.cols
        held = r.layers[0].k.shape[0] * r.page
        assert r.seen == 9 * n and (held < r.seen if window is not None and window < 100 else held >= r.seen)
        ans = r.answer(3)
        i, at = torch.arange(9 * n), max(9, r.rows, r.cols)
        pos = torch.cat([torch.stack([i // n, i % n // r.cols, i % r.cols]), torch.tensor([[at, at + 1, at + 2]] * 3)], 1)
        want = decoder64(r, torch.cat(feats + [torch.ones((1, r.C), device="cuda"), ans[:2]]), pos)
        got = torch.cat([got, ans]).double().cpu()
        assert float((got - want).abs().max() / want.abs().max()) < (0.1 if bits == 8 else 1e-4)
        assert r.status() == 0
    finally:
        r.close()


@pytest.mark.gpu
def test_reader_watches_on(reader):
    """A video many times longer than the cache, in 8 bits: the same again on the same frames, and no call met anything."""
    def run():
        r = reader.FrameReader(small_trunk(), keep=None, max_tokens=35 * 60 + 8, bits=8, window=100, sinks=4)
        try:
            g = torch.Generator(device="cuda")
            g.manual_seed(4)
            for _ in range(60):
                y = r.watch(torch.rand((1, 3, 20, 28), device="cuda", generator=g))
            y = torch.cat([y, r.answer(8)])
            assert torch.isfinite(y).all() and r.status() == 0 and r.layers[0].k.shape[0] * r.page < 200
            return y
        finally:
            r.close()

    assert torch.equal(run(), run())


@pytest.mark.gpu
def test_reader_command(reader, capsys):
    reader.main(["--frames", "3", "--tokens", "2", "--bits", "8", "--window", "300"])
    out = capsys.readouterr().out
    assert "3 frames, 590 tokens in the cache" in out and "status 0" in out


@pytest.mark.parametrize("argv", [["--window", "-1"], ["--sinks", "-1"]])
def test_reader_command_refuses(reader, argv, capsys):
    with pytest.raises(SystemExit) as e:
        reader.main(argv)
    assert e.value.code == 2 and "at least" in capsys.readouterr().err


@pytest.mark.parametrize("how", [dict(bits=4), dict(window=0, keep=None), dict(sinks=-1), dict(bits=8), dict(window=5), dict(bits=8, keep=4)])
def test_reader_refuses(reader, how):
    with pytest.raises(ValueError):
        reader.FrameReader(small_trunk(), **how)
