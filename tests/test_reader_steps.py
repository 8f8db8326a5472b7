"""Steps of more tokens than the frame reader's pages have room for at once: pages used in turn behind a window."""
import pytest
import torch

from test_reader_gpu import small_trunk


@pytest.fixture(scope="module")
def reader():
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import reader
    return reader


@pytest.mark.parametrize("tokens,page,window,sinks,most", [(512, 16, 20, 3, 35), (512, 16, 50, 0, 35), (4000, 64, 1, 70, 196), (300, 8, 7, 8, 1), (640, 16, 1000, 5, 35),
                                                           (512, 16, None, 3, 35)])
def test_a_step_names_no_page_twice(reader, tokens, page, window, sinks, most):
    """Of the pages that a step writes and those that its tokens read no two are the same, wherever the step begins."""
    pages, entries, limit = reader.pages_in_turn(tokens, page, window, sinks, most)
    assert len(entries) == -(-tokens // page) and set(entries) == set(range(pages))
    for T in {1, min(most, limit or most)} if limit else {1, most, 3 * most}:
        for n in range(0, tokens - T, 1 + tokens // 200):
            low = 0 if window is None else max(0, n + 1 - window)
            seen = {w for w in range(-(-(n + T) // page)) if (w + 1) * page > low or w * page < sinks}
            assert len({entries[w] for w in seen}) == len(seen), (T, n)


def test_a_long_step_is_taken_in_parts(reader, monkeypatch):
    """No part is of more tokens than the pages have room for, and they come in order."""
    r = reader.FrameReader.__new__(reader.FrameReader)
    r.page, r.seen = 16, 0
    _, entries, r.most = reader.pages_in_turn(512, 16, 20, 3, 35)
    r.table = torch.tensor([entries])
    calls = []

    def part(self, x, pos):
        calls.append((self.seen, x.shape[0], pos.clone()))
        assert pos.is_contiguous() and pos.shape == (3, x.shape[0])
        self.seen += x.shape[0]
        return 2 * x
    monkeypatch.setattr(reader.FrameReader, "_step", part)
    x, pos = torch.randn(200, 4), torch.arange(600, dtype=torch.int32).view(3, 200)
    assert torch.equal(r.step(x, pos), 2 * x) and torch.equal(torch.cat([c[2] for c in calls], 1), pos)
    assert [c[:2] for c in calls] == [(0, 35), (35, 35), (70, 35), (105, 35), (140, 35), (175, 25)]
    with pytest.raises(ValueError):
        r.step(torch.randn(313, 4), torch.zeros((3, 313), dtype=torch.int32))
    assert len(calls) == 6 and r.step(torch.randn(312, 4), torch.zeros((3, 312), dtype=torch.int32)).shape == (312, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8])
def test_a_long_step_gives_what_frames_give(reader, bits):
    """Nine frames' tokens in one step, and a frame after the other: the same bits."""
    got = []
    for whole in (False, True):
        r = reader.FrameReader(small_trunk(), keep=None, dtype=torch.float32, max_tokens=512, bits=bits, window=20, sinks=3)
        try:
            g = torch.Generator(device="cuda")
            g.manual_seed(3)
            frames = [torch.rand((1, 3, 20, 28), device="cuda", generator=g) for _ in range(9)]
            n = r.rows * r.cols
            assert r.layers[0].k.shape[0] * r.page < 9 * n
            if whole:
                i = torch.arange(9 * n, device="cuda", dtype=torch.int32)
                y = r.step(torch.cat([r.features(f).clone() for f in frames]), torch.stack([i // n, i % n // r.cols, i % r.cols]))
                r.frames = 9
            else:
                y = torch.cat([r.watch(f) for f in frames])
            got.append(torch.cat([y, r.answer(3)]))
            assert r.seen == 9 * n + 3 and r.status() == 0
        finally:
            r.close()
    assert torch.equal(*got)
