"""The frame reader's command and answers at the ends of their ranges."""
import pytest


@pytest.fixture(scope="module")
def reader():
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import reader
    return reader


@pytest.mark.parametrize("argv", [["--frames", "0"], ["--frames", "-1"], ["--tokens", "-1"], ["--keep", "2"], ["--keep", "-1"]])
def test_reader_command_refuses(reader, argv, capsys):
    """Before anything is done on a GPU."""
    with pytest.raises(SystemExit) as e:
        reader.main(argv)
    assert e.value.code == 2 and "at least" in capsys.readouterr().err


@pytest.mark.gpu
def test_reader_without_an_answer(reader, capsys):
    reader.main(["--frames", "1", "--tokens", "0"])
    out = capsys.readouterr().out
    assert "1 frames, 196 tokens in the cache" in out and "answer" not in out and "status 0" in out


@pytest.mark.gpu
def test_an_answer_of_no_tokens_is_empty(reader):
    r = reader.FrameReader(max_tokens=196)
    try:
        assert r.answer(0).shape == (0, r.C) and r.seen == 0
    finally:
        r.close()
