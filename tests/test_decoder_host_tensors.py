"""The decoder operators take GPU memory only: a host tensor in any place is refused before the library is called (CPU)."""
import pytest
import torch


class Lib:
    """In the library's place: any call but the one that names a status is a failure."""

    def __init__(self, lib):
        self.pp_status_string = lib.pp_status_string

    def __getattr__(self, name):
        def called(*a):
            raise AssertionError(f"{name} was called")
        return called


class OnGpu:
    """A host tensor that says it is on the GPU."""

    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def pp(monkeypatch):
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import ppconv
    monkeypatch.setattr(ppconv, "lib", Lib(ppconv.lib))
    return ppconv


def calls(pp):
    """name -> (call of its tensors, the tensors)."""
    T, Hq, H, D, page, pages, W = 3, 4, 2, 64, 16, 5, 2
    i32, f16 = torch.int32, torch.float16
    rope, cache = pp.Rope(1), pp.Cache(1)
    rope.D, rope.axes = D, 1
    cache.dtype, cache.shape = f16, (pages, H, page, D)
    z = lambda *s, dtype=f16: torch.zeros(s, dtype=dtype)  # noqa: E731
    q, k, w = z(T, Hq, D), z(T, H, D), z(D, dtype=torch.float32)
    pos, slots, table, lens, starts = z(1, T, dtype=i32), z(T, dtype=i32), z(1, W, dtype=i32), z(1, dtype=i32), z(2, dtype=i32)
    sel, pool = z(T, H, 2, dtype=i32), z(pages, H, page, D)
    codes, scales = z(pages, H, 2, D, dtype=torch.int8), z(pages, H, dtype=torch.float32)
    return {
        "rotate": (lambda pos, q, qw, qo, k, kw, ko: pp.pp_qk_rotate(rope, pos, 0.0, q, qw, qo, k, kw, ko), [pos, q, w, q, k, w, k]),
        "store": (lambda pos, slots, q, qw, qo, k, kw, v: pp.pp_qkv_store(rope, cache, pos, slots, 0.0, q, qw, qo, k, kw, v),
                  [pos, slots, q, w, q, k, w, k]),
        "cache": (lambda *a: pp.pp_cache_create(*a), [pool, pool, codes, scales]),
        "summarize": (lambda ids: pp.pp_cache_summarize(cache, ids), [lens]),
        "select": (lambda q, starts, table, lens, sel: pp.pp_cache_select(cache, q, starts, table, lens, 0, 0, 1, sel), [q, starts, table, lens, sel]),
        "attend": (lambda q, starts, table, lens, sel, out, lse: pp.pp_attn_forward(cache, q, starts, table, lens, 1.0, 0, sel, out, lse),
                   [q, starts, table, lens, sel, q, z(T, Hq, dtype=torch.float32)]),
    }


@pytest.mark.parametrize("name", ["rotate", "store", "cache", "summarize", "select", "attend"])
def test_host_tensors_are_refused(pp, name):
    call, tensors = calls(pp)[name]
    with pytest.raises(AssertionError, match="was called"):  # all on the GPU: on to the library
        call(*[OnGpu(t) for t in tensors])
    for i in range(len(tensors)):
        with pytest.raises(pp.PPError) as e:
            call(*[t if j == i else OnGpu(t) for j, t in enumerate(tensors)])
        assert e.value.code == pp.PP_ERR_INVALID_ARG
