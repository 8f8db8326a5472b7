"""Refusals of the cache in 8 bits and of attention with a window that need no GPU, and their reference against
independent formulas (CPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import cache8_ref as ref8
import decoder_ref as ref


@pytest.fixture(scope="module")
def pp():
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import ppconv
    return ppconv


def test_null_handles_and_sizes(pp):
    bad, no = pp.PP_ERR_INVALID_ARG, pp.PP_ERR_UNSUPPORTED
    L = pp.lib
    out = ctypes.c_void_p()
    to = ctypes.byref(out)
    buf = np.zeros(64, np.float32)
    at = (buf.ctypes.data + 15) // 16 * 16
    assert L.pp_attn_window(None, 1, at, 64, 64, 1, 1, None, at, 1, at, 1.0, 0, 1, 0, at, None, None) == bad
    assert L.pp_cache_append(None, 1, at, 64, 64, at, 64, 64, 1, None, at, 1, at, None) == bad
    assert L.pp_cache_read(None, 1, 1, None, at, 1, at, at, at, None) == bad
    for args in [(7, 1, 16, 1, 64, at, at, at, at), (0, 0, 16, 1, 64, at, at, at, at), (0, 1, 16, 0, 64, at, at, at, at),
                 (0, 1, 16, 1, 64, None, at, at, at), (0, 1, 16, 1, 64, at, None, at, at), (0, 1, 16, 1, 64, at, at, None, at),
                 (0, 1, 16, 1, 64, at, at, at, None), (0, 1, 16, 1, 64, at, at + 4, at, at), (0, 1, 16, 1, 64, at, at, at, at + 4)]:
        assert L.pp_cache8_create(*args, to) == bad
    assert L.pp_cache8_create(0, 1, 16, 1, 64, at, at, at, at, None) == bad
    for args in [(0, 1, 12, 1, 64), (0, 1, 512, 1, 64), (1, 1, 4, 1, 64), (2, 1, 16, 1, 72), (2, 1, 16, 1, 8), (0, 1, 16, 1, 272),
                 (1, 2 ** 30, 16, 8, 64)]:
        assert L.pp_cache8_create(*args, at, at, at, at, to) == no
    assert out.value is None


def test_window_sizes_come_first(pp):
    """Refused before the handle is looked at."""
    for window, sinks in ((0, 0), (-1, 0), (1, -1), (-2 ** 31, 0)):
        assert pp.lib.pp_attn_window(1, 1, 1, 1, 1, 1, 1, None, 1, 1, 1, 1.0, 0, window, sinks, 1, None, None) == pp.PP_ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["append", "read", "create"])
def test_host_tensors_are_refused(pp, call):
    y = pp._torch_types()
    c = pp.Cache(1)
    c.dtype, c.shape = torch.float16, (2, 1, 16, 64)
    k8, s = torch.zeros((2, 1, 16, 64), dtype=torch.int8), torch.zeros((2, 1))
    x, i = torch.zeros((1, 1, 64), dtype=torch.float16), torch.zeros((1, 1), dtype=torch.int32)
    with pytest.raises(pp.PPError) as e:
        if call == "append":
            pp.pp_cache_append(c, x, x, None, i, i[0])
        elif call == "read":
            pp.pp_cache_read(c, None, i, i[0], x, x)
        else:
            pp.pp_cache8_create(k8, k8, s, s, torch.float16)
    assert e.value.code == pp.PP_ERR_INVALID_ARG
    assert torch.int8 is y.i8


def test_reference_stays_within_half_a_step():
    """Each value is read back within half a step of its page's scale, plus half a step for each time that the scale grew."""
    g = torch.Generator().manual_seed(0)
    page, H, D = 16, 2, 16
    codes, scales = torch.zeros((3, H, page, D), dtype=torch.int8), torch.full((3, H), 1e9)
    table = torch.tensor([[2, 0, 1]])
    x = torch.randn((37, H, D), generator=g) * torch.linspace(0.5, 3, 37)[:, None, None]
    grown = torch.zeros((3, H))
    for lo, hi in ((0, 5), (5, 6), (6, 20), (20, 21), (21, 37)):
        was = scales.clone()
        ref8.append(codes, scales, x[lo:hi], table, [0, hi - lo], [hi], page)
        grown += ((scales > was) | (was > 1e8)).float()
    back = ref8.read(codes, scales, table, [0, 37], [37], page, torch.float32)
    for t in range(37):
        id = int(table[0, t // page])
        step = scales[id][:, None] * (0.5 + 1e-5) * (1 + grown[id][:, None])
        assert ((back[t] - x[t]).abs() <= step).all()
    assert (codes.abs().amax((2, 3))[[2, 0]] == 127).all()


def test_reference_window_is_a_mask():
    g = torch.Generator().manual_seed(1)
    n, H, G, D, page = 21, 2, 3, 16, 8
    k, v = torch.randn((3, H, page, D), generator=g), torch.randn((3, H, page, D), generator=g)
    q = torch.randn((9, H * G, D), generator=g)
    table = torch.tensor([[0, 1, 2]])
    out, lse, _, _ = ref8.attend(q, k, v, table, [0, 9], [n], 0.25, True, 5, 2, False)
    kk = k.transpose(1, 2).reshape(-1, H, D)[:n].double().repeat_interleave(G, 1).transpose(0, 1)
    vv = v.transpose(1, 2).reshape(-1, H, D)[:n].double().repeat_interleave(G, 1).transpose(0, 1)
    seen = torch.arange(n - 9 + 1, n + 1)[:, None]
    at = torch.arange(n)[None]
    on = (at < seen) & ((at >= seen - 5) | (at < 2))
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), kk, vv, attn_mask=on, scale=0.25)
    assert torch.allclose(out, want.transpose(0, 1), atol=1e-12)
    full, _, _, _ = ref8.attend(q, k, v, table, [0, 9], [n], 0.25, True, 100, 0, False)
    same, _, _, _ = ref.attend(q, k, v, table, [0, 9], [n], 0.25, True)
    assert torch.allclose(full, same, atol=1e-12) and math.isfinite(float(lse[0, 0]))
