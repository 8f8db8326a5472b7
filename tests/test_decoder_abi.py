"""Refusals of the decoder operators that need no GPU, and their reference against independent formulas (CPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import decoder_ref as ref


@pytest.fixture(scope="module")
def pp():
    from paper_2004_11250_gb300 import build
    build.build()
    from paper_2004_11250_gb300 import ppconv
    return ppconv


def test_null_handles_and_sizes(pp):
    bad = pp.PP_ERR_INVALID_ARG
    L = pp.lib
    out = ctypes.c_void_p()
    ref_ = ctypes.byref(out)
    buf = np.zeros(64, np.float32)
    at = (buf.ctypes.data + 15) // 16 * 16
    assert L.pp_attn_forward(None, 1, at, 64, 64, 1, 1, None, at, 1, at, 1.0, 0, None, 0, at, None, None) == bad
    assert L.pp_cache_select(None, 1, at, 64, 64, 1, 1, None, at, 1, at, 0, 0, 1, 1, at, None) == bad
    assert L.pp_cache_summarize(None, at, 1, None) == bad
    assert L.pp_cache_device_status(None, None) == bad
    assert L.pp_qkv_store(None, None, 1, at, at, 0.0, None, 0, 0, 0, None, None, at, 1, 1, None, at, 1, 1, None) == bad
    assert L.pp_qk_rotate(None, 0, 1, at, 0.0, at, 1, 1, 1, None, at, None, 0, 0, 0, None, None, None) == bad
    for args in [(7, 1, 16, 1, 64, at, at, None, None), (0, 0, 16, 1, 64, at, at, None, None), (0, 1, 16, 1, 64, None, at, None, None),
                 (0, 1, 16, 1, 64, at, None, None, None), (0, 1, 16, 1, 64, at + 4, at, None, None), (0, 1, 16, 1, 64, at, at, at, None)]:
        assert L.pp_cache_create(*args, ref_) == bad
    assert L.pp_cache_create(0, 1, 16, 1, 64, at, at, None, None, None) == bad
    for args in [(0, 1, 12, 1, 64), (0, 1, 512, 1, 64), (0, 1, 4, 1, 64), (0, 1, 16, 1, 12), (0, 1, 16, 1, 264), (1, 2 ** 30, 16, 8, 64)]:
        assert L.pp_cache_create(*args, at, at, None, None, ref_) == pp.PP_ERR_UNSUPPORTED
    assert out.value is None
    L.pp_cache_destroy(None)
    L.pp_rope_destroy(None)


def test_rope_refusals(pp):
    f = [1.0, 0.5]
    for kw in [dict(axes=0), dict(axes=9), dict(axis=[0, 1]), dict(freq=[1.0, math.nan]), dict(freq=[math.inf, 1.0]), dict(D=2)]:
        a = {**dict(D=8, axis=None, freq=f, axes=1), **kw}
        with pytest.raises(pp.PPError) as e:
            pp.pp_rope_create(a["D"], a["axis"], a["freq"], a["axes"])
        assert e.value.code == pp.PP_ERR_INVALID_ARG
    for D in (7, 258):
        with pytest.raises(pp.PPError) as e:
            pp.pp_rope_create(D, None, f)
        assert e.value.code == pp.PP_ERR_UNSUPPORTED


def test_reference_rotation_is_a_complex_product():
    g = torch.Generator().manual_seed(0)
    x = torch.randn((3, 2, 10), generator=g, dtype=torch.float64).float()
    pos = torch.tensor([[1, 5, 9], [0, 2, 40]], dtype=torch.int32)
    f = [1.0, 0.3, 0.01]
    for inter in (False, True):
        y, _ = ref.rotate(x, None, -1.0, pos, [0, 1, 1], f, inter)
        lo, hi = (x[..., 0:6:2], x[..., 1:6:2]) if inter else (x[..., :3], x[..., 3:6])
        ang = torch.stack([pos[0].double() * f[0], pos[1].double() * f[1], pos[1].double() * f[2]], 1)
        z = torch.complex(lo.double(), hi.double()) * torch.polar(torch.ones_like(ang), ang)[:, None]
        a, b = (y[..., 0:6:2], y[..., 1:6:2]) if inter else (y[..., :3], y[..., 3:6])
        assert torch.allclose(a, z.real, atol=1e-12) and torch.allclose(b, z.imag, atol=1e-12)
        assert torch.equal(y[..., 6:], x[..., 6:].double())


def test_reference_attention_is_torch_attention():
    """One sequence in order: the library routine on the same numbers."""
    g = torch.Generator().manual_seed(0)
    n, H, G, D, page = 21, 2, 3, 16, 8
    k, v = torch.randn((3, H, page, D), generator=g), torch.randn((3, H, page, D), generator=g)
    q = torch.randn((n, H * G, D), generator=g)
    out, lse, _, _ = ref.attend(q, k, v, torch.tensor([[0, 1, 2]]), [0, n], [n], 0.25, True)
    kk = k.transpose(1, 2).reshape(-1, H, D)[:n].double().repeat_interleave(G, 1).transpose(0, 1)
    vv = v.transpose(1, 2).reshape(-1, H, D)[:n].double().repeat_interleave(G, 1).transpose(0, 1)
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), kk, vv, is_causal=True, scale=0.25)
    assert torch.allclose(out, want.transpose(0, 1), atol=1e-12)
    assert math.isclose(float(lse[0, 0]), 0.25 * float(q[0, 0].double() @ kk[0, 0]), abs_tol=1e-12)


def test_reference_score_bounds_the_best_key():
    """Before the rounding of the query, a page's score is no less than any sum over the group of q.k in it."""
    g = torch.Generator().manual_seed(0)
    k = torch.randn((5, 1, 8, 32), generator=g)
    codes, scales = ref.summarize(k)
    q = torch.randn((3, 32), generator=g)
    up, down = q.clamp(min=0).sum(0).double(), q.clamp(max=0).sum(0).double()
    for p in range(5):
        bound = float(scales[p, 0]) * float((up * codes[p, 0, 0]).sum() + (down * codes[p, 0, 1]).sum())
        best = float((q.double() @ k[p, 0].double().T).amax(1).sum())
        assert bound >= best - 1e-5
