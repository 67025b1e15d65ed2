"""Refusals of the rotary, cache and paged attention entry points, on the host: made-up addresses, nothing is launched."""
import ctypes
import os

import pytest
import torch

from paper_2505_12044_amd import api

NULL, SHAPE, UNSUPPORTED, ALIGN = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(api.LIB_PATH):
        from paper_2505_12044_amd import build
        build.build(force=False)
    return api.load_library()


def six(*x):
    return (ctypes.c_longlong * 6)(*x)


def four(*x):
    return (ctypes.c_int * 4)(*x)


def test_rotary_refusals(lib):
    for f in (lib.fb_rotary_fwd, lib.fb_rotary_bwd):
        def call(x0=64, y0=128, H0=2, x1=64, y1=128, H1=1, strides=six(1, 1, 64, 1, 1, 64), pos=64, freqs=64, sections=four(8, 8),
                 B=1, N=4, C=64, dtype=api.FB_BF16):
            return f(x0, y0, H0, x1, y1, H1, strides, pos, 0, 0, freqs, sections, B, N, C, 0, dtype, None)

        for name in ("x0", "y0", "x1", "y1", "strides", "pos", "freqs", "sections"):
            assert call(**{name: None}) == NULL, name
        assert call(B=0) == SHAPE and call(N=0) == SHAPE and call(H0=0) == SHAPE and call(H1=-1) == SHAPE
        assert call(sections=four(0)) == SHAPE                   # nothing to turn
        assert call(sections=four(20, 13)) == SHAPE              # more pairs than a row has
        assert call(sections=four(9, -1)) == SHAPE
        assert call(B=1 << 20, N=1 << 10, H0=1 << 3) == SHAPE
        assert call(C=48) == UNSUPPORTED and call(dtype=5) == UNSUPPORTED
        assert call(x0=65) == ALIGN and call(y0=136) == ALIGN and call(y1=130) == ALIGN and call(pos=66) == ALIGN and call(freqs=65) == ALIGN
        assert call(x0=66, dtype=api.FB_F32) == ALIGN
        assert call(y0=64) == UNSUPPORTED                        # in place, rows not where the result has them


def test_plan_refusals(lib):
    base = dict(lens=64, new_lens=128, table=64, ring=64, state=64, lens_out=256, state_out=256, slots=64, positions=64, B=2, N=1,
                page=16, n_pages=8, max_blocks=4)

    def call(**kw):
        a = {**base, **kw}
        return lib.fb_paged_plan(*(a[n] for n in base), None)

    for name in ("lens", "new_lens", "table", "ring", "state", "lens_out", "state_out", "slots"):
        assert call(**{name: None}) == NULL, name
    for name in ("B", "N", "n_pages", "max_blocks"):
        assert call(**{name: 0}) == SHAPE, name
    assert call(page=8) == UNSUPPORTED and call(page=24) == UNSUPPORTED and call(page=512) == UNSUPPORTED
    assert call(n_pages=1 << 27) == SHAPE and call(max_blocks=1 << 30) == SHAPE and call(N=1 << 30) == SHAPE
    assert call(B=4097) == UNSUPPORTED
    assert call(slots=66) == ALIGN and call(positions=65) == ALIGN
    assert call(lens_out=64) == UNSUPPORTED and call(lens_out=128) == UNSUPPORTED and call(state_out=64) == UNSUPPORTED


def test_append_refusals(lib):
    base = dict(k=64, v=64, phi_k=64, slots=64, k_pages=64, v_pages=64, phi_pages=64, strides=six(1, 1, 64, 1, 1, 64), B=2, Hkv=2, N=3,
                C=64, R=2, page=16, n_pages=8, dtype=api.FB_BF16, phi=api.FB_F32, bcast=0)

    def call(**kw):
        a = {**base, **kw}
        return lib.fb_paged_append(*(a[n] for n in base), None)

    for name in ("k", "v", "phi_k", "slots", "k_pages", "v_pages", "phi_pages", "strides"):
        assert call(**{name: None}) == NULL, name
    for name in ("B", "Hkv", "N", "n_pages"):
        assert call(**{name: 0}) == SHAPE, name
    assert call(R=-1) == SHAPE and call(R=65) == UNSUPPORTED and call(C=80) == UNSUPPORTED and call(page=40) == UNSUPPORTED
    assert call(dtype=api.FB_F32, phi=api.FB_BF16) == UNSUPPORTED and call(dtype=9) == UNSUPPORTED
    assert call(k=65) == ALIGN and call(k_pages=72) == ALIGN and call(phi_pages=68) == ALIGN and call(phi_k=66) == ALIGN
    assert call(slots=66) == ALIGN


def test_attention_refusals(lib):
    base = dict(q=64, k_pages=64, v_pages=64, phi_q=64, phi_pages=64, slopes=None, table=64, lens=64, starts=64, out=64, lse=64, B=2, H=4,
                Hkv=2, N=1, C=64, R=2, page=16, n_pages=8, max_blocks=4, causal=1, dtype=api.FB_BF16, phi=api.FB_F32, bcast=0,
                scale=0.0, ws=None, wsb=0)

    def call(**kw):
        a = {**base, **kw}
        return lib.fb_paged_attn_fwd(*(a[n] for n in base), None)

    for name in ("q", "k_pages", "v_pages", "phi_q", "phi_pages", "table", "lens", "out", "lse"):
        assert call(**{name: None}) == NULL, name
    for name in ("B", "H", "Hkv", "N", "n_pages", "max_blocks"):
        assert call(**{name: 0}) == SHAPE, name
    assert call(Hkv=3) == SHAPE and call(max_blocks=1 << 30) == SHAPE and call(n_pages=1 << 28) == SHAPE
    assert call(C=96) == UNSUPPORTED and call(R=65) == UNSUPPORTED and call(page=12) == UNSUPPORTED
    assert call(slopes=64) == UNSUPPORTED                       # two biases
    assert call(dtype=api.FB_F32, phi=api.FB_BF16) == UNSUPPORTED and call(dtype=3) == UNSUPPORTED
    for name in ("q", "k_pages", "v_pages", "phi_pages", "out", "lse", "ws"):
        assert call(**{name: 72}) == ALIGN, name
    assert call(table=66) == ALIGN and call(lens=65) == ALIGN and call(starts=66) == ALIGN and call(phi_q=66) == ALIGN
    assert call(R=0, slopes=66) == ALIGN


def test_workspace_query(lib):
    f = lib.fb_paged_attn_fwd_workspace_bytes
    assert f(8, 16, 16, 1, 128, 16, 512, api.FB_BF16) > 0
    assert f(8, 16, 16, 1, 128, 16, 8, api.FB_BF16) == 0           # short requests are not split
    for bad in ((0, 16, 16, 1, 128, 16, 512), (8, 16, 3, 1, 128, 16, 512), (8, 16, 16, 1, 100, 16, 512), (8, 16, 16, 1, 128, 20, 512),
                (8, 16, 16, 1, 128, 16, 0), (8, 16, 16, 0, 128, 16, 512)):
        assert f(*bad, api.FB_BF16) == 0


def test_wrappers_refuse_host_tensors():
    q = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    pages = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    ints = torch.zeros((1, 4), dtype=torch.int32)
    with pytest.raises(api.FlashBiasError):
        api.fb_rotary_fwd(q, None, torch.zeros((1, 1, 4), dtype=torch.int32), torch.ones(8), (8,))
    with pytest.raises(api.FlashBiasError):
        api.fb_rotary_fwd(q.transpose(2, 3), None, torch.zeros((1, 1, 64), dtype=torch.int32), torch.ones(2), (2,))
    with pytest.raises(api.FlashBiasError):
        api.fb_paged_plan(ints[0], ints[0], ints, ints[0], ints[0, :2], 4, 16)
    with pytest.raises(api.FlashBiasError):
        api.fb_paged_append(q, q, ints, pages, pages)
    with pytest.raises(api.FlashBiasError):
        api.fb_paged_attn_fwd(q, pages, pages, ints, ints[0, :1])
