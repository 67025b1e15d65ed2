"""The serving operators together, as a program uses them: prompts, decode steps, drafted tokens that are cut back, requests
that end and begin, against attention in 64 bits over each request's own history; and a decode step in a graph."""
import math

import numpy as np
import pytest
import torch

from paper_2505_12044_amd import api
from paper_2505_12044_amd.paged import PagedCache
from tests._paged_util import HALF, i32, randn

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def freqs_of(P):
    return torch.tensor([10000.0 ** (-p / P) for p in range(P)], dtype=F32).cuda()


def turn64(x, pos, freqs):
    P = freqs.numel()
    angle = pos[:, None].double() * freqs.double().cpu()
    c, s = angle.cos(), angle.sin()
    return torch.cat((x[..., :P] * c - x[..., P:] * s, x[..., P:] * c + x[..., :P] * s), -1)


class History:
    """What a request's layer has seen: rotated keys as stored, values, factors, in 64 bits."""

    def __init__(self):
        self.k, self.v, self.f = [], [], []


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bias", ["rotary", "alibi", "factors"])
def test_prompts_and_decode_steps(dtype, bias):
    B, H, Hkv, C, page, layers = 5, 8, 2, 64, 16, 2
    R = 2 if bias == "factors" else 0
    rng = np.random.default_rng(1)
    g = torch.Generator().manual_seed(2)
    cache = PagedCache(layers, B, Hkv, C, page, 24, 320, rank=R, dtype=dtype)
    freqs = freqs_of(C // 2)
    slopes = torch.tensor([2.0 ** (-h - 1) for h in range(H)], device="cuda") if bias == "alibi" else None
    hist = [[History() for _ in range(B)] for _ in range(layers)]
    lens = np.zeros(B, np.int64)
    plans = [(np.array([37, 0, 150, 16, 1]), 150)]                     # prompts
    for t in range(12):
        n = 1 if t % 3 else 4                                          # decode, or a few drafted tokens
        plans.append((None, n))
    refused = 0
    for step, (want, n) in enumerate(plans):
        if want is None:
            want = lens + (1 if n == 1 else rng.integers(0, n + 1, B))
            if step == 4:
                want[2] = 0                                            # ended
            if step == 5:
                want[2], want[0] = 3, max(int(lens[0]) - 3, 0)         # a new one; drafted tokens cut back
                n = 4
            if step == 7:
                want[1] = 0
            if step == 8:
                want[1], n = 310, 310                                  # more than is left now and then
        cache.step(i32(want), n)
        got = cache.lens.cpu().numpy().astype(np.int64)
        refused += int((got != want).sum())
        assert all(w == x or x == o for w, x, o in zip(want, got, lens))
        for layer in range(layers):
            x = randn(g, (B, n, H + 2 * Hkv, C), dtype)                # a fused projection
            q, k, v = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2), x[:, :, H + Hkv:].transpose(1, 2)
            phi_q = randn(g, (B, H, n, R), F32) if R else None
            phi_k = randn(g, (B, Hkv, n, R), F32) if R else None
            if bias == "rotary":
                q, k = api.fb_rotary_fwd(q, k, cache.positions[None], freqs, (C // 2,))
            cache.append(layer, k, v, phi_k)
            out, lse = cache.attend(layer, q.contiguous(), phi_q, slopes)
            torch.cuda.synchronize()
            for b in range(B):
                h, o, m = hist[layer][b], int(lens[b]), int(got[b])
                del h.k[m:], h.v[m:], h.f[m:]
                for i in range(max(m - o, 0)):
                    if bias == "rotary":                               # keys at their positions, before their rounding
                        raw = x[b, i, H:H + Hkv].double().cpu()
                        exact = turn64(raw, torch.tensor([o + i]), freqs)
                        assert ((k[b, :, i].double().cpu() - exact).abs() <= exact.abs() * HALF[dtype] * 1.001 + raw.abs().amax() * 2.0 ** -20).all()
                    h.k.append(k[b, :, i].double().cpu())
                    h.v.append(v[b, :, i].double().cpu())
                    if R:
                        h.f.append(phi_k[b, :, i].double().cpu())
                for i in range(n):
                    if i >= m - o:
                        assert (out[b, :, i] == 0).all() and (lse[b, :, i] == -math.inf).all()
                        continue
                    K, V = (torch.stack(y[:o + i + 1], 1).repeat_interleave(H // Hkv, 0) for y in (h.k, h.v))
                    qi = q[b, :, i].double().cpu()
                    s = (K * qi[:, None]).sum(-1) / math.sqrt(C)
                    size = (K * qi[:, None]).abs().sum(-1).amax(-1) / math.sqrt(C)
                    if R:
                        F = torch.stack(h.f[:o + i + 1], 1).repeat_interleave(H // Hkv, 0)
                        s = s + (F * phi_q[b, :, i, None].double().cpu()).sum(-1)
                        size = size + (F * phi_q[b, :, i, None].double().cpu()).abs().sum(-1).amax(-1)
                    if bias == "alibi":
                        far = o + i - torch.arange(o + i + 1).double()
                        s = s - slopes.double().cpu()[:, None] * far
                        size = size + slopes.double().cpu() * far.amax()
                    p = s.softmax(-1)
                    ref = (p[..., None] * V).sum(1)
                    # as in attend64: scores, sums, two limbs, the result's rounding
                    dp = 2 * (C + 80) * 2.0 ** -24 * size + (o + i + 16) * 2.0 ** -23 + (2.0 ** -16 if dtype == BF else 0)
                    tol = ref.abs() * HALF[dtype] + 2 * dp[:, None] * (p[..., None] * V.abs()).sum(1)
                    assert ((out[b, :, i].double().cpu() - ref).abs() <= tol).all(), (step, layer, b, i)
                    assert ((lse[b, :, i].double().cpu() - s.logsumexp(-1)).abs() <= dp + (s.logsumexp(-1).abs() + 1) * 2.0 ** -22).all()
        lens = got
    assert refused > 0


def test_a_decode_step_in_a_graph():
    B, H, Hkv, C, page = 6, 4, 2, 64, 16
    cache, eager = (PagedCache(1, B, Hkv, C, page, 60, 700, dtype=BF) for _ in range(2))
    freqs = freqs_of(C // 2)
    g = torch.Generator().manual_seed(2)
    prompt = i32([100, 15, 600, 16, 0, 31])
    for c in (cache, eager):
        c.step(prompt, 600)
    k, v = randn(g, (B, Hkv, 600, C), BF), randn(g, (B, Hkv, 600, C), BF)
    for c in (cache, eager):
        c.append(0, k, v)
    want = prompt.clone()
    x = torch.empty((B, 1, H + 2 * Hkv, C), dtype=BF, device="cuda")

    def step(c):
        c.step(want, 1)
        q, k, v = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2), x[:, :, H + Hkv:].transpose(1, 2)
        q, k = api.fb_rotary_fwd(q, k, c.positions[None], freqs, (C // 2,))
        c.append(0, k, v)
        return c.attend(0, q)

    # warm up on a copy of the state: a step with unchanged lengths changes nothing
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x.zero_()
        step(cache)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(cache)
    for t in range(20):
        x.copy_(randn(g, x.shape, BF))
        want += i32([1, 1, 1, 1, 1, 0])
        if t == 6:
            want[2] = 0
        if t == 9:
            want[2], want[5] = 1, 32
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eo, el = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eo) and torch.equal(lse, el), t
        assert torch.equal(cache.lens, eager.lens) and torch.equal(cache.table, eager.table) and torch.equal(cache._now, eager._now)
    assert cache.lens.tolist() == want.tolist()


def test_refusals_of_the_cache():
    cache = PagedCache(1, 2, 1, 64, 16, 8, 64)
    z = torch.zeros((2, 1, 1, 64), dtype=BF, device="cuda")
    with pytest.raises(api.FlashBiasError):
        cache.append(0, z, z)                                          # no step yet
    with pytest.raises(api.FlashBiasError):
        PagedCache(1, 2, 1, 64, 16, 0, 64)
    with pytest.raises(api.FlashBiasError):
        cache.step(torch.zeros(2, dtype=torch.int64, device="cuda"), 1)
    with pytest.raises(api.FlashBiasError):
        cache.step(torch.zeros(3, dtype=torch.int32, device="cuda"), 1)
    cache.step(torch.ones(2, dtype=torch.int32, device="cuda"), 1)
    with pytest.raises(api.FlashBiasError):
        cache.append(0, z.float(), z.float())
    with pytest.raises(api.FlashBiasError):
        cache.append(0, z, z, torch.zeros((2, 1, 1, 2), device="cuda"))       # factors without pages
    with pytest.raises(api.FlashBiasError):
        cache.attend(0, torch.zeros((2, 3, 1, 32), dtype=BF, device="cuda"))
