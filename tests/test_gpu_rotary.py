"""Rotary positions against the definition in 64 bits: axes, layouts, types, far positions, gradients."""
import math

import pytest
import torch

from paper_2505_12044_amd import api, autograd
from tests._paged_util import HALF, randn

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def turn64(x, pos, freqs, sections, interleaved, inverse=False):
    """The turned rows and a bound of the kernel's error."""
    x = x.double().cpu()
    P = sum(sections)
    axis = sum(([a] * n for a, n in enumerate(sections)), [])
    angle = pos.double().cpu()[axis].permute(1, 2, 0) * freqs.double().cpu()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
    i1, i2 = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    y, size = x.clone(), torch.zeros_like(x)
    x1, x2 = x[..., i1], x[..., i2]
    y[..., i1], y[..., i2] = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    # sine and cosine within 6 * 2^-24 (the reduced angle's three roundings, the polynomial), the products 2 * 2^-24; the
    # angle itself in 64 bits: two roundings here, two in the kernel
    size[..., i1] = size[..., i2] = (x1.abs() + x2.abs()) * (2.0 ** -21 + angle.abs()[:, None] * 2.0 ** -51)
    return y, size


def check(got, x, *args, **kw):
    y, tol = turn64(x, *args, **kw)
    assert got.is_contiguous() and got.shape == x.shape and got.dtype == x.dtype
    err = (got.double().cpu() - y).abs()
    assert (err <= tol + y.abs() * HALF[x.dtype] * (1 + 2.0 ** -10)).all(), (err - tol - y.abs() * HALF[x.dtype]).max()


def inputs(B, N, H, Hkv, C, dtype, axes, far=1000, shared=False, layout="heads", seed=0, f32_pos=False):
    g = torch.Generator().manual_seed(seed)
    if layout == "heads":
        q, k = randn(g, (B, H, N, C), dtype), randn(g, (B, Hkv, N, C), dtype)
    else:           # slices of one projection; "odd": rows that start at odd elements
        x = randn(g, (B, N, H + 2 * Hkv, C), dtype)
        if layout == "odd":
            wide = torch.zeros((B, N, (H + 2 * Hkv) * C + 3), dtype=dtype, device="cuda")
            wide[..., 1:-2] = x.flatten(2)
            x = wide[..., 1:-2].unflatten(2, (H + 2 * Hkv, C))
        q, k = x[:, :, :H].transpose(1, 2), x[:, :, H:H + Hkv].transpose(1, 2)
    pos = torch.randint(0, far, (axes, 1 if shared else B, N), generator=g)
    pos = (pos.float() + 0.37).cuda() if f32_pos else pos.int().cuda()
    return q, k, pos


def freqs_of(P, base=10000.0):
    return torch.tensor([base ** (-p / P) for p in range(P)], dtype=F32).cuda()


@pytest.mark.parametrize("C", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["heads", "fused", "odd"])
def test_layouts_and_types(C, dtype, interleaved, layout):
    for B, N, H, Hkv in ((1, 1, 4, 1), (3, 37, 5, 2), (2, 130, 3, 3)):
        q, k, pos = inputs(B, N, H, Hkv, C, dtype, 1, layout=layout, seed=N)
        f = freqs_of(C // 2)
        yq, yk = api.fb_rotary_fwd(q, k, pos, f, (C // 2,), interleaved=interleaved)
        torch.cuda.synchronize()
        check(yq, q, pos, f, (C // 2,), interleaved)
        check(yk, k, pos, f, (C // 2,), interleaved)


@pytest.mark.parametrize("sections", [(32,), (16, 16), (8, 12, 12), (4, 4, 4, 4), (1, 30), (7,), (3, 5, 1), (1,), (0, 20), (16, 0, 4)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_axes_and_partial_rows(sections, interleaved, dtype):
    q, k, pos = inputs(2, 19, 4, 2, 64, dtype, len(sections), shared=len(sections) % 2 == 0, seed=3)
    f = freqs_of(sum(sections))
    yq, yk = api.fb_rotary_fwd(q, k, pos, f, sections, interleaved=interleaved)
    torch.cuda.synchronize()
    check(yq, q, pos, f, sections, interleaved)
    check(yk, k, pos, f, sections, interleaved)
    rest = 2 * sum(sections)
    assert torch.equal(yq[..., rest:], q[..., rest:])


@pytest.mark.parametrize("far", [1 << 17, 1 << 24, (1 << 31) - 1])
def test_far_positions(far):
    q, k, pos = inputs(2, 40, 2, 2, 64, F32, 1, far=far, seed=5)
    pos[0, 0, 0], pos[0, 0, 1] = far - 1 if far < (1 << 31) - 1 else far, -far
    f = freqs_of(32)
    yq, yk = api.fb_rotary_fwd(q, k, pos, f, (32,))
    torch.cuda.synchronize()
    check(yq, q, pos, f, (32,), False)


def test_fractional_positions_one_tensor_and_in_place():
    q, _, pos = inputs(2, 33, 3, 1, 32, BF, 2, f32_pos=True, seed=6)
    f = freqs_of(16)
    yq, none = api.fb_rotary_fwd(q, None, pos, f, (8, 8))
    assert none is None
    check(yq, q, pos, f, (8, 8), False)
    x = q.clone()
    api.fb_rotary_fwd(x, None, pos, f, (8, 8), out=(x, None))
    assert torch.equal(x, yq)
    wide = torch.empty((2, 33, 3, 32), dtype=BF, device="cuda").transpose(1, 2)
    with pytest.raises(api.FlashBiasError):
        api.fb_rotary_fwd(q, None, pos, f, (8, 8), out=(wide, None))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients(dtype, interleaved):
    sections = (4, 6, 6)
    q, k, pos = inputs(2, 21, 4, 2, 32, dtype, 3, layout="fused", seed=7)
    f = freqs_of(16)
    q, k = q.detach().requires_grad_(), k.detach().requires_grad_()
    yq, yk = autograd.rotary_positions(q, k, pos, f, sections, interleaved=interleaved)
    g = torch.Generator().manual_seed(1)
    dq, dk = randn(g, yq.shape, dtype), randn(g, yk.shape, dtype)
    gq, gk = torch.autograd.grad((yq, yk), (q, k), (dq, dk))
    check(yq, q.detach(), pos, f, sections, interleaved)
    check(gq.contiguous(), dq, pos, f, sections, interleaved, inverse=True)
    check(gk.contiguous(), dk, pos, f, sections, interleaved, inverse=True)
    # only one of the two is used; a gradient that is an expanded view
    yq, yk = autograd.rotary_positions(q, k, pos, f, sections, interleaved=interleaved)
    gq, gk = torch.autograd.grad(yk.float().sum(), (q, k))
    assert (gq == 0).all()
    check(gk.contiguous(), torch.ones_like(gk, memory_format=torch.contiguous_format), pos, f, sections, interleaved, inverse=True)
    y = autograd.rotary_positions(q, None, pos, f, sections, interleaved=interleaved)
    assert torch.equal(y, autograd.rotary_positions(q, k, pos, f, sections, interleaved=interleaved)[0])


def test_gradients_against_differences():
    q, k, pos = inputs(1, 5, 2, 1, 16, F32, 2, seed=8)
    f = freqs_of(8)
    g = torch.Generator().manual_seed(1)
    w, d = randn(g, q.shape, F32), randn(g, q.shape, F32)
    q.requires_grad_()

    def loss(x):
        return (autograd.rotary_positions(x, None, pos, f, (4, 4)).double() * w.double()).sum()

    grad, = torch.autograd.grad(loss(q), q)
    h = 2.0 ** -6
    with torch.no_grad():
        diff = ((loss(q + h * d) - loss(q - h * d)) / (2 * h)).item()
    # linear in q: only rounding is left, 2^-20 of the magnitudes over the step
    assert abs(diff - (grad.double() * d.double()).sum().item()) <= 2.0 ** -20 / h * (q.abs() + d.abs() + 1).sum().item() * w.abs().max().item()


def test_attention_after_rotary_trains_as_one_graph():
    q, k, pos = inputs(2, 48, 4, 4, 32, BF, 1, layout="fused", seed=9)
    f = freqs_of(16)
    v = randn(torch.Generator().manual_seed(2), (2, 4, 48, 32), BF).requires_grad_()
    q, k = q.detach().requires_grad_(), k.detach().requires_grad_()
    yq, yk = autograd.rotary_positions(q, k, pos, f, (16,))
    out = autograd.lowrank_bias_attention(yq, yk, v, causal=True)
    out.float().square().sum().backward()
    rq, rk, rv = (x.detach().float().cpu().requires_grad_() for x in (q, k, v))

    def turn(x):
        angle = pos.double().cpu()[0][..., None] * f.double().cpu()
        c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
        a, b = x[..., :16], x[..., 16:]
        return torch.cat((a * c - b * s, b * c + a * s), -1)

    score = turn(rq) @ turn(rk).transpose(-1, -2) / math.sqrt(32)
    score = score.masked_fill(torch.ones(48, 48).triu(1).bool(), -math.inf)
    (score.softmax(-1) @ rv).square().sum().backward()
    for got, want in ((q.grad, rq.grad), (k.grad, rk.grad), (v.grad, rv.grad)):
        rel = (got.float().cpu() - want).norm() / want.norm()
        assert rel < 4 * 2.0 ** -8, rel        # bf16 inputs of the attention, its probabilities and the two gradients' rounding


@pytest.mark.parametrize("replays", [3])
def test_forward_and_backward_in_a_graph(replays):
    q, k, pos = inputs(2, 64, 4, 2, 64, BF, 2, seed=10)
    f = freqs_of(32)
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    out, grad = (torch.empty_like(q), torch.empty_like(k)), (torch.empty_like(q), torch.empty_like(k))

    def step():
        api.fb_rotary_fwd(q, k, pos, f, (16, 16), out=out)
        api.fb_rotary_bwd(dq, dk, pos, f, (16, 16), out=grad)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(replays):
        for t in (q, k, dq, dk):
            t.normal_()
        pos += 7
        want = api.fb_rotary_fwd(q, k, pos, f, (16, 16)) + api.fb_rotary_bwd(dq, dk, pos, f, (16, 16))
        for t in (*out, *grad):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, *grad), want))
