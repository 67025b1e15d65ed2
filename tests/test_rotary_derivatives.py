"""Which gradients the rotary function forms, and that they can be differentiated again: on the host with elementary operations
in the kernels' place, on the GPU with the kernels."""
import pytest
import torch

from paper_2505_12044_amd import api, autograd

F32 = torch.float32


def turn(x, positions, freqs, sections, interleaved, sign):
    axis = sum(([a] * n for a, n in enumerate(sections)), [])
    angle = positions.double()[axis].permute(1, 2, 0) * freqs.double()
    cos, sin = angle.cos()[:, None].to(x.dtype), sign * angle.sin()[:, None].to(x.dtype)
    P = freqs.numel()
    i1, i2 = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    y = torch.zeros_like(x)
    y[..., 2 * P:] = x[..., 2 * P:]
    y[..., i1] = x[..., i1] * cos - x[..., i2] * sin
    y[..., i2] = x[..., i2] * cos + x[..., i1] * sin
    return y


def inputs(device, seed=1):
    g = torch.Generator().manual_seed(seed)
    q, k = (torch.randn(2, h, 7, 16, generator=g).to(device).requires_grad_() for h in (3, 2))
    w = torch.randn(2, 3, 7, 16, generator=g).to(device)
    pos = torch.randint(0, 500, (2, 2, 7), generator=g).int().to(device)
    freqs = (10.0 ** -torch.arange(7.0)).to(device)
    return q, k, w, pos, freqs, (3, 4)


@pytest.fixture(params=["host", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cuda":
        return "cuda"

    def stand_in(sign):
        def call(q, k, positions, freqs, sections, interleaved=False):
            called.append((q is not None, k is not None))
            with torch.no_grad():
                return tuple(None if x is None else turn(x, positions, freqs, sections, interleaved, sign) for x in (q, k))
        return call

    called = []
    monkeypatch.setattr(api, "fb_rotary_fwd", stand_in(1))
    monkeypatch.setattr(api, "fb_rotary_bwd", stand_in(-1))
    monkeypatch.setattr(api, "called", called, raising=False)
    return "cpu"


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_penalty_on_the_gradient(device, interleaved):
    q, k, w, pos, freqs, sections = inputs(device)

    def penalty(q, k, rotary):
        yq, yk = rotary(q, k)
        loss = (yq.sin() * w).sum() + (yq[:, :2] * yk ** 3).sum()
        gq, gk = torch.autograd.grad(loss, (q, k), create_graph=True)
        return loss + (gq ** 2).sum() + (gk ** 3).sum()

    got = torch.autograd.grad(penalty(q, k, lambda q, k: autograd.rotary_positions(q, k, pos, freqs, sections, interleaved)), (q, k))
    ref = [x.detach().double().cpu().requires_grad_() for x in (q, k)]
    w = w.double().cpu()
    cpu = (pos.cpu(), freqs.cpu(), sections, interleaved)
    want = torch.autograd.grad(penalty(*ref, lambda q, k: (turn(q, *cpu, 1), turn(k, *cpu, 1))), ref)
    # A turn is within 8 * 2^-24 of |x1| + |x2| <= 1.5 |x|; three of them follow each other, their errors pass through powers up to
    # the third, and two such terms meet: 8 * 1.5 * 3 * 3 * 2 = 216 units, and a few for the elementary operations.
    for a, b in zip(got, want):
        assert (a.double().cpu() - b).abs().max() <= 256 * 2.0 ** -24 * b.abs().max()


def test_one_tensor_twice_differentiated(device):
    q, _, w, pos, freqs, sections = inputs(device)
    gq, = torch.autograd.grad((autograd.rotary_positions(q, None, pos, freqs, sections) * w).square().sum(), q, create_graph=True)
    h, = torch.autograd.grad(gq, q, w)
    # the Hessian is R^T diag(2 w^2) R
    y = turn(w.double().cpu(), pos.cpu(), freqs.cpu(), sections, False, 1)
    want = turn(2 * w.double().cpu() ** 2 * y, pos.cpu(), freqs.cpu(), sections, False, -1)
    assert (h.double().cpu() - want).abs().max() <= 64 * 2.0 ** -24 * want.abs().max()      # three turns of 12 units, the products


@pytest.mark.parametrize("create_graph", [False, True])
def test_only_the_gradient_that_is_asked_for(device, create_graph):
    q, k, w, pos, freqs, sections = inputs(device)
    for leaf, other in ((q, k), (k, q)):
        yq, yk = autograd.rotary_positions(q, k, pos, freqs, sections)
        both = torch.autograd.grad((yq.sum() + yk.square().sum()), (q, k))
        yq, yk = autograd.rotary_positions(*(x if x is leaf else x.detach() for x in (q, k)), pos, freqs, sections)
        if device == "cpu":
            api.called.clear()
        got, = torch.autograd.grad(yq.sum() + yk.square().sum(), leaf, create_graph=create_graph)
        assert torch.equal(got, both[0] if leaf is q else both[1])
        if device == "cpu":
            assert len(api.called) == 1 and sum(api.called[0]) == 1
