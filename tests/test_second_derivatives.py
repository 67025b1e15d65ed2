"""The attention functions have first derivatives only: with create_graph=True they give the same gradients, and differentiating
those raises, whatever the inputs' layout and whichever tensor is asked for.  On the host with stand-ins for the kernels."""
import pytest
import torch

from paper_2505_12044_amd import api, autograd

B, H, N, C, R = 2, 3, 8, 16, 4
NAMES = ("lowrank", "cross", "mul", "alibi", "dense")


def leaf(g, device, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g).to(dtype).to(device).requires_grad_()


def make(name, device, strided):
    """The function of its leaves, and the leaves."""
    g = torch.Generator().manual_seed(3)
    M = 12 if name == "cross" else N

    def rows(n):
        return leaf(g, device, B, n, H, C) if strided else leaf(g, device, B, H, n, C)

    def t(x):
        return x.transpose(1, 2) if strided else x

    x = [rows(N), rows(M), rows(M)]
    if name == "alibi":
        x.append(leaf(g, device, H, dtype=torch.float32))
        return lambda q, k, v, s: autograd.alibi_attention(t(q), t(k), t(v), s), x
    if name == "dense":
        x.append(leaf(g, device, B, H, N, N))
        return lambda q, k, v, b: autograd.dense_bias_attention(t(q), t(k), t(v), b), x
    x += [leaf(g, device, B, H, N, R, dtype=torch.float32), leaf(g, device, B, H, M, R, dtype=torch.float32)]
    f = autograd.multiplicative_bias_attention if name == "mul" else autograd.lowrank_bias_attention
    return lambda q, k, v, a, b: f(t(q), t(k), t(v), a, b), x


@pytest.fixture(params=["host", pytest.param("cuda", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cuda":
        return "cuda"

    def forward(q, k, v, *rest, **kw):
        assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        return q * v.mean(), q[..., 0].float()

    def backward(*args, **kw):          # (the inputs, out, lse, dout): some gradient for each input
        grads = [2 * x + args[-1].mean().to(x.dtype) for x in args[:-3]]
        return grads[:3] if "dslope_rows" in kw else grads

    for n in ("lowrank_attn", "lowrank_xattn", "lowrank_mulbias_attn", "alibi_attn", "dense_bias_attn"):
        monkeypatch.setattr(api, f"fb_{n}_fwd", forward)
        monkeypatch.setattr(api, f"fb_{n}_bwd", backward)
    monkeypatch.setattr(torch, "empty", torch.zeros)          # the slopes' rows, which no kernel fills
    return "cpu"


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("strided", [False, True])
def test_first_derivatives_with_a_graph(device, name, strided):
    f, x = make(name, device, strided)
    plain = torch.autograd.grad(f(*x).float().square().sum(), x)
    graph = torch.autograd.grad(f(*x).float().square().sum(), x, create_graph=True)
    for a, b in zip(plain, graph):
        assert torch.equal(a, b) and not a.requires_grad and b.requires_grad


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("strided", [False, True])
def test_second_derivatives_raise(device, name, strided):
    f, x = make(name, device, strided)
    for i in range(len(x)):
        out = f(*x)
        # constant upstream gradient: the gradients depend on the inputs alone
        g, = torch.autograd.grad(out.float().sum(), x[i], create_graph=True)
        for j in range(len(x)):
            # a loss that stays differentiable by another path
            with pytest.raises(api.FlashBiasError, match="second derivatives"):
                torch.autograd.grad(g.float().square().sum() + x[j].float().sum(), x[j], retain_graph=True)


def test_a_gradient_that_does_not_pass_through_again(device):
    f, x = make("lowrank", device, True)
    w = torch.ones(3, device=device, requires_grad=True)
    g = torch.autograd.grad((f(*x).float() * w.sum()).sum() + w.square().sum(), (x[0], w), create_graph=True)
    second, = torch.autograd.grad(g[1].sum(), w, retain_graph=True)          # of w's own terms: nothing of the attention's backward
    assert torch.equal(second, torch.full_like(w, 2.0))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("create_graph", [False, True])
def test_under_a_checkpoint(device, name, create_graph):
    """What a recomputed function saved can be read once only."""
    from torch.utils.checkpoint import checkpoint
    f, x = make(name, device, True)
    plain = torch.autograd.grad(f(*x).float().square().sum(), x)
    again = torch.autograd.grad(checkpoint(f, *x, use_reentrant=False).float().square().sum(), x, create_graph=create_graph)
    assert all(torch.equal(a, b) for a, b in zip(plain, again))
