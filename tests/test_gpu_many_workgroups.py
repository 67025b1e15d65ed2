"""Calls of more work than one launch takes (2^32 threads): rotary positions of odd pairs, append of rows at odd starts, attention
of many short requests.  Rows overlap in memory, or lie in few pages, where that keeps the inputs small."""
import pytest
import torch

from paper_2505_12044_amd import api
from tests._paged_util import HALF, i32, randn

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def test_rotary_of_2_26_tokens():
    B, N, C, P = 17, 1 << 22, 128, 63                    # 64 threads a token
    g = torch.Generator().manual_seed(1)
    base = randn(g, (C + B * N,), BF)
    x = base.as_strided((B, 1, N, C), (N, 0, 1, 1))      # row t begins at element t
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[None, None]
    f = torch.tensor([10000.0 ** (-p / P) for p in range(P)], dtype=F32).cuda()
    print("[rotary] 71 million tokens", flush=True)
    y, _ = api.fb_rotary_fwd(x, None, pos, f, (P,))
    torch.cuda.synchronize()
    tokens = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, N - 1])
    for b in range(B):
        raw = x[b, 0][tokens.cuda()].double().cpu()
        angle = tokens[:, None].double() * f.double().cpu()
        c, s = angle.cos(), angle.sin()
        x1, x2 = raw[:, :P], raw[:, P:2 * P]
        want = torch.cat((x1 * c - x2 * s, x2 * c + x1 * s, raw[:, 2 * P:]), -1)
        size = (x1.abs() + x2.abs()) * (2.0 ** -21 + angle.abs() * 2.0 ** -51)
        tol = torch.cat((size, size, torch.zeros(len(tokens), C - 2 * P)), -1) + want.abs() * HALF[BF] * (1 + 2.0 ** -10)
        assert ((y[b, 0][tokens.cuda()].double().cpu() - want).abs() <= tol).all(), b
    # nothing was left out: each row's last two channels are copies, spread over all of the result
    assert torch.equal(y[..., 2 * P:], x[..., 2 * P:])


def test_append_of_2_25_tokens():
    B, N, C, page = 9, 1 << 22, 128, 16                   # 128 threads a token
    g = torch.Generator().manual_seed(2)
    base = randn(g, (C + 1 + B * N,), BF)
    k = base[1:].as_strided((B, 1, N, C), (N, 0, 1, 1))
    v = base.as_strided((B, 1, N, C), (N, 0, 1, 1))
    slots = torch.full((B, N), -1, dtype=torch.int32, device="cuda")
    places = [(b, n) for b in range(B) for n in (0, 1 << 19, N - 1)]
    for i, (b, n) in enumerate(places):
        slots[b, n] = i
    pages = -(-len(places) // page)
    kp, vp = (torch.zeros((pages, 1, page, C), dtype=BF, device="cuda") for _ in range(2))
    print("[append] 38 million tokens", flush=True)
    api.fb_paged_append(k, v, slots, kp, vp)
    torch.cuda.synchronize()
    for i, (b, n) in enumerate(places):
        assert torch.equal(kp[i // page, 0, i % page], k[b, 0, n]) and torch.equal(vp[i // page, 0, i % page], v[b, 0, n]), (b, n)


def test_attention_of_2_24_groups():
    B, H, C, page = (1 << 20) + 5, 16, 16, 16              # a workgroup of 256 threads for each request and head
    g = torch.Generator().manual_seed(3)
    kp, vp = (randn(g, (7, H, page, C), BF) for _ in range(2))
    q = randn(g, (1, H, 1, C), BF).expand(B, H, 1, C).contiguous()
    table = (torch.arange(B, dtype=torch.int32, device="cuda") % 7)[:, None].contiguous()
    lens = (torch.arange(B, dtype=torch.int32, device="cuda") % 17)
    print("[paged] 17 million groups", flush=True)
    o, l = api.fb_paged_attn_fwd(q, kp, vp, table, lens, causal=False, out=torch.full_like(q, 9.0), lse=torch.full((B, H, 1), 9.0, device="cuda"))
    torch.cuda.synchronize()
    # requests of one page and length are the same: 7 * 17 of them, checked against each other and against a small call
    few, few_l = api.fb_paged_attn_fwd(q[:119].contiguous(), kp, vp, table[:119].contiguous(), lens[:119].contiguous(), causal=False)
    torch.cuda.synchronize()
    whole = B // 119 * 119
    assert torch.equal(o[:whole].unflatten(0, (-1, 119)), few.expand(whole // 119, *few.shape))
    assert torch.equal(l[:whole].unflatten(0, (-1, 119)), few_l.expand(whole // 119, *few_l.shape))
    assert torch.equal(o[whole:], few[:B - whole]) and torch.equal(l[whole:], few_l[:B - whole])
