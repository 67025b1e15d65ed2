"""Paged attention counts every key of a request once.  With q = 0 and no bias every key weighs exactly 1, so lse is the logarithm of
the number of keys seen; the values are signs that mark the key's place, so that out times that number is a small whole number in
each channel, and another one where a step of keys is lost, repeated, or taken for another.  And random scores against bounds
that follow from the depth of the kernel's sums."""
import math

import numpy as np
import pytest
import torch

from paper_2505_12044_amd import api
from tests._paged_util import HALF, gather, i32, make_cache, randn

BF, F32 = torch.bfloat16, torch.float32


def masks(B, Hkv, C, seed=5):
    """A key's sign in channel c of head h of request b is (-1) to the number of bits that its position shares with the mask.
    The lowest bit of a mask, 1 to 128, is the most that signs 0..n - 1 can add up to; the bits above it are random."""
    rng = np.random.default_rng(seed)
    low = 1 << np.array([0, 2, 4, 5, 6, 6, 6] + [7] * 9)[np.arange(C) % 16]
    return (rng.integers(0, 1 << 15, (B, Hkv, C)) & ~(2 * low - 1)) | low


def signs(mask, n):
    x = np.arange(n)[:, None] & mask                               # [n, C]
    for s in (16, 8, 4, 2, 1):
        x = x ^ (x >> s)
    return 1 - 2 * (x & 1)


def test_marks_tell_every_step_from_every_other():
    """The oracle with keys left out, taken twice, or one step in another's place is outside the bounds used below."""
    n = 20000
    for C in (16, 128):
        for step in (16, 32, 64):
            sums = signs(masks(1, 1, C)[0, 0], n // step * step).reshape(-1, step, C).sum(1)         # of the steps, [steps, C]
            assert (np.abs(sums).max(1) > 2 * 128 * 2.0 ** -8 * 1.01).all()                          # one lost, or twice
            # one in another's place: steps of the same sums could be taken for each other, and they are few
            assert len({r.tobytes() for r in sums}) >= (0.9 if C == 128 else 0.5) * len(sums)
        assert np.abs(np.cumsum(signs(masks(1, 1, C)[0, 0], n), 0)).max() <= 128
    assert math.log(n / (n - 1)) > 2 * (math.log(n) + 1) * 2.0 ** -22                               # one key, in lse


def marked(lens, Hkv, page, C, dtype, R, room):
    c = make_cache(lens, Hkv, page, C, R, dtype, F32, 3, extra_blocks=room)
    table, m = c["table"].cpu().numpy(), masks(len(lens), Hkv, C)
    v = c["v_pages"].cpu()
    for b, n in enumerate(lens):
        if n:
            s = np.stack([signs(m[b, h], n) for h in range(Hkv)], 1)                                 # [n, Hkv, C]
            t = np.arange(n)
            v[torch.from_numpy(table[b, t // page]).long(), :, torch.from_numpy(t % page)] = torch.from_numpy(s).to(dtype)
    c["v_pages"] = v.cuda()
    if R:
        c["phi_pages"] = torch.nan_to_num(c["phi_pages"]) * 0 + 3.0
    return c, m


def count(lens, N, H, Hkv, C, page, dtype=BF, R=0, alibi=False, causal=True, room=1, workspace=True):
    lens = [int(n) for n in lens]
    c, m = marked(lens, Hkv, page, C, dtype, R, room)
    B, dev = len(lens), "cuda"
    q = torch.zeros((B, H, N, C), dtype=dtype, device=dev)
    kw = {} if workspace else {"out": torch.full_like(q, 7.0), "lse": torch.full((B, H, N), 7.0, device=dev)}
    # a cleared factor or slope: the bias is 0, the kernel another one
    phi_q = torch.zeros((B, H, N, R), device=dev) if R else None
    slopes = torch.zeros(H, device=dev) if alibi else None
    o, l = api.fb_paged_attn_fwd(q, c["k_pages"], c["v_pages"], c["table"], c["lens"], None, phi_q, c["phi_pages"], slopes, causal=causal, **kw)
    torch.cuda.synchronize()
    o, l = o.double().cpu().numpy().reshape(B, Hkv, H // Hkv, N, C), l.double().cpu().numpy().reshape(B, Hkv, H // Hkv, N)
    for b, n in enumerate(lens):
        total = np.stack([np.cumsum(np.concatenate((np.zeros((1, C)), signs(m[b, h], n))), 0) for h in range(Hkv)])      # [Hkv, n + 1, C]
        for i in range(N):
            seen = max(n - N + i + 1, 0) if causal else n
            if seen == 0:
                assert (o[b, :, :, i] == 0).all() and (l[b, :, :, i] == -math.inf).all()
                continue
            # the sums are whole numbers below 2^24, exact; then a reciprocal and a product (2^-22), the result's rounding, and a
            # logarithm in fp32
            want = total[:, None, seen]
            assert (np.abs(o[b, :, :, i] * seen - want) <= np.abs(want) * (HALF[dtype] * 1.01 + 2.0 ** -22)).all(), (b, n, i)
            assert (np.abs(l[b, :, :, i] - math.log(seen)) <= (math.log(seen) + 1) * 2.0 ** -22).all(), (b, n, i)


LENGTHS = [1, 31, 33, 639, 1025, 2049, 9001, 20000]


@pytest.mark.gpu
@pytest.mark.parametrize("C", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("workspace", [True, False])
def test_every_length(C, dtype, page, workspace):
    for n in LENGTHS:
        print(f"[count] {n} keys", flush=True)
        count([n], 1, 4, 2, C, page, dtype, workspace=workspace)
    count(LENGTHS, 3, 4, 2, C, page, dtype, workspace=workspace)


@pytest.mark.gpu
@pytest.mark.parametrize("C,dtype", [(64, BF), (128, BF), (64, F32), (16, BF)])
@pytest.mark.parametrize("R,alibi", [(2, False), (16, False), (21, False), (0, True)])
def test_every_bias(C, dtype, R, alibi):
    for n in (700, 2049, 9001):
        count([n, 50], 2, 4, 2, C, 32, dtype, R, alibi, causal=n > 2000)


@pytest.mark.gpu
@pytest.mark.parametrize("B", [3, 64, 65, 257, 600])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_ragged_batches_in_a_wide_table(B, dtype):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 300, B)
    lens[B // 2] = 20000 if B < 100 else 3000
    count(lens, 1, 4, 2, 32, 16, dtype)
    count(rng.integers(0, 40, B), 1, 2, 1, 16, 16, dtype, room=300)


@pytest.mark.gpu
@pytest.mark.parametrize("C", [64, 128])
@pytest.mark.parametrize("G,N", [(4, 5), (1, 17), (1, 33), (20, 1), (4, 16)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("workspace", [True, False])
def test_more_rows_than_a_tile(C, G, N, causal, workspace):
    # by the table's width the two-tile kernel, and one whose groups have as many steps as in earnest
    count([9001, 1, 20000, 300], N, 2 * G, 2, C, 256, causal=causal, room=400, workspace=workspace)
    count([2049, 640, 33], N, 2 * G, 2, C, 64, causal=causal, workspace=workspace)


@pytest.mark.gpu
def test_more_groups_than_waves():
    rng = np.random.default_rng(1)
    count(rng.integers(0, 60, 700), 1, 8, 8, 128, 16, room=60)           # a group is a wave's whole share, or several are
    count(rng.integers(200, 1500, 300), 2, 8, 8, 32, 256)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2049, 9001, 20000])
@pytest.mark.parametrize("C,dtype", [(64, BF), (128, BF), (32, BF), (64, F32)])
@pytest.mark.parametrize("workspace", [True, False])
def test_random_scores_within_the_depth_of_the_sums(n, C, dtype, workspace):
    c = make_cache([n], 2, 64, C, 0, dtype, F32, n)
    q = randn(torch.Generator().manual_seed(8), (1, 2, 1, C), dtype)
    kw = {} if workspace else {"out": torch.empty_like(q), "lse": torch.empty((1, 2, 1), device="cuda")}
    o, l = api.fb_paged_attn_fwd(q, c["k_pages"], c["v_pages"], c["table"], c["lens"], **kw)
    torch.cuda.synchronize()
    k, v = (gather(c[x], c["table"], 0, n) for x in ("k_pages", "v_pages"))
    x = q[0].double().cpu()
    s, size = (k @ x.transpose(1, 2))[..., 0] * C ** -0.5, (k.abs() @ x.abs().transpose(1, 2)).amax((1, 2)) * C ** -0.5
    p, lse = s.softmax(-1), s.logsumexp(-1)
    out = (p[..., None] * v).sum(1)
    # Of a chain of sums each adds 2^-24.  In one workgroup of four waves (or eight) of W keys a step, n / (4 W) steps of W / 4 sums a
    # lane, n / 16 in all; with its own share a wave has two steps, of up to 64 keys, and a group's parts, at most n / 32, are joined
    # eight at a time.  A step that raises the maximum adds four roundings.  Then lanes, waves and the ends.
    steps = n / 64 if not workspace else 4
    depth = (n / 16 if not workspace else 64 + n / 256) + 4 * steps + 64
    dp = 2 * (C + 80) * 2.0 ** -24 * size + depth * 2.0 ** -24 + (2.0 ** -16 if dtype == BF else 0)
    over = (o[0, :, 0].double().cpu() - out).abs() / (2 * dp[:, None] * (p[..., None] * v.abs()).sum(1) + out.abs() * HALF[dtype])
    over_l = (l[0, :, 0].double().cpu() - lse).abs() / (dp + (lse.abs() + 1) * 2.0 ** -22)
    print(f"[paged] out at {over.max():.3f}, lse at {over_l.max():.3f} of the bound", flush=True)
    assert over.max() <= 1 and over_l.max() <= 1
    assert (2 * dp < math.log(n / (n - 32))).all()                        # 32 keys of mean weight are seen in lse
