"""Paged attention over a table as wide as positions go (2^31 tokens), where few entries are pages: the last keys are found and
the walk ends, with the keys split over the GPU and in one workgroup."""
import pytest
import torch

from paper_2505_12044_amd import api
from tests._paged_util import HALF, i32, randn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("split", [True, False])
def test_the_longest_length(split):
    C, page, blocks = 16, 256, 1 << 23
    g = torch.Generator().manual_seed(1)
    k, v = (randn(g, (4, 1, page, C), BF) for _ in range(2))
    q = randn(g, (1, 1, 1, C), BF)
    table = torch.full((1, blocks), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, 1 << 20], table[0, blocks - 2], table[0, blocks - 1] = 2, 0, 3, 1        # the last lies behind 2^31 - 256
    kw = {} if split else {"out": torch.empty_like(q), "lse": torch.empty((1, 1, 1), device="cuda")}
    print(f"[paged] 2^31 keys, split {split}", flush=True)
    o, l = api.fb_paged_attn_fwd(q, k, v, table, i32([(1 << 31) - 1]), causal=False, **kw)
    torch.cuda.synchronize()
    kd, vd = (x[[2, 0, 3], 0].flatten(0, 1).double().cpu() for x in (k, v))
    s = kd @ q[0, 0, 0].double().cpu() / 4
    size = (kd.abs() @ q[0, 0, 0].abs().double().cpu()).max().item() / 4
    p = s.softmax(0)
    # scores: 16 products and sums and the exponent's argument in fp32; sums over 768 keys; two bf16 limbs
    dp = 2 * (C + 80) * 2.0 ** -24 * size + 784 * 2.0 ** -23 + 2.0 ** -16
    ref = p @ vd
    assert ((o[0, 0, 0].double().cpu() - ref).abs() <= ref.abs() * HALF[BF] + 2 * dp * (p @ vd.abs())).all()
    assert abs(l.item() - s.logsumexp(0).item()) <= dp + (abs(s.logsumexp(0).item()) + 1) * 2.0 ** -22
