"""A step of PagedCache that is refused leaves the cache as it was; sizes that no step could take are refused at once."""
import pytest
import torch

from paper_2505_12044_amd import api
from paper_2505_12044_amd.paged import PagedCache


def refused(new_lens_like, b):
    """Arguments that step refuses, for a cache of b requests."""
    ok = torch.full((b,), 3, dtype=torch.int32, device=new_lens_like)
    return [(ok.long(), 1), (ok.float(), 1), (ok[:-1], 1), (torch.cat((ok, ok)), 1), (ok[:, None], 1), (torch.cat((ok, ok))[::2], 1),
            (ok, 0), (ok, -1), (ok, 1 << 31)]


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_a_refused_step_changes_nothing(device):
    cache = PagedCache(1, 3, 1, 16, 16, 8, 64, device=device)
    if device == "cuda":
        cache.step(torch.tensor([5, 0, 20], dtype=torch.int32, device=device), 20)
        cache.step(torch.tensor([6, 2, 21], dtype=torch.int32, device=device), 2)
    else:                                  # on the host every step is refused
        cache._now.copy_(torch.tensor([6, 2, 21, 4, 4]))
        cache._before.copy_(torch.tensor([5, 0, 20, 3, 5]))
    names = ("_now", "_before", "table", "ring", "slots", "positions")
    held = {n: getattr(cache, n) for n in names}
    copies = {n: None if t is None else t.clone() for n, t in held.items()}
    more = [(torch.full((3,), 4, dtype=torch.int32), 1)]                     # a host tensor
    for new_lens, n_new in refused(device, 3) + more:
        with pytest.raises(api.FlashBiasError):
            cache.step(new_lens, n_new)
        for n in names:
            assert getattr(cache, n) is held[n] and (held[n] is None or torch.equal(held[n], copies[n])), n
    assert cache.starts.tolist() == [5, 0, 20] and cache.lens.tolist() == [6, 2, 21]


def test_sizes_that_no_step_takes():
    for kw in (dict(requests=4097), dict(n_pages=1 << 27), dict(requests=4096, max_tokens=1 << 24)):
        with pytest.raises(api.FlashBiasError):
            PagedCache(**{**dict(layers=1, requests=2, kv_heads=1, head_dim=16, page=16, n_pages=8, max_tokens=64, device="meta"), **kw})
    assert PagedCache(1, 4096, 1, 16, 16, 8, 64, device="meta").lens.shape == (4096,)
