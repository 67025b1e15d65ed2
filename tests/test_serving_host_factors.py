"""Factors shared over the batch in the paged operators: the shape decides, and a flag that contradicts it is refused (on the
host: nothing is launched)."""
import pytest
import torch

from paper_2505_12044_amd import api

BF = torch.bfloat16


def calls(batch_q, batch_phi, flag):
    q = torch.zeros((batch_q, 2, 1, 64), dtype=BF)
    phi = torch.zeros((batch_phi, 2, 1, 3))
    pages, phi_pages = torch.zeros((4, 2, 16, 64), dtype=BF), torch.zeros((4, 2, 16, 3))
    ints = torch.zeros((batch_q, 4), dtype=torch.int32)
    yield lambda: api.fb_paged_append(q, q, ints[:, :1], pages, pages, phi, phi_pages, phi_batch_broadcast=flag)
    yield lambda: api.fb_paged_attn_fwd(q, pages, pages, ints, ints[:, 0], phi_q=phi, phi_pages=phi_pages, phi_batch_broadcast=flag)


@pytest.mark.parametrize("batch_q,batch_phi,flag", [(3, 1, False), (3, 3, True)])
def test_a_flag_against_the_shape_is_refused(batch_q, batch_phi, flag):
    for call in calls(batch_q, batch_phi, flag):
        with pytest.raises(api.FlashBiasError, match="contradicts"):
            call()


@pytest.mark.parametrize("batch_q,batch_phi,flag", [(3, 1, True), (3, 1, None), (3, 3, False), (3, 3, None), (1, 1, True), (1, 1, False), (1, 1, None)])
def test_a_flag_that_agrees_is_taken(batch_q, batch_phi, flag):
    for call in calls(batch_q, batch_phi, flag):
        with pytest.raises(api.FlashBiasError, match="CUDA tensors"):        # the next check: these are host tensors
            call()


def test_the_shape_decides():
    one, three = torch.zeros((1, 2, 1, 3)), torch.zeros((3, 2, 1, 3))
    assert api._shared_factors(one, 3, None) and api._shared_factors(one, 3, True)
    assert not api._shared_factors(three, 3, None) and not api._shared_factors(three, 3, False)
    assert not api._shared_factors(one, 1, True) and not api._shared_factors(one, 1, False)
