"""A lookup in a weight with a forward-mode derivative is refused, where it would return rows without one."""
import pytest
import torch
import torch.autograd.forward_ad as forward

import paper_2507_11941_amd as bpe


def test_refusal():
    weight, ids = torch.ones(5, 3), torch.zeros(4, dtype=torch.int32)
    with forward.dual_level():
        for recorded in (False, True):
            with torch.set_grad_enabled(recorded), pytest.raises(ValueError, match="forward-mode"):
                bpe.embed_tokens(forward.make_dual(weight, torch.ones_like(weight)), ids)


@pytest.mark.gpu
def test_an_ordinary_weight_beside_dual_tensors():
    dev = torch.device("cuda:0")
    weight, ids = torch.randn(5, 3, device=dev), torch.tensor([4, 0, 3], dtype=torch.int32, device=dev)
    with forward.dual_level():
        forward.make_dual(torch.ones(2, device=dev), torch.ones(2, device=dev))
        assert torch.equal(bpe.embed_tokens(weight, ids), weight[ids.long()])
