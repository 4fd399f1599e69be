"""Tensors with a forward-mode derivative: the operators at a model's output end refuse them, where they would return results without one."""
import pytest
import torch
import torch.autograd.forward_ad as forward

import paper_2507_11941_amd as bpe


def calls(dev, dual):
    """Every call, with one tensor after another that `dual` makes of an ordinary one."""
    x, w, v = torch.ones(3, 6, device=dev), torch.ones(6, device=dev), torch.ones(3, device=dev)
    q, head = torch.ones(3, 6, dtype=torch.int8, device=dev), torch.ones(9, 6, dtype=torch.int8, device=dev)
    ids, at = torch.ones(3, dtype=torch.int32, device=dev), torch.zeros(3, dtype=torch.int64, device=dev)
    return [lambda: bpe.add_norm(dual(x), w, x), lambda: bpe.add_norm(x, dual(w), x), lambda: bpe.add_norm(x, w, dual(x)),
            lambda: bpe.add_norm_8bit(dual(x), w, x), lambda: bpe.add_norm_8bit(x, dual(w), x), lambda: bpe.add_norm_8bit(x, w, dual(x)),
            lambda: bpe.quantize_rows(dual(x)), lambda: bpe.project_8bit(q, dual(v), head, torch.ones(9, device=dev)),
            lambda: bpe.project_8bit(q, v, head, dual(torch.ones(9, device=dev))),
            lambda: bpe.add_norm_grad(dual(x), x, w, v, x), lambda: bpe.add_norm_grad(x, dual(x), w, v, x), lambda: bpe.add_norm_grad(x, x, dual(w), v, x),
            lambda: bpe.add_norm_grad(x, x, w, dual(v), x), lambda: bpe.add_norm_grad(x, x, w, v, dual(x)),
            lambda: bpe.adjust_logits(dual(x), ids, at, at), lambda: bpe.adjust_logits(x, ids, at, at, dual(x[:, :3].contiguous())),
            lambda: bpe.adjust_logits(x, bias=(ids, dual(v), at, at)), lambda: bpe.adjust_logits_grad(dual(x), x, ids, at, at),
            lambda: bpe.adjust_logits_grad(x, dual(x), ids, at, at), lambda: bpe.adjust_logits_grad(x, x, ids, at, at, dual(x[:, :3].contiguous()))]


@pytest.mark.parametrize("recorded", [False, True])
def test_refusals(recorded):
    """Before anything else is looked at, so that it can be seen without a GPU."""
    with forward.dual_level(), torch.set_grad_enabled(recorded):
        for call in calls("cpu", lambda t: forward.make_dual(t, torch.ones_like(t))):
            with pytest.raises(ValueError, match="forward-mode"):
                call()


@pytest.mark.gpu
def test_ordinary_tensors_beside_dual_ones():
    want = [call() for call in calls("cuda:0", lambda t: t)]
    with forward.dual_level():
        other = forward.make_dual(torch.ones(2, device="cuda:0"), torch.ones(2, device="cuda:0"))
        for call, results in zip(calls("cuda:0", lambda t: t), want):
            for a, b in zip(*(r if isinstance(r, tuple) else (r,) for r in (call(), results))):
                assert torch.equal(a, b)
        for call in calls("cuda:0", lambda t: forward.make_dual(t, torch.ones_like(t))):
            with pytest.raises(ValueError, match="forward-mode"):
                call()
        assert forward.unpack_dual(other).tangent is not None
