"""Penalties for all rows count as they were when the call was made."""
import pytest
import torch

from test_gpu_adjust import arguments, dev, logits_of, without_bias

pytestmark = pytest.mark.gpu


def test_a_list_that_changes_before_the_backward_pass():
    import paper_2507_11941_amd as bpe

    n, vocab = 5, 300
    more = {**without_bias(arguments("all", n, vocab, 4)), "penalties": [1.5, 0.5, 0.25]}
    logits, grad = logits_of(n, vocab, torch.float32, 1), logits_of(n, vocab, torch.float32, 2)
    want = bpe.adjust_logits_grad(grad, logits, **more)
    leaf = logits.clone().requires_grad_()
    got = bpe.adjust_logits(leaf, **more)
    more["penalties"][0] = 3.0
    got.backward(grad)
    assert torch.equal(leaf.grad, want) and not torch.equal(bpe.adjust_logits_grad(grad, logits, **more), want)
