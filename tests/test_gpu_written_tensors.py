"""Tensors that a call writes into are known to torch to be others afterwards: what has saved one for a gradient refuses to use it."""
import pytest
import torch

import workloads
from test_gpu_embed import dev, matrix, some_ids
from test_gpu_logits import some_logits, some_targets, some_upstream

pytestmark = pytest.mark.gpu


def test_what_is_written_is_another_tensor_afterwards():
    """Something that saved the logits for its own gradient does not use what has taken their place."""
    import paper_2507_11941_amd as bpe

    n, vocab = 6, 40
    targets, upstream = some_targets(n, vocab, 2), some_upstream(n, 3)
    offsets = torch.tensor([0, 3, n], device=dev())
    scores = torch.zeros(n, device=dev())
    for call in (lambda y: bpe.token_logprobs_and_grad(y, targets, upstream, out=y)[2], lambda y: bpe.token_logprobs_grad(y, targets, scores, upstream, out=y),
                 lambda y: bpe.preference_loss(y, targets, offsets, out=y)[-1], lambda y: bpe.policy_loss(y, targets, offsets, scores, scores + 1, out=y)[-1]):
        leaf = some_logits(n, vocab, torch.float32, 1).requires_grad_()
        logits = torch.tanh(leaf)                    # (its gradient is made of its result)
        before = logits._version
        with torch.no_grad():
            grad = call(logits)
        assert grad is logits and logits._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            logits.backward(torch.ones_like(logits))
        leaf = some_logits(n, vocab, torch.float32, 1).requires_grad_()
        logits = leaf * 2.0                              # (its gradient is not)
        grad = call(logits)
        want = call((leaf * 2.0).detach())
        logits.backward(grad.detach())
        assert torch.equal(leaf.grad, want * 2.0)
        with torch.inference_mode():                     # (there is nothing to tell)
            assert torch.equal(call(leaf * 2.0), want)
    ids = some_ids("padded", 50, 17, 2).to(dev())
    out, total, weight = torch.zeros(50, 3, device=dev()), torch.zeros(17, 3, device=dev()), matrix(17, 3, torch.float32, 1)
    following = torch.zeros_like(ids)
    before = [t._version for t in (out, total, following, weight, ids)]
    bpe.embed_tokens(weight, ids, out=out)
    bpe.embed_tokens_grad(out, ids, 17, out=total, accumulate=True)
    bpe.next_tokens(ids, torch.tensor([0, 50], device=dev()), out=following)
    after = [t._version for t in (out, total, following, weight, ids)]
    assert all(a > b for a, b in zip(after[:3], before)) and after[3:] == before[3:]


def test_ids_that_an_encoder_has_written_over():
    """The gradient of a lookup needs the ids that were looked up."""
    import paper_2507_11941_amd as bpe

    merges = workloads.load_merges("1k")
    table = bpe.build_table(merges)
    weight = torch.randn(256 + len(merges), 8, device=dev()).requires_grad_()
    data, ends = (torch.from_numpy(a).to(dev()) for a in workloads.batch(1))
    ids, offsets = bpe.encode_batch(table, data, ends, 256)
    for encode in (lambda: bpe.encode_batch(table, data, ends, 256, ids, offsets), lambda: bpe.encode_batch_static(table, data, ends, 256, ids, offsets)):
        x = bpe.embed_tokens(weight, ids, count=offsets[-1:])
        x.backward(torch.ones_like(x))
        for _ in range(2):
            x = bpe.embed_tokens(weight, ids, count=offsets[-1:])
            encode()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                x.backward(torch.ones_like(x))
