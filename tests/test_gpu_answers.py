"""The example that continues prompts: it runs, its answers keep to the grammar, and what trains it has the formulas' gradients."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_it_runs():
    import answer_strings

    losses, answers = answer_strings.main(steps=8, length=6)
    assert len(losses) == 8 and all(x == x for x in losses)
    assert len(answers) == 8
    for _, answer in answers:
        assert answer.endswith(b".") and all(c in b" abcdefghijklmnopqrstuvwxyz" for c in answer[:-1])


def test_gradients():
    """All parameters' gradients against torch's, of the same model in 64 bits.

    The loss's gradient is O(1) in every logit; 32-bit products over 64 columns and sums over 300 tokens are off by some 64 + 300 roundings of
    2^-24 of their terms' magnitudes, 3e-5, which is compared with the largest element of each gradient."""
    import answer_strings
    import paper_2507_11941_amd as bpe

    dev = torch.device("cuda:0")
    vocab, n = 70, 300
    model = answer_strings.Model(vocab, 64, dev)
    ids = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(dev)
    upstream = torch.randn(n, vocab, generator=torch.Generator().manual_seed(2)).to(dev)
    model(ids).backward(upstream)
    got = [p.grad.double().cpu() for p in model.parameters()]
    e, b, g, h = (p.detach().double().cpu().requires_grad_() for p in model.parameters())
    x = e[ids.cpu().long()]
    s = x + torch.relu(x @ b)
    logits = s / (s.square().mean(1, keepdim=True) + 1e-6).sqrt() * g @ h.t()
    logits.backward(upstream.double().cpu())
    for a, p in zip(got, (e, b, g, h)):
        assert float((a - p.grad).abs().max()) < 3e-5 * float(p.grad.abs().max())
    assert bpe.embed_tokens(model.embedding, ids).requires_grad
