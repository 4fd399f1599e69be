"""The operators beside torch's automatic differentiation: a lookup in a weight that wants a gradient is recorded; what returns a
gradient itself is not."""
import pytest
import torch

from test_gpu_embed import dev, matrix, some_ids
from test_gpu_logits import some_logits, some_targets, some_upstream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("side", [False, True])
@pytest.mark.parametrize("count", [None, 0, 30, 99])
def test_lookup_in_a_weight_that_wants_a_gradient(dtype, side, count):
    import paper_2507_11941_amd as bpe

    n, vocab, dim = 50, 17, 33
    weight, ids = matrix(vocab, dim, dtype, 1).requires_grad_(), some_ids("padded", n, vocab, 2).to(dev())
    counted = None if count is None else torch.tensor([count], device=dev())
    used = n if count is None else min(n, count)
    more = {}
    if side:
        more["stream"] = torch.cuda.Stream()
        more["stream"].wait_stream(torch.cuda.current_stream())
    x = bpe.embed_tokens(weight, ids, 0.5, counted, **more)
    torch.cuda.synchronize()
    assert x.requires_grad and torch.equal(x[:used], bpe.embed_tokens(weight.detach(), ids, 0.5)[:used])
    g = matrix(n, dim, dtype, 3)
    x.backward(g)
    torch.cuda.synchronize()
    want = bpe.embed_tokens_grad(g, ids, vocab, 0.5, counted)
    assert weight.grad.dtype == dtype and torch.equal(weight.grad, want)
    # a gradient whose rows share their memory, and one that lies by columns
    for g in (torch.ones(1, 1, dtype=dtype, device=dev()).expand(n, dim), matrix(dim, n, dtype, 3).t()):
        weight.grad = None
        bpe.embed_tokens(weight, ids, 0.5, counted).backward(g)
        assert torch.equal(weight.grad, bpe.embed_tokens_grad(g.contiguous(), ids, vocab, 0.5, counted))


def test_lookup_that_is_not_recorded():
    import paper_2507_11941_amd as bpe

    weight, ids = matrix(17, 33, torch.float32, 1).requires_grad_(), some_ids("padded", 50, 17, 2).to(dev())
    with torch.no_grad():
        out = torch.empty(50, 33, device=dev())
        x = bpe.embed_tokens(weight, ids, out=out)
        assert x is out and not x.requires_grad and not bpe.embed_tokens(weight, ids).requires_grad
    with torch.inference_mode():
        assert torch.equal(bpe.embed_tokens(weight, ids, out=torch.empty(50, 33, device=dev())), out)
    assert not bpe.embed_tokens(weight.detach(), ids).requires_grad
    with pytest.raises(ValueError):
        bpe.embed_tokens(weight, ids, out=out)           # (as torch's own functions)
    x = bpe.embed_tokens(weight, ids)
    ids[0] = 3
    with pytest.raises(RuntimeError):                    # what the gradient needs has changed
        x.sum().backward()


def test_an_embedding_is_trained_by_the_rest_of_a_model():
    """Whole numbers: exact in any order."""
    import paper_2507_11941_amd as bpe

    weight = torch.randint(-4, 5, (11, 6), device=dev()).float().requires_grad_()
    head = torch.randint(-4, 5, (6, 5), device=dev()).float()
    ids = some_ids("skewed", 40, 11, 2).to(dev())
    (bpe.embed_tokens(weight, ids, 2.0) @ head).sum().backward()
    got, weight.grad = weight.grad, None
    kept = (ids >= 0) & (ids < 11)
    (torch.where(kept[:, None], 2.0 * weight[torch.where(kept, ids, 0).long()], 0.0) @ head).sum().backward()
    assert torch.equal(got, weight.grad)


def test_logits_that_want_a_gradient_are_given_it_by_hand():
    import paper_2507_11941_amd as bpe

    n, vocab = 6, 40
    leaf, targets, upstream = some_logits(n, vocab, torch.float32, 1).requires_grad_(), some_targets(n, vocab, 2), some_upstream(n, 3)
    logits = leaf * 2.0
    lp, lse, grad = bpe.token_logprobs_and_grad(logits, targets, upstream)
    assert not (lp.requires_grad or lse.requires_grad or grad.requires_grad)
    logits.backward(grad)
    assert torch.equal(leaf.grad, grad * 2.0)
