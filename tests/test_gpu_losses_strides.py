"""Both losses on logits that lie with a stride and an odd beginning, into gradients that lie otherwise, and in place: against 64
bits, each element of the gradient by its own size, and the same bits wherever it goes."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from ops_reference import LOG_SUM, TYPES, U, assert_near
from test_gpu_logits import dev, some_logits
from test_gpu_losses import batch_of, up

pytestmark = pytest.mark.gpu

CASES = [(13, 13, 1), (1256, 1257, 0), (1001, 1003, 3), (1256, 1264, 8), (32256, 32261, 7), (33001, 33024, 5), (100260, 100267, 1), (8, 11, 2)]


def batch(vocab):
    """(ids, offsets, targets on the GPU and on the host); the first row is scored, but in no string."""
    import paper_2507_11941_amd as bpe

    ids, offsets, first = batch_of([5, 7, 0, 6], vocab, 3, 1, 2)
    targets = bpe.next_tokens(up(ids), up(offsets), up(first))
    targets[0] = 1
    return offsets, targets, targets.cpu()


def every_way(call, make, want, hidden):
    """call(logits, out): into other strides and beginnings, with nothing written between the rows; and in the logits' place."""
    x = make()
    n, vocab = x.shape
    for stride, at in ((vocab + 3, 1), (vocab + 8, 0), (vocab, 5), (x.stride(0), 0)):
        memory = torch.full((at + n * stride + 8,), 9.0, dtype=x.dtype, device=dev())
        out = memory.as_strided((n, vocab), (stride, 1), at)
        got = call(x, out)
        assert got[-1] is out and all(torch.equal(a, b) for a, b in zip(got, want)), (stride, at)
        out.fill_(9.0)
        assert (memory == 9).all(), "written between the rows"
    y = make()
    memory = y.as_strided((y.untyped_storage().nbytes() // y.element_size(),), (1,), 0)
    between = torch.ones_like(memory, dtype=torch.bool)
    between.as_strided(y.shape, y.stride(), y.storage_offset()).fill_(False)
    before = memory.clone()
    got = call(y, y)
    assert all(torch.equal(a, b) for a, b in zip(got, want)), "in place"
    assert torch.equal(memory[between], before[between]), "written between the rows"
    # Rows that are not scored hold anything.
    y = make()
    y[hidden] = float("nan")
    assert y.stride() == x.stride() and all(torch.equal(a, b) for a, b in zip(call(y, None), want)), "rows that are not scored"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,stride,at", CASES)
def test_preference(dtype, vocab, stride, at):
    import paper_2507_11941_amd as bpe

    offsets, targets, t = batch(vocab)
    n, beta, smoothing, scale = len(t), 0.25, 0.125, 64.0

    def make():
        return some_logits(n, vocab, TYPES[dtype], 1, stride, at)

    x = make()
    assert x.stride() == (stride, 1) and x.storage_offset() == at
    lp, _ = ref.logprobs(x, t)
    reference = (lp + torch.randn(n, generator=torch.Generator().manual_seed(5)).double()).float()

    def call(logits, out):
        return bpe.preference_loss(logits, targets, up(offsets), reference.to(dev()), beta, smoothing, scale, out=out)

    leaf = lp.clone().requires_grad_()
    want_loss, want_z = ref.preference(leaf, t, offsets, vocab, reference, beta, smoothing)
    want_loss.backward()
    upstream = leaf.grad * scale
    loss, margins, got_lp, grad = want = call(x, None)
    far = beta * (n * LOG_SUM + U * lp.abs().sum())
    assert_near(got_lp, lp, LOG_SUM, "logprobs")
    assert_near(margins, want_z.detach(), far, "margins")
    assert_near(loss, want_loss.detach(), far + 4 * U, "loss")
    want_grad, off = ref.logits_grad(x, t, upstream)
    element = ref.logits_grad(x, t, torch.ones(n))[0].abs()
    inside = (ref.strings_of(n, offsets) >= 0)[:, None]
    slope = scale * beta / 2 * far / 4 + 4 * U * upstream.abs()[:, None]
    assert_near(grad, want_grad, off + inside * slope * element, "gradient")
    every_way(call, make, want, (t < 0).to(dev()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,stride,at", CASES)
@pytest.mark.parametrize("per,kl_weight", [("token", 0.0), ("string", 0.05)])
def test_policy(dtype, vocab, stride, at, per, kl_weight):
    import paper_2507_11941_amd as bpe

    offsets, targets, t = batch(vocab)
    n, strings, scale = len(t), len(offsets) - 1, 64.0
    low, high, kl = (float(np.float32(v)) for v in (0.2, 0.28, kl_weight))

    def make():
        return some_logits(n, vocab, TYPES[dtype], 1, stride, at)

    x = make()
    lp, _ = ref.logprobs(x, t)
    g = torch.Generator().manual_seed(6)
    away = (0.4 * torch.randn(n, generator=g).double()).clamp(-1.0, 1.0)
    for bound in (1 - low, 1 + high):                    # no ratio within 1e-3 of a bound, where there is no derivative
        away = torch.where((away.exp() - bound).abs() < 1e-3, 0.0, away)
    old = (lp - away).float()
    reference = (lp + (0.5 * torch.randn(n, generator=g).double()).clamp(-1.0, 1.0)).float()
    advantages = torch.randn(n, generator=g).clamp(-3.0, 3.0)

    def call(logits, out):
        return bpe.policy_loss(logits, targets, up(offsets), old.to(dev()), advantages.to(dev()), reference.to(dev()), low, high, kl, per, scale,
                               out=out)

    leaf = lp.clone().requires_grad_()
    want_loss = ref.policy(leaf, t, offsets, vocab, old, advantages, reference if kl else None, low, high, kl, per == "string")
    want_loss.backward()
    upstream = leaf.grad * scale
    loss, got_lp, grad = want = call(x, None)
    string = ref.strings_of(n, offsets)
    inside = (t >= 0) & (string >= 0)
    assert_near(got_lp, torch.where(inside, lp, 0.0), LOG_SUM, "logprobs")
    # Of a token: |ratio A| and |kl (e^d - 1)|, each with relative errors of the log-probability's and 8 U more.
    near = LOG_SUM + U * lp.abs().max() + 8 * U
    size = 3 * np.e + kl * np.e
    assert_near(loss, want_loss.detach(), size * near, "loss")
    share = torch.zeros(n, dtype=torch.float64)
    for i in range(strings):
        rows = inside & (string == i)
        share[rows] = 1 / (strings * max(1, int(rows.sum()))) if per == "string" else 1 / int(inside.sum())
    want_grad, off = ref.logits_grad(x, t, upstream)
    element = ref.logits_grad(x, t, torch.ones(n))[0].abs()
    assert_near(grad, want_grad, off + (scale * share * size * near)[:, None] * element, "gradient")
    every_way(call, make, want, (t < 0).to(dev()))
