"""The preference loss's gradient where a row's sum of exponentials is not to be had from a 32-bit logarithm of it: logits far from
0, rows of the type's lowest value, targets that are all but certain.  From 64 bits, each element by its own size."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from ops_reference import LOG_SUM, TYPES, U, assert_near
from test_gpu_logits import dev, some_logits

pytestmark = pytest.mark.gpu

BETA, SCALE = 0.25, 2.0


def check(x, lens, near=LOG_SUM, **more):
    """`near`: of a log-probability.  The factor of a row's gradient is off by a quarter of the margin's error at most, and this
    error goes into an element in the proportion of the element itself."""
    import paper_2507_11941_amd as bpe

    n, vocab = x.shape
    ends = np.concatenate([[0], np.cumsum(lens)])
    assert ends[-1] == n
    t = torch.arange(n, dtype=torch.int32) * 7 % vocab
    lp, _ = ref.logprobs(x, t)
    leaf = lp.clone().requires_grad_()
    ref.preference(leaf, t, ends, vocab, None, BETA, 0.0)[0].backward()
    upstream = leaf.grad * SCALE
    want, off = ref.logits_grad(x, t, upstream)
    element = (ref.logits_grad(x, t, torch.ones(n))[0]).abs()
    slope = SCALE * BETA / (len(lens) // 2) * BETA * (n * near + U * lp.abs().sum()) / 4 + 4 * U * upstream.abs()[:, None]
    _, _, got_lp, grad = bpe.preference_loss(x, t.to(dev()), torch.from_numpy(ends).to(dev()), None, BETA, 0.0, SCALE, **more)
    assert_near(got_lp, lp, near, "logprobs")
    assert_near(grad, want, off + slope * element, "gradient")
    return t, grad, upstream


@pytest.mark.parametrize("vocab", [7, 1000, 33001])
@pytest.mark.parametrize("shift", [0.0, 1e3, 1e4, 1e5, 1e6, -1e6])
def test_logits_far_from_zero(vocab, shift):
    """32-bit logits shifted together: what the shift leaves of them is what they are."""
    check(some_logits(11, vocab, torch.float32, 1) + shift, [2, 3, 1, 5])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [7, 1256, 100260])
def test_rows_of_the_lowest_value(dtype, vocab):
    """All logits the same: each has 1 / vocab, whatever they are; and one above the others by more than the type holds."""
    low = torch.finfo(TYPES[dtype]).min
    x = torch.full((6, vocab), low, dtype=TYPES[dtype], device=dev())
    x[1], x[3] = -low, 0.0
    x[2, 1:] = -float("inf")
    x[4, 3] = -low
    t = torch.arange(6) * 7 % vocab
    x[4, int(t[4])] = -low                               # (a target of probability 1/2, or 1)
    x[2, int(t[2])] = low
    check(x, [3, 3])


def test_targets_that_are_all_but_certain():
    """The target 14 above the others, at 200.  A lane's terms besides the target's have their relative errors; the target's 1 joins
    them by some 16 additions, each of which rounds by U at most.  So 1 - p is off by 24 U and 100 U of itself."""
    vocab, n = 1000, 4
    x = some_logits(n, vocab, torch.float32, 3, spread=0.5) + 186.0
    x[torch.arange(n), torch.arange(n) * 7 % vocab] = 200.0
    t, grad, upstream = check(x, [2, 2])
    d = x.double().cpu() - x.double().cpu().amax(1, keepdim=True)
    others = d.exp()
    others[torch.arange(n), t.long()] = 0
    left = others.sum(1) / (1 + others.sum(1))           # 1 - p
    assert (left > 1e-5).all() and (left < 1e-2).all()
    want = upstream * left
    got = grad.cpu().double()[torch.arange(n), t.long()]
    # (the factor is off by 4 U of itself and a quarter of the margin's error, n LOG_SUM BETA)
    assert ((got - want).abs() <= upstream.abs() * (24 * U + (104 * U + n * LOG_SUM * BETA) * left)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [33001, 32256])
def test_more_than_the_caches_hold(dtype, vocab):
    """Rows of a large batch against the one-pass gradient of some of them, whose factors follow from the margin."""
    import paper_2507_11941_amd as bpe

    size = torch.empty(0, dtype=TYPES[dtype]).element_size()
    n = 128_000_000 // (vocab * size) + 101
    x, t = some_logits(n, vocab, TYPES[dtype], 1), (torch.arange(n, dtype=torch.int32) * 7 % vocab).to(dev())
    middle = n // 2
    _, margins, lp, grad = bpe.preference_loss(x, t, torch.tensor([0, middle, n], device=dev()), None, 0.001, 0.1, 256.0)
    c = 256.0 * 0.001 * (0.1 - 1 / (1 + np.exp(margins.double().item())))
    for rows in (slice(0, 60), slice(middle - 30, middle + 30), slice(n - 60, n)):
        upstream = torch.where(torch.arange(n, device=dev())[rows] < middle, c, -c).float()
        few = bpe.token_logprobs_and_grad(x[rows], t[rows], upstream)
        assert torch.allclose(few[0], lp[rows], rtol=2 * U, atol=2 * LOG_SUM)
        # (each p off by U (102 + 2 |x - lse|) of itself, |x - lse| below 50, each rounded; the margin was rounded to 32 bits)
        bound = few[2].double().abs() * (torch.finfo(TYPES[dtype]).eps + 2 * 202 * U + 16 * U) + 2 * ref.SMALLEST[TYPES[dtype]]
        assert ((grad[rows].double() - few[2].double()).abs() <= bound).all()
