"""The policy loss where a scored row has no log-probability, or what it is compared with is NaN: the loss and the row's gradient are
NaN, as the formula's are, and no other row is touched by it.  What is large or masked but has a value keeps it."""
import pytest
import torch

from ops_reference import LOG_SUM, TYPES, U, assert_near
from test_gpu_logits import dev, some_logits

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def inputs(dtype, vocab, rows=7):
    g = torch.Generator().manual_seed(3)
    x = some_logits(rows, vocab, TYPES[dtype], 1, spread=2.0)
    targets = torch.arange(rows, dtype=torch.int32, device=dev()) % vocab
    offsets = torch.tensor([0, 3, rows], device=dev())
    lp = (x.double().log_softmax(1)[torch.arange(rows, device=dev()), targets.long()]).float()
    near = [(lp.cpu() + 0.1 * torch.randn(rows, generator=g)).to(dev()) for _ in range(2)]
    return x, targets, offsets, *near, torch.randn(rows, generator=g).to(dev())


@pytest.mark.parametrize("dtype,vocab", [("f32", 5), ("f16", 1256), ("bf16", 33000), ("bf16", 204809)])
@pytest.mark.parametrize("per", ["token", "string"])
@pytest.mark.parametrize("kl_weight", [None, 0.0, 0.1])
@pytest.mark.parametrize("odd", ["no finite logit", "logit", "old", "advantage"])
def test_nan_is_not_hidden(dtype, vocab, per, kl_weight, odd):
    import paper_2507_11941_amd as bpe

    x, targets, offsets, old, reference, advantages = inputs(dtype, vocab)

    def run():
        return bpe.policy_loss(x, targets, offsets, old, advantages, None if kl_weight is None else reference, 0.2, 0.28, kl_weight or 0.0, per)

    _, lp, grad = run()
    others = torch.arange(7, device=dev()) != 4
    for sign in (1.0, -1.0):                             # of the row's advantage: either side of the clipping
        advantages[4] = sign
        if odd == "no finite logit":
            x[4] = -INF
        elif odd == "logit":
            x[4, vocab - 1] = NAN
        elif odd == "old":
            old[4] = NAN
        else:
            advantages[4] = NAN
        loss, got_lp, got = run()
        assert loss.isnan() and got[4].isnan().all()
        assert got_lp[4].isnan().item() == ("logit" in odd)
        assert torch.equal(got_lp[others], lp[others]) and torch.equal(got[others], grad[others])
    targets[4] = -1                                      # not scored: not read
    loss, _, got = run()
    assert loss.isfinite() and (got[4] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_large_ratios_and_masked_targets(dtype):
    """Two logits, both 0 (p = 1/2), or the target's -inf (p = 0): (advantage, old, value, slope), clipped to [0.75, 1.25]."""
    import paper_2507_11941_amd as bpe

    targets, offsets = torch.zeros(1, dtype=torch.int32, device=dev()), torch.tensor([0, 1], device=dev())
    for masked, advantage, old, value, slope in ((False, 0.0, -1000.0, 0.0, 0.0), (False, 1.0, -1000.0, -1.25, 0.0), (False, -1.0, -1000.0, INF, INF),
                                                 (False, 1.0, 1000.0, 0.0, 0.0), (False, -1.0, 1000.0, 0.75, 0.0), (True, 1.0, -1.0, 0.0, 0.0),
                                                 (True, -1.0, -1.0, 0.75, 0.0), (True, 0.0, -1.0, 0.0, 0.0), (False, INF, 1000.0, NAN, NAN)):
        x = torch.zeros(1, 2, dtype=TYPES[dtype], device=dev())
        if masked:
            x[0, 0] = -INF
        loss, lp, grad = bpe.policy_loss(x, targets, offsets, torch.tensor([old], device=dev()), torch.tensor([advantage], device=dev()),
                                         clip_low=0.25, clip_high=0.25)
        assert_near(loss, torch.tensor(value), 4 * U, f"loss of {masked, advantage, old}")
        assert lp.item() == (-INF if masked else lp.item())
        share = torch.tensor([[1.0, 0.0]]) if masked else torch.tensor([[0.5, -0.5]])
        want = torch.zeros(1, 2) if slope == 0 else slope * share
        assert_near(grad, want, 0.0, f"gradient of {masked, advantage, old}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [7, 1256, 100260, 204809])
def test_rows_of_the_lowest_value(dtype, vocab):
    """Logits that are all the type's lowest value are all as likely: log-probability -log vocab, ratio 1."""
    import paper_2507_11941_amd as bpe

    x = torch.full((3, vocab), torch.finfo(TYPES[dtype]).min, dtype=TYPES[dtype], device=dev())
    targets, offsets = torch.tensor([0, vocab // 2, vocab - 1], dtype=torch.int32, device=dev()), torch.tensor([0, 1, 3], device=dev())
    even = torch.full((3,), 1 / vocab, dtype=torch.float64)
    advantages = torch.tensor([1.0, -2.0, 0.5])
    loss, lp, grad = bpe.policy_loss(x, targets, offsets, even.log().float().to(dev()), advantages.to(dev()), scale=3.0)
    near = LOG_SUM + 2 * U * torch.tensor(vocab).log().item()         # of a log-probability and an old one
    assert_near(lp, even.log(), LOG_SUM, "logprobs")
    assert_near(loss, torch.tensor(0.5 / 3, dtype=torch.float64), 3.5 / 3 * (near + 8 * U), "loss")
    want = (advantages.double() * 3 / 3)[:, None] * even[:, None].expand(3, vocab)
    want[torch.arange(3), targets.cpu().long()] -= advantages.double()
    assert_near(grad, want, want.abs() * (2 * near + 16 * U), "gradient")
