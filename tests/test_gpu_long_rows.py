"""Rows of tens of millions of logits: a lane's sum does not lose what it adds late."""
import math

import pytest
import torch

from ops_reference import LOG_SUM, TYPES, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,vocab,n", [("bf16", (1 << 26) + 3, 2), ("f16", (1 << 25) + 5, 1), ("f32", 1 << 25, 1), ("bf16", 1 << 22, 200),
                                           ("f32", 1 << 21, 199)])
def test_many_equal_terms(dtype, vocab, n):
    """A sixteenth of the logits is 0, in stretches that all lanes have a part of, and the others are x: sum m + (vocab - m) e^x.
    Every term has the same rounding error, so that errors do not cancel: of up to 150 additions one after another each rounds by U / 2
    of the sum so far, which is half of the whole on average, 38 U; the exponential is off by 4 U, joins by less than 24 U."""
    import paper_2507_11941_amd as bpe

    dev = torch.device("cuda:0")
    x = torch.tensor(-0.7, dtype=TYPES[dtype])
    logits = torch.full((n, vocab), x.item(), dtype=TYPES[dtype], device=dev)
    zeros = 0
    for begin in range(0, vocab, 1 << 17):
        logits[:, begin:begin + (1 << 13)] = 0.0
        zeros += min(1 << 13, vocab - begin)
    targets = torch.full((n,), 1 << 17, dtype=torch.int32, device=dev)
    want = math.log(zeros + (vocab - zeros) * math.exp(x.double().item()))
    near = LOG_SUM + U * want
    lp, lse = bpe.token_logprobs(logits, targets)
    assert ((lse.double() - want).abs() <= near).all() and ((lp.double() + want).abs() <= near).all()
    if n > 2:
        return
    lp, lse, grad = bpe.token_logprobs_and_grad(logits, targets, torch.ones(n, device=dev))
    assert ((lse.double() - want).abs() <= near).all() and ((lp.double() + want).abs() <= near).all()
    p = math.exp(x.double().item() - want)
    if dtype != "f16":                                   # (p is below its smallest number)
        eps = torch.finfo(TYPES[dtype]).eps
        assert ((grad[:, [1 << 14, (1 << 17) - 1, vocab - 1 - (1 << 13)]].double() + p).abs() <= p * (eps / 2 + 2 * near)).all()
