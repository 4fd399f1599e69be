"""include/bpe_head.h: a repetition penalty whose reciprocal is no ordinary 32-bit number is refused, as logits are multiplied by that."""
import pytest
import torch

import paper_2507_11941_amd as bpe
from test_head_abi import HISTORY, LOGITS, MASK, OUT, call

BAD = [2.0 ** -127, 2.0 ** -149, 1e-45, 2.0 ** 126 * (1 + 2.0 ** -23), 2.0 ** 127, 3.4e38]


def test_repetitions():
    more = dict(presence=0.0, frequency=0.0, bias_ids=None, bias_values=None, n_biases=0, bias_begin=None, bias_end=None)
    call("adjust_logits", dict(LOGITS, **HISTORY, **more, **MASK, **OUT), [("repetition", r) for r in BAD])
    call("adjust_logits_grad", dict(LOGITS, from_=LOGITS["logits"], from_stride=40, **HISTORY, **MASK, **OUT), [("repetition", r) for r in BAD])


@pytest.mark.gpu
@pytest.mark.parametrize("repetition", [2.0 ** -126, 2.0 ** -100, 3.0, 2.0 ** 100, 2.0 ** 126])
def test_the_largest_and_smallest(repetition):
    """Logits that the penalty leaves in range, against 64 bits: one rounding of the reciprocal and one of the product."""
    dev = torch.device("cuda:0")
    logits = torch.tensor([[1.5, -1.5, 2.5, -0.75, 1.0]], device=dev)
    logits = torch.where(logits > 0, logits * repetition, logits / repetition)
    ids, at = torch.arange(4, dtype=torch.int32, device=dev), torch.tensor([0, 4], device=dev)
    want = logits.double()
    want = torch.where(want > 0, want / repetition, want * repetition)
    want[0, 4] = logits[0, 4]
    got = bpe.adjust_logits(logits, ids, at[:1], at[1:], (repetition, 0.0, 0.0))
    assert bool(((got.double() - want).abs() <= 2.0 ** -23 * want.abs()).all())
    got = bpe.adjust_logits_grad(torch.ones_like(logits), logits, ids, at[:1], at[1:], (repetition, 0.0, 0.0)).double()
    want = torch.where(logits > 0, 1 / repetition, repetition).double()
    want[0, 4] = 1.0
    assert bool(((got - want).abs() <= 2.0 ** -23 * want.abs()).all())
