"""The gradient of adjusted logits depends on the logits of tokens in histories alone, whatever lies beside them and behind the rows."""
import math

import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near
from test_gpu_adjust import arguments, dev, logits_of, without_bias

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logits_of_other_tokens(dtype, fill):
    import paper_2507_11941_amd as bpe

    for n, vocab, spread, at in ((5, 1256, 0, 0), (4, 999, 1, 1), (3, 10001, 5, 3)):
        more = without_bias(arguments("all", n, vocab, vocab))
        logits, grad = logits_of(n, vocab, TYPES[dtype], 1, spread, at), logits_of(n, vocab, TYPES[dtype], 2)
        want, off = ref.adjust_grad(grad, logits, **more)
        room = torch.full((n * (vocab + spread) + at,), fill, dtype=TYPES[dtype], device=dev())
        only = room[at:].as_strided(logits.shape, logits.stride())
        named = ref.counts(vocab, more["ids"], more["begin"], more["end"]).to(dev()) > 0
        only[named] = logits[named]
        assert_near(bpe.adjust_logits_grad(grad, only, **more), want, off, "gradient")
        assert bpe.adjust_logits_grad(grad, only, **more, out=grad) is grad
        assert_near(grad, want, off, "in place")
