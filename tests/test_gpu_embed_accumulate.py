"""The embedding's gradient added to what there is, of more ids than are sorted by counting: micro-batches."""
import numpy as np
import pytest
import torch

from ops_reference import TYPES, U, assert_near
from test_gpu_embed import dev, grad_want, matrix, some_ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,into", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("kind,n,vocab,dim,stride,at", [("skewed", 8193, 511, 33, 40, 1), ("skewed", 20001, 3000, 100, 107, 3), ("one", 30000, 7, 24, 24, 0),
                                                        ("none", 9000, 20, 5, 9, 0), ("even", 65536, 100260, 64, 72, 8), ("padded", 300000, 300000, 3, 3, 0),
                                                        ("skewed", 500, 600000, 5, 5, 2)])
def test_added(dtype, into, kind, n, vocab, dim, stride, at):
    import paper_2507_11941_amd as bpe

    grad, ids = matrix(n, dim, TYPES[dtype], 1, stride, at), some_ids(kind, n, vocab, 2)
    for count in (None, n - n // 3):
        used = n if count is None else count
        out = matrix(vocab, dim, TYPES[into], 3, dim + 3, at)
        memory = out.as_strided((vocab, dim + 3), (dim + 3, 1))
        before = memory.clone()
        counted = None if count is None else torch.tensor([count], device=dev())
        got = bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 0.5, count=counted, out=out, accumulate=True)
        assert got is out
        want, off = grad_want(grad[:used], ids[:used], vocab, 0.5)
        held = before[:, :dim].double().cpu()
        assert_near(out, held + want, off + U * (held.abs() + want.abs()), "gradient")
        absent = torch.ones(vocab, dtype=torch.bool)
        kept = ids[:used]
        absent[kept[(kept >= 0) & (kept < vocab)].long()] = False
        after = memory.cpu()
        assert torch.equal(after[:, dim:], before.cpu()[:, dim:]), "written between the rows"
        assert torch.equal(after[absent], before.cpu()[absent]), "rows that no id names were touched"
        again = matrix(vocab, dim, TYPES[into], 3, dim + 3, at)
        bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 0.5, count=counted, out=again, accumulate=True)
        assert torch.equal(again, out), "not the same bits again"


def test_micro_batches_add_up():
    """Whole numbers, so that sums are exact: four micro-batches against one of all."""
    import paper_2507_11941_amd as bpe

    n, vocab, dim = 40000, 1256, 130
    g = torch.Generator().manual_seed(1)
    grad, ids = torch.randint(-8, 9, (n, dim), generator=g).to(torch.bfloat16).to(dev()), some_ids("skewed", n, vocab, 2).to(dev())
    total = torch.zeros(vocab, dim, device=dev())
    for part in np.array_split(np.arange(n), 4):
        rows = slice(int(part[0]), int(part[-1]) + 1)
        bpe.embed_tokens_grad(grad[rows], ids[rows], vocab, out=total, accumulate=True)
    assert torch.equal(total, bpe.embed_tokens_grad(grad, ids, vocab, dtype=torch.float32))
