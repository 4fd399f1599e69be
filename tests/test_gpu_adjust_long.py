"""Adjusted logits by workgroups of 512 and 1,024 threads, which long histories take: several stretches of columns each, in all types; and more
workgroups than one launch has."""
import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near
from test_gpu_adjust import arguments, check, dev, histories, logits_of, masks, without_bias

pytestmark = pytest.mark.gpu


MEANS = {256: 1999, 512: 2000, 1024: 8000}               # threads by the mean number of ids a row: the least of them, and the most


def long_arguments(form, n, vocab, threads):
    """Histories that have so many ids on average; the first row's is all of them, others are cut off at their end or shorter."""
    more, ids = arguments(form, n, vocab, 5, 4 * MEANS[threads]), n * MEANS[threads]
    spare = torch.arange(ids, dtype=torch.int32, device=dev()) * 7919 % (vocab + 3)
    more["ids"] = torch.cat([more["ids"], spare])[:ids]
    more["begin"][0], more["end"][0] = 0, ids
    return more


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [40003, 32768, 16391])
@pytest.mark.parametrize("threads", [256, 512, 1024])
def test_several_stretches(threads, vocab, dtype):
    n = 4
    for form in ("all", "lists", "rows"):
        print(form, flush=True)
        check(logits_of(n, vocab, TYPES[dtype], 1, vocab % 3, 1), long_arguments(form, n, vocab, threads), 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("threads", [512, 1024])
def test_nothing_else_is_written_with_long_histories(threads, dtype):
    import paper_2507_11941_amd as bpe

    n, vocab, T = 3, 33001, TYPES[dtype]
    more = long_arguments("all", n, vocab, threads)
    logits = logits_of(n, vocab, T, 1)
    want = bpe.adjust_logits(logits, **more)
    room = torch.full((n + 2, vocab + 7), 5.0, dtype=T, device=dev())
    out = room[1:-1, 3:vocab + 3]
    bpe.adjust_logits(logits, **more, out=out)
    assert torch.equal(out, want)
    out.fill_(5.0)
    assert bool((room == 5.0).all())
    grad = logits_of(n, vocab, T, 2)
    want = bpe.adjust_logits_grad(grad, logits, **without_bias(more))
    bpe.adjust_logits_grad(grad, logits, **without_bias(more), out=out)
    assert torch.equal(out, want)
    out.fill_(5.0)
    assert bool((room == 5.0).all())


@pytest.mark.parametrize("n,vocab", [(2 ** 21 + 9, 2), (2 ** 20 + 9, 4099)])
def test_more_workgroups_than_one_launch_has(n, vocab):
    """One stretch of columns a row and two: about the row with which the second launch begins, and all rows against calls of one launch."""
    import paper_2507_11941_amd as bpe

    ids = histories(3, vocab, 40, 1)[0]
    row = torch.arange(n, device=dev())
    begin = row % 7
    more = dict(ids=ids, begin=begin, end=begin + row % 5, penalties=(1.25, 0.5, 0.25))
    mask, _ = masks(4, n, vocab, 2)
    more.update(mask=mask, state=((row % 6) - 1).to(torch.int32))
    g = torch.Generator(device=dev()).manual_seed(1)
    logits, grad = (torch.randn(n, vocab, generator=g, device=dev(), dtype=torch.bfloat16) for _ in range(2))
    rows = lambda some: {**more, **{k: more[k][some] for k in ("begin", "end", "state")}}
    border = 2 ** 21 // ((vocab + 4095) // 4096)
    for call, source, wanted in ((lambda x, **k: bpe.adjust_logits(x, **k), logits, lambda some: ref.adjust(logits[some], **rows(some))),
                                 (lambda x, some=slice(None), **k: bpe.adjust_logits_grad(x, logits[some], **k), grad,
                                  lambda some: ref.adjust_grad(grad[some], logits[some], **rows(some)))):
        got = call(source, **more)
        for some in (slice(0, 13), slice(border - 13, n)):
            want, off = wanted(some)
            assert_near(got[some], want, off, "adjusted")
        for some in (slice(0, border // 2), slice(border // 2, n)):
            again = call(source[some], **rows(some)) if source is logits else call(source[some], some=some, **rows(some))
            assert torch.equal(again, got[some])
        in_place = source.clone()
        call(in_place, **more, out=in_place)
        assert torch.equal(in_place, got)
