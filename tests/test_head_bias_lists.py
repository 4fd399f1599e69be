"""A list of biases may be any sequence of its four tensors: each is kept for the stream that a call is given, and others are refused."""
import pytest
import torch

import paper_2507_11941_amd as bpe
from paper_2507_11941_amd import _head


class Stream:
    """What the binding asks of a stream, without a GPU."""
    device = torch.device("cpu")


class Kept(torch.Tensor):
    """A tensor that says for which stream its memory was kept."""
    def record_stream(self, stream):
        self.kept_for = stream


@pytest.mark.parametrize("kind", [tuple, list, iter])
def test_all_of_it_is_kept_for_the_stream(monkeypatch, kind):
    _head._load()
    monkeypatch.setattr(_head, "_on", lambda stream, function, *args: None)        # the call itself
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: None)
    logits = torch.zeros(2, 5)
    parts = [torch.zeros(3, dtype=t).as_subclass(Kept) for t in (torch.int32, torch.float32, torch.int64, torch.int64)]
    stream = Stream()
    bpe.adjust_logits(logits, bias=kind(parts), stream=stream)
    assert all(getattr(p, "kept_for", None) is stream for p in parts)


def test_other_lists_are_refused():
    logits, ids = torch.zeros(2, 5), torch.zeros(3, dtype=torch.int32)
    for bad in ((), (ids,), [ids, ids, ids], (ids, ids, ids, ids, ids)):
        with pytest.raises(ValueError, match="bias"):
            bpe.adjust_logits(logits, bias=bad)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [tuple, list])
def test_memory_of_biases_of_a_call_on_another_stream(kind):
    """What is freed while the other stream still reads it is not given away."""
    dev = torch.device("cuda:0")
    n, vocab, many = 64, 100260, 1 << 21
    logits = torch.randn(n, vocab, device=dev)
    ids = torch.randint(0, vocab, (many,), dtype=torch.int32, device=dev)
    values, begin = torch.randn(many, device=dev), torch.zeros(n, dtype=torch.int64, device=dev)
    end = begin + many
    want = bpe.adjust_logits(logits, bias=(ids, values, begin, end))
    side, kept = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for _ in range(4):
        parts = kind([t.clone() for t in (ids, values, begin, end)])
        side.wait_stream(torch.cuda.current_stream())
        result = bpe.adjust_logits(logits, bias=parts, stream=side)
        del parts
        kept.append((result, [torch.zeros_like(t) for t in (ids, values, begin, end)]))
    torch.cuda.synchronize()
    assert all(torch.equal(result, want) for result, _ in kept)
