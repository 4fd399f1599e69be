"""The example that takes strings through the encoder, a model and the losses: each of them falls, and the encoder's count of ids
is taken from the device."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_losses_fall():
    spec = importlib.util.spec_from_file_location("token_batches", os.path.join(ROOT, "examples", "token_batches.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.main()
    assert set(losses) == {"next token", "preference", "policy"}
    assert losses["next token"][-1] < 0.9 * losses["next token"][0]
    for values in losses.values():
        assert all(v == v for v in values) and values[-1] < values[0]


def test_ids_of_an_encoded_batch_whose_number_stays_on_the_device():
    import torch

    import paper_2507_11941_amd as bpe
    import workloads

    dev = torch.device("cuda:0")
    merges = workloads.load_merges("1k")
    data, ends = workloads.batch(1)
    ids, offsets = bpe.encode_batch(bpe.build_table(merges), torch.from_numpy(data).to(dev), torch.from_numpy(ends).to(dev), 256)
    ids.view(-1)[int(offsets[-1]):] = 7                      # what is behind the ids is anything
    weight = torch.randn(256 + len(merges), 48, device=dev)
    out = torch.zeros(len(ids), 48, device=dev)
    bpe.embed_tokens(weight, ids, 1.0, count=offsets[-1:], out=out)
    used = int(offsets[-1])
    assert 0 < used < len(ids)
    assert torch.equal(out[:used], weight[ids[:used].long()]) and not out[used:].any()
    targets = bpe.next_tokens(ids, offsets)
    assert (targets[used - 1:] == -1).all() and int((targets >= 0).sum()) == used - (len(offsets) - 1)
    grad = bpe.embed_tokens_grad(torch.ones_like(out), ids, len(weight), count=offsets[-1:])
    assert torch.equal(grad[:, 0], torch.bincount(ids[:used].long(), minlength=len(weight)).float())
