"""The operators at a model's output end on another stream than the current one, and captured in a graph that is replayed on new inputs
with eager work in between: the same bits as of the eager calls."""
import pytest
import torch

import test_gpu_adjust as adjust
import test_gpu_norm as norm
import test_gpu_project as project
from test_gpu_norm import dev

pytestmark = pytest.mark.gpu


def calls(n=70, dim=136, vocab=900):
    """(inputs that may change, calls on them)"""
    import paper_2507_11941_amd as bpe

    x, more, g, gs = (norm.matrix(n, dim, torch.bfloat16, seed) for seed in (1, 2, 3, 4))
    weight = norm.matrix(1, dim, torch.float32, 5).reshape(-1)
    _, total, rstd = bpe.add_norm(x, weight, more)
    head, head_scales = project.bytes_of(vocab, dim, 6), project.scales_of(vocab, 7)
    logits, grad = adjust.logits_of(n, vocab, torch.bfloat16, 8), adjust.logits_of(n, vocab, torch.bfloat16, 9)
    form = adjust.arguments("all", n, vocab, 10)
    plain = adjust.without_bias(form)

    def chain(**k):
        q, scales, _ = bpe.add_norm_8bit(x, weight, more, **k)
        return q, scales, bpe.project_8bit(q, scales, head, head_scales, **k)

    return (x, more, g, gs, logits, grad), [
        lambda **k: bpe.add_norm(x, weight, more, **k), lambda **k: bpe.add_norm_8bit(x, weight, more, **k),
        lambda **k: bpe.quantize_rows(x, **k), lambda **k: bpe.add_norm_grad(g, total, weight, rstd, gs, **k), chain,
        lambda **k: (bpe.adjust_logits(logits, **form, **k),), lambda **k: (bpe.adjust_logits_grad(grad, logits, **plain, **k),)]


def test_another_stream():
    for call in calls()[1]:
        want = call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_memory_of_a_call_on_another_stream():
    """What is freed while the other stream still works on it is not given away."""
    import paper_2507_11941_amd as bpe

    side = torch.cuda.Stream()
    weight = torch.ones(4096, device=dev())
    x = torch.randn(4096, 4096, device=dev())
    want = bpe.add_norm_8bit(x, weight)[0]
    kept = []
    for _ in range(6):
        y = x.clone()
        side.wait_stream(torch.cuda.current_stream())
        q, scales, _ = bpe.add_norm_8bit(y, weight, stream=side)
        del y
        kept.append((q, torch.zeros(4096, 4096, device=dev())))
    torch.cuda.synchronize()
    assert all(torch.equal(q, want) for q, _ in kept)


@pytest.mark.parametrize("which", range(7))
def test_replays(which):
    inputs, made = calls()
    call = made[which]
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call()
    for seed in (1, 2, 3):
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(seed)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        want = call()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_training_step_in_a_graph():
    """Forward and backward passes of the recorded functions, captured together."""
    import paper_2507_11941_amd as bpe

    n, dim = 40, 72
    x = norm.matrix(n, dim, torch.float32, 1)
    weight = torch.ones(dim, device=dev(), requires_grad=True)
    ids = torch.randint(0, dim, (200,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).to(dev())
    begin = torch.arange(n, device=dev()) * 5

    def step():
        y, _, _ = bpe.add_norm(x, weight)
        z = bpe.adjust_logits(y, ids, begin, begin + 4, (1.5, 0.25, 0.0))
        return torch.autograd.grad(z, weight, torch.ones_like(z))[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (2, 3):
        x.copy_(norm.matrix(n, dim, torch.float32, seed))
        graph.replay()
        torch.cuda.synchronize()
        got = captured.clone()
        assert torch.equal(got, step())
