"""Embedding lookup and its gradient against 64 bits: types, odd sizes, strides, ids outside the vocabulary, ids that all are
the same token, counts on the device, accumulation."""
import numpy as np
import pytest
import torch

from ops_reference import TYPES, U, assert_near

pytestmark = pytest.mark.gpu


def dev():
    assert torch.cuda.is_available(), "these tests need the GPU"
    return torch.device("cuda:0")


def matrix(rows, columns, dtype, seed, stride=None, at=0):
    """Random values in a matrix that begins `at` elements into its memory, with `stride` elements between rows."""
    stride = stride or columns
    g = torch.Generator().manual_seed(seed)
    memory = torch.randn(at + rows * stride + 8, generator=g).to(dtype).to(dev())
    return memory[at:].as_strided((rows, columns), (stride, 1), memory.storage_offset() + at)


def some_ids(kind, n, vocab, seed):
    rng = np.random.default_rng(seed)
    if kind == "one":
        ids = np.full(n, vocab - 1)
    elif kind == "none":
        ids = np.where(rng.random(n) < 0.5, -1, vocab)
    elif kind == "skewed":
        ids = np.minimum(rng.zipf(1.2, n) - 1, vocab - 1)
    else:
        ids = rng.integers(0, vocab, n)
    if kind in ("skewed", "padded"):
        ids[rng.random(n) < 0.2] = rng.choice([-1, -2**31, vocab, 2**31 - 1])
    return torch.from_numpy(ids.astype(np.int32))


def embed_want(weight, ids, scale):
    kept = (ids >= 0) & (ids < len(weight))
    return torch.where(kept[:, None], weight.double().cpu()[torch.where(kept, ids, 0).long()] * scale, 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,dim,stride,at", [(1, 1, 1, None, 0), (1, 300, 4096, None, 0), (7, 1256, 387, None, 0), (64, 257, 8, 13, 1),
                                                   (1000, 500, 129, 131, 3), (33, 100, 2048, 2056, 8), (5, 64, 20001, None, 5),
                                                   (70000, 50, 24, None, 0)])
def test_lookup(dtype, n, vocab, dim, stride, at):
    import paper_2507_11941_amd as bpe

    weight, ids = matrix(vocab, dim, TYPES[dtype], 1, stride, at), some_ids("padded", n, vocab, 2)
    scale = np.float32(5.6568542)
    out = matrix(n, dim, TYPES[dtype], 3, dim + 5, 1)
    around = out.as_strided((n, dim + 5), (dim + 5, 1)).clone()
    got = bpe.embed_tokens(weight, ids.to(dev()), float(scale), out=out)
    assert got is out
    want = embed_want(weight, ids, float(scale))
    assert_near(got, want, U * want.abs(), "out")
    assert torch.equal(out.as_strided((n, dim + 5), (dim + 5, 1))[:, dim:], around[:, dim:]), "written between the rows"
    own = bpe.embed_tokens(weight, ids.to(dev()), float(scale))
    assert torch.equal(own, got)


def test_lookup_leaves_rows_from_the_count_on_alone():
    import paper_2507_11941_amd as bpe

    weight, ids = matrix(100, 33, torch.float32, 1), some_ids("even", 50, 100, 2).to(dev())
    for count in (0, 1, 49, 50, 51, -3):
        out = torch.full((50, 33), 7.0, device=dev())
        bpe.embed_tokens(weight, ids, count=torch.tensor([5, count], device=dev())[1:], out=out)
        used = min(50, max(0, count))
        assert torch.equal(out[:used], weight[ids[:used].long()]) and (out[used:] == 7).all()


def test_lookup_of_nothing_and_of_odd_values():
    import paper_2507_11941_amd as bpe

    weight = matrix(10, 5, torch.bfloat16, 1)
    assert bpe.embed_tokens(weight, torch.empty(0, dtype=torch.int32, device=dev())).shape == (0, 5)
    weight[3] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3.3895e38, -0.0])
    got = bpe.embed_tokens(weight, torch.tensor([3, -1], dtype=torch.int32, device=dev()), 1.0)
    assert torch.equal(got[0].view(torch.int16)[1:], weight[3].view(torch.int16)[1:]) and got[0, 0].isnan()
    assert (got[1] == 0).all()


def grad_want(grad, ids, vocab, scale):
    """(gradient, bound on the error of its sums) in 64 bits"""
    kept = ((ids >= 0) & (ids < vocab)).nonzero().squeeze(1)
    rows, at = grad.double().cpu()[kept], ids[kept].long()
    want = torch.zeros(vocab, grad.shape[1], dtype=torch.float64).index_add_(0, at, rows) * scale
    size = torch.zeros_like(want).index_add_(0, at, rows.abs()) * abs(scale)
    times = torch.zeros(vocab, dtype=torch.float64).index_add_(0, at, torch.ones(len(at), dtype=torch.float64))
    # additions one after another err like a random walk: sqrt(k) roundings of a sum no larger than the magnitudes'
    return want, size * U * (times.sqrt() * 2 + 4)[:, None]


@pytest.mark.parametrize("dtype,into", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("kind,n,vocab,dim", [("even", 1, 1, 1), ("even", 1, 40, 9), ("skewed", 63, 5, 65), ("one", 64, 3, 8), ("one", 5000, 7, 130),
                                              ("skewed", 2003, 1256, 387), ("none", 300, 20, 12), ("skewed", 9001, 33000, 40),
                                              ("even", 20000, 300, 136), ("skewed", 40000, 100260, 17), ("padded", 4097, 513, 512),
                                              ("even", 500, 12, 5000), ("skewed", 8192, 524287, 3), ("even", 500, 600000, 3), ("skewed", 8193, 511, 33),
                                              ("skewed", 300000, 3000, 5), ("one", 270000, 2, 9)])
def test_gradient(dtype, into, kind, n, vocab, dim):
    import paper_2507_11941_amd as bpe

    grad, ids = matrix(n, dim, TYPES[dtype], 1), some_ids(kind, n, vocab, 2)
    got = bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 0.3, dtype=TYPES[into])
    want, off = grad_want(grad, ids, vocab, float(np.float32(0.3)))
    assert_near(got, want, off, "gradient")
    assert torch.equal(got, bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 0.3, dtype=TYPES[into])), "not the same bits again"


@pytest.mark.parametrize("dtype,into", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("kind,n,dim,stride,at", [("skewed", 3001, 100, 107, 1), ("one", 700, 64, 64, 3), ("none", 100, 5, 9, 0),
                                                  ("even", 90, 512, 520, 8)])
def test_gradient_is_added_where_it_is_accumulated(dtype, into, kind, n, dim, stride, at):
    import paper_2507_11941_amd as bpe

    vocab = 400
    grad, ids = matrix(n, dim, TYPES[dtype], 1, stride, at), some_ids(kind, n, vocab, 2)
    out = matrix(vocab, dim, TYPES[into], 3, dim + 3, at)
    before = out.as_strided((vocab, dim + 3), (dim + 3, 1)).clone()
    bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 2.0, out=out, accumulate=True)
    want, off = grad_want(grad, ids, vocab, 2.0)
    held = before[:, :dim].double().cpu()
    assert_near(out, held + want, off + U * (held.abs() + want.abs()), "gradient")
    after = out.as_strided((vocab, dim + 3), (dim + 3, 1))
    assert torch.equal(after[:, dim:], before[:, dim:]), "written between the rows"
    absent = torch.ones(vocab, dtype=torch.bool)
    absent[ids[(ids >= 0) & (ids < vocab)].long()] = False
    assert torch.equal(after.cpu()[absent], before.cpu()[absent]), "rows that no id names were touched"
    # the next micro-batch: twice the same is the same again
    bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, -2.0, out=out, accumulate=True)
    assert_near(out, held, 2 * off + 3 * U * (held.abs() + want.abs()) + 2 * torch.finfo(out.dtype).eps * (held + want).abs(), "and back")


def test_gradient_does_not_read_what_is_padding_or_beyond_the_count():
    import paper_2507_11941_amd as bpe

    n, vocab, dim = 3000, 70, 41
    grad, ids = matrix(n, dim, torch.float32, 1), some_ids("padded", n, vocab, 2)
    for count in (0, 1, 64, 2500, 3000, 4000, -1):
        used = min(n, max(0, count))
        g = grad.clone()
        g[used:] = float("nan")
        g[((ids < 0) | (ids >= vocab)).to(dev())] = float("inf")
        got = bpe.embed_tokens_grad(g, ids.to(dev()), vocab, 1.0, count=torch.tensor([count], device=dev()))
        want, off = grad_want(grad[:used], ids[:used], vocab, 1.0)
        assert_near(got, want, off, f"count {count}")


def test_gradient_against_differences():
    """d/dW of sum(G * embed(W)) by central differences of the lookup itself; the lookup is linear, so the step may be large."""
    import paper_2507_11941_amd as bpe

    n, vocab, dim = 40, 6, 5
    weight, grad, ids = matrix(vocab, dim, torch.float32, 1), matrix(n, dim, torch.float32, 2), some_ids("padded", n, vocab, 3)
    got = bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 0.7).cpu()
    for v in range(vocab):
        for c in range(dim):
            values = []
            for step in (4.0, -4.0):
                w = weight.clone()
                w[v, c] += step
                values.append((grad.double() * bpe.embed_tokens(w, ids.to(dev()), 0.7).double()).sum().item())
            # a product of up to 8 x 0.7 is rounded to 32 bits, 40 of them, over a step of 8
            assert abs((values[0] - values[1]) / 8 - got[v, c].item()) <= 40 * 8 * U * 4 / 8 + 40 * U * 4


def test_refusals():
    import paper_2507_11941_amd as bpe

    weight, ids = matrix(10, 6, torch.float32, 1), torch.zeros(4, dtype=torch.int32, device=dev())
    grad = matrix(4, 6, torch.float32, 2)
    for bad in (lambda: bpe.embed_tokens(weight.cpu(), ids), lambda: bpe.embed_tokens(weight, ids.long()), lambda: bpe.embed_tokens(weight.double(), ids),
                lambda: bpe.embed_tokens(weight, ids.cpu()), lambda: bpe.embed_tokens(weight.t(), ids), lambda: bpe.embed_tokens(weight[0], ids),
                lambda: bpe.embed_tokens(weight, torch.zeros(8, dtype=torch.int32, device=dev())[::2]),
                lambda: bpe.embed_tokens(weight, ids, out=torch.empty(4, 5, device=dev())),
                lambda: bpe.embed_tokens(weight, ids, out=torch.empty(4, 6, device=dev(), dtype=torch.float16)),
                lambda: bpe.embed_tokens(weight, ids, count=torch.zeros(1, device=dev())),
                lambda: bpe.embed_tokens(torch.zeros(1, 6, device=dev()).expand(10, 6), ids),
                lambda: bpe.embed_tokens_grad(grad, ids[:3], 10), lambda: bpe.embed_tokens_grad(grad, ids, 10, accumulate=True),
                lambda: bpe.embed_tokens_grad(grad, ids, 10, dtype=torch.float16), lambda: bpe.embed_tokens_grad(grad, ids, 0),
                lambda: bpe.embed_tokens_grad(grad, ids, 10, out=torch.empty(11, 6, device=dev())),
                lambda: bpe.embed_tokens_grad(grad, ids, 10, workspace=torch.empty(8, dtype=torch.uint8, device=dev()))):
        with pytest.raises(ValueError):
            bad()
    torch.cuda.synchronize()


def test_more_rows_than_one_launch_takes():
    import paper_2507_11941_amd as bpe

    n, vocab, dim = (1 << 21) + 1003, 700, 3
    weight, ids = matrix(vocab, dim, torch.float32, 1), some_ids("skewed", n, vocab, 2)
    want = embed_want(weight, ids, 2.0)
    assert torch.equal(bpe.embed_tokens(weight, ids.to(dev()), 2.0).cpu().double(), want)
    grad = matrix(n, dim, torch.float32, 3)
    got = bpe.embed_tokens_grad(grad, ids.to(dev()), vocab, 1.0)
    assert_near(got, *grad_want(grad, ids, vocab, 1.0), "gradient")


def test_outputs_belong_to_the_stream_that_writes_them():
    """A block that the caller's stream has freed but is still writing to must not become the output of a call on another stream."""
    import paper_2507_11941_amd as bpe

    n, dim = 4096, 1024
    weight, ids = torch.randn(1000, dim, device=dev()), torch.arange(n, dtype=torch.int32, device=dev()) % 1000
    want = weight[ids.long()]
    grad_want = bpe.embed_tokens_grad(want, ids, 1000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    late = [torch.empty(n, dim, device=dev()), torch.empty(1000, dim, device=dev())]
    torch.cuda._sleep(20_000_000)
    for t in late:
        t.fill_(7.0)
    del late, t
    got = bpe.embed_tokens(weight, ids, stream=side)
    grad = bpe.embed_tokens_grad(got, ids, 1000, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(grad, grad_want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,stride", [(1024, 1024), (1000, 1024), (1000, 1000)])
def test_more_than_the_caches_hold(dtype, dim, stride):
    import paper_2507_11941_amd as bpe

    vocab, n = 3000, 256_000_000 // (1000 * torch.empty(0, dtype=TYPES[dtype]).element_size()) + 1000
    g = torch.Generator(device=dev()).manual_seed(1)
    weight = torch.randn(vocab, dim, generator=g, device=dev()).to(TYPES[dtype])
    ids = torch.randint(-1, vocab, (n,), generator=g, device=dev(), dtype=torch.int32)
    out = torch.empty(n, stride, dtype=TYPES[dtype], device=dev())[:, :dim]
    bpe.embed_tokens(weight, ids, out=out)
    assert torch.equal(out, torch.where(ids[:, None] < 0, 0, weight[ids.long().clamp(min=0)]))
    # Whole numbers of up to 8: sums are exact in any order.
    out.copy_(torch.randint(-8, 9, (n, dim), generator=g, device=dev()))
    got = bpe.embed_tokens_grad(out, ids, vocab, dtype=torch.float32)
    want = torch.zeros(vocab + 1, dim, device=dev()).index_add_(0, torch.where(ids < 0, vocab, ids).long(), out.float())
    assert torch.equal(got, want[:vocab])
