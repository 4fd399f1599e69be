"""Log-probabilities and their gradient against 64 bits: types, rows from one logit to more than any on-chip store holds, strides
and alignments, masked entries, rows that are not scored whatever they hold, offsets beyond 32 bits, streams, graphs."""
import numpy as np
import pytest
import torch

from ops_reference import LOG_SUM, TYPES, U, assert_near, logits_grad, logprobs

pytestmark = pytest.mark.gpu


def dev():
    assert torch.cuda.is_available(), "these tests need the GPU"
    return torch.device("cuda:0")


def some_logits(n, vocab, dtype, seed, stride=None, at=0, spread=3.0):
    stride = stride or vocab
    g = torch.Generator(device=dev()).manual_seed(seed)
    memory = (torch.randn(at + n * stride + 8, generator=g, device=dev()) * spread).to(dtype)
    return memory.as_strided((n, vocab), (stride, 1), at)


def some_targets(n, vocab, seed, unscored=0.25):
    rng = np.random.default_rng(seed)
    t = rng.integers(0, vocab, n)
    if n > 1:
        t = np.where(rng.random(n) < unscored, rng.choice([-1, -2**31, vocab, 2**31 - 1], n), t)
    return torch.from_numpy(t.astype(np.int32)).to(dev())


def some_upstream(n, seed):
    u = torch.randn(n, generator=torch.Generator().manual_seed(seed))
    u[torch.arange(n) % 5 == 3] = 0.0
    return u.to(dev())


def check_all(x, targets, upstream, what=""):
    """The three entry points on one input."""
    import paper_2507_11941_amd as bpe

    want_lp, want_lse = logprobs(x, targets)
    want_grad, off = logits_grad(x, targets, upstream)
    lp, lse = bpe.token_logprobs(x, targets)
    assert_near(lp, want_lp, LOG_SUM, f"{what} logprobs")
    assert_near(lse, want_lse, LOG_SUM, f"{what} lse")
    grad = bpe.token_logprobs_grad(x, targets, lse, upstream)
    assert_near(grad, *logits_grad(x, targets, upstream, lse), f"{what} gradient")
    lp1, lse1, grad1 = bpe.token_logprobs_and_grad(x, targets, upstream)
    assert_near(lp1, want_lp, LOG_SUM, f"{what} logprobs in one pass")
    assert_near(lse1, want_lse, LOG_SUM, f"{what} lse in one pass")
    assert_near(grad1, want_grad, off, f"{what} gradient in one pass")
    return lp, lse, grad, grad1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab", [(1, 1), (3, 2), (5, 7), (2, 64), (9, 255), (4, 1256), (300, 1257), (6, 4097), (3, 8192), (5, 10001), (3, 16390),
                                     (70, 32256), (3, 40003), (4, 65537), (9, 100260), (2, 102401), (3, 150001), (2, 204805), (2, 300007)])
def test_sizes(dtype, n, vocab):
    check_all(some_logits(n, vocab, TYPES[dtype], n), some_targets(n, vocab, vocab), some_upstream(n, 3))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,stride,at", [(1256, 1256, 1), (1256, 1257, 0), (1001, 1003, 3), (33, 40, 8), (32256, 32261, 7), (100260, 100267, 1),
                                             (16, 17, 5), (7, 8, 2)])
def test_strides_and_alignments(dtype, vocab, stride, at):
    import paper_2507_11941_amd as bpe

    n = 12
    x, targets, upstream = some_logits(n, vocab, TYPES[dtype], 4, stride, at), some_targets(n, vocab, 5), some_upstream(n, 6)
    _, lse, grad, grad1 = check_all(x, targets, upstream)
    # gradients with strides and alignments of their own, and in the place of the logits: the same bits, nothing between the rows
    for out_stride, out_at in ((vocab + 3, 1), (vocab + 8, 0), (vocab, 5)):
        memory = torch.full((out_at + n * out_stride + 8,), 9.0, dtype=x.dtype, device=dev())
        out = memory.as_strided((n, vocab), (out_stride, 1), out_at)
        for call, want in ((lambda: bpe.token_logprobs_grad(x, targets, lse, upstream, out=out), grad),
                           (lambda: bpe.token_logprobs_and_grad(x, targets, upstream, out=out)[2], grad1)):
            assert call() is out and torch.equal(out, want)
            rest = memory.clone()
            rest.as_strided((n, vocab), (out_stride, 1), out_at).fill_(9.0)
            assert (rest == 9).all()
    for k in range(2):
        y = some_logits(n, vocab, TYPES[dtype], 4, stride, at)
        got = bpe.token_logprobs_grad(y, targets, lse, upstream, out=y) if k else bpe.token_logprobs_and_grad(y, targets, upstream, out=y)[2]
        assert torch.equal(got, grad if k else grad1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [5, 1256, 100260])
def test_masked_and_odd_logits(dtype, vocab):
    import paper_2507_11941_amd as bpe

    low, inf, nan = torch.finfo(TYPES[dtype]).min, float("inf"), float("nan")
    x = some_logits(14, vocab, TYPES[dtype], 1)
    targets = torch.full((14,), 2, dtype=torch.int32, device=dev())
    x[0, 3:] = -inf                                  # most are masked
    x[1, :2], x[1, 3:] = -inf, -inf                  # all but the target
    x[2, 2] = -inf                                   # the target itself
    x[3, 3:] = low
    x[4] = low                                       # all the lowest value: evenly likely
    x[5, :2], x[5, 3:] = low, -inf
    x[6], x[6, 2] = low, -low                        # the highest among the lowest
    x[7] = 0.0
    x[8] *= 0.01
    x[9, 0] = 30000.0                                # one far above the rest
    x[10, 0], x[10, 4] = -inf, nan                   # a row that is not scored may hold anything
    targets[10] = -1
    x[11] = nan
    targets[11] = vocab
    x[12] = -inf
    targets[12] = -7
    x[13, 4] = nan                                   # ... and one that is scored becomes NaN
    want_lp, want_lse = logprobs(x, targets)
    upstream = some_upstream(14, 2)
    upstream[13], upstream[2] = 1.0, 0.5
    want_grad, off = logits_grad(x, targets, upstream)
    off[torch.isnan(off)] = 0
    lp, lse = bpe.token_logprobs(x, targets)
    near = LOG_SUM + 3 * U * 30000                   # (differences of up to 30,000 are rounded)
    assert_near(lp, want_lp, near, "logprobs")
    assert_near(lse, want_lse, near, "lse")
    lp1, lse1, grad1 = bpe.token_logprobs_and_grad(x, targets, upstream)
    assert_near(lp1, want_lp, near, "logprobs in one pass")
    assert_near(lse1, want_lse, near, "lse in one pass")
    assert_near(grad1, want_grad, off, "gradient in one pass")
    want_grad, off = logits_grad(x, targets, upstream, lse)
    off[torch.isnan(off)] = 0
    assert_near(bpe.token_logprobs_grad(x, targets, lse, upstream), want_grad, off, "gradient")
    for g in (grad1, bpe.token_logprobs_grad(x, targets, lse, upstream)):
        assert (g[10:13] == 0).all() and g[13].isnan().all()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_a_finite_logit_are_nan(dtype):
    import paper_2507_11941_amd as bpe

    for vocab in (3, 1256, 100260):
        x = torch.full((2, vocab), -float("inf"), dtype=TYPES[dtype], device=dev())
        x[1, 0] = 1.0
        targets, upstream = torch.zeros(2, dtype=torch.int32, device=dev()), torch.ones(2, device=dev())
        lp, lse = bpe.token_logprobs(x, targets)
        lp1, _, grad = bpe.token_logprobs_and_grad(x, targets, upstream)
        for got in (lp, lp1):
            assert got[0].isnan() and got[1] == 0
        assert grad[0].isnan().all() and (grad[1] == 0).all()
        assert bpe.token_logprobs_grad(x, targets, lse, upstream)[0].isnan().all()


def test_gradient_against_differences():
    """Central differences of the log-probabilities themselves; a step of 2^-4 leaves h^2 / 6 of a third derivative that is at
    most 1/4, and 2 x LOG_SUM and two roundings of a value below 16 over 2 h."""
    import paper_2507_11941_amd as bpe

    x, targets = some_logits(3, 9, torch.float32, 8, spread=1.0), torch.tensor([4, 0, 8], dtype=torch.int32, device=dev())
    upstream = torch.tensor([1.0, -0.5, 2.0], device=dev())
    grad = bpe.token_logprobs_and_grad(x, targets, upstream)[2].cpu()
    h = 2.0 ** -4
    for j in range(9):
        up, down = x.clone(), x.clone()
        up[:, j] += h
        down[:, j] -= h
        change = (bpe.token_logprobs(up, targets)[0].double() - bpe.token_logprobs(down, targets)[0].double()) / (2 * h)
        far = h * h / 24 + (2 * LOG_SUM + 64 * U) / (2 * h)
        assert ((change * upstream).cpu() - grad[:, j]).abs().max() <= 2 * far


def test_nothing_and_equal_bits():
    import paper_2507_11941_amd as bpe

    none = torch.empty(0, dtype=torch.int32, device=dev())
    x = torch.empty(0, 100, device=dev())
    assert bpe.token_logprobs(x, none)[0].shape == (0,)
    assert bpe.token_logprobs_and_grad(x, none, x[:, 0].contiguous())[2].shape == (0, 100)
    assert bpe.token_logprobs_grad(x, none, x[:, 0].contiguous(), x[:, 0].contiguous()).shape == (0, 100)
    for n, vocab in ((2, 100260), (50, 100260), (600, 1256)):
        x, targets, upstream = some_logits(n, vocab, torch.bfloat16, 1), some_targets(n, vocab, 2), some_upstream(n, 3)
        first = [t.clone() for t in (*bpe.token_logprobs(x, targets), *bpe.token_logprobs_and_grad(x, targets, upstream))]
        again = (*bpe.token_logprobs(x, targets), *bpe.token_logprobs_and_grad(x, targets, upstream))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_elements_beyond_32_bits():
    """More than 2^32 logits: rows far beyond are read and written where they are."""
    import paper_2507_11941_amd as bpe

    n, vocab = 43000, 100260
    assert n * vocab > 1 << 32
    x = torch.zeros(n, vocab, dtype=torch.bfloat16, device=dev())
    targets = torch.full((n,), -1, dtype=torch.int32, device=dev())
    rows = [0, 21419, 21420, 42837, 42838, 42999]                   # about 2^31 and 2^32 elements on
    x[rows] = some_logits(len(rows), vocab, torch.bfloat16, 5)
    targets[rows] = some_targets(len(rows), vocab, 6, 0.0)
    upstream = torch.ones(n, device=dev())
    want_lp, _ = logprobs(x[rows], targets[rows])
    lp, lse = bpe.token_logprobs(x, targets)
    assert_near(lp[rows], want_lp, LOG_SUM)
    grad = torch.full_like(x, 3.0)
    bpe.token_logprobs_grad(x, targets, lse, upstream, out=grad)
    assert_near(grad[rows], *logits_grad(x[rows], targets[rows], upstream[rows], lse[rows]))
    grad[rows] = 0
    assert not grad.any()
    want, off = logits_grad(x[rows], targets[rows], upstream[rows])
    bpe.token_logprobs_and_grad(x, targets, upstream, out=x)
    assert_near(x[rows], want, off)
    x[rows] = 0
    assert not x.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,shift", [(33001, 0), (32256, 0), (32256, 1), (1000, 0)])
def test_more_than_the_caches_hold(dtype, vocab, shift):
    """A row's results do not depend on how many others there are, nor on whether they pass the caches by."""
    import paper_2507_11941_amd as bpe

    n = 256_000_000 // (vocab * torch.empty(0, dtype=TYPES[dtype]).element_size()) + 100
    x, targets, upstream = some_logits(n, vocab, TYPES[dtype], 1), some_targets(n, vocab, 2), some_upstream(n, 3)
    out = torch.empty(n * vocab + shift, dtype=TYPES[dtype], device=dev())[shift:].view(n, vocab)
    lp, lse = bpe.token_logprobs(x, targets)
    grad = bpe.token_logprobs_grad(x, targets, lse, upstream, out=out).clone()
    lp1, lse1, grad1 = bpe.token_logprobs_and_grad(x, targets, upstream, out=out)
    for rows in (slice(0, 70), slice(n // 2, n // 2 + 70), slice(n - 70, n)):
        few = bpe.token_logprobs(x[rows], targets[rows])
        assert torch.equal(few[0], lp[rows]) and torch.equal(few[1], lse[rows])
        assert torch.equal(bpe.token_logprobs_grad(x[rows], targets[rows], few[1], upstream[rows]), grad[rows])
        few = bpe.token_logprobs_and_grad(x[rows], targets[rows], upstream[rows])
        assert torch.equal(few[0], lp1[rows]) and torch.equal(few[1], lse1[rows]) and torch.equal(few[2], grad1[rows])
        check_all(x[rows], targets[rows], upstream[rows])
    # In place, and a policy loss at the old policy, which is a step with -advantage / (number of scored tokens).
    advantages = torch.where(upstream == 0, 1.0, upstream)
    many = ((targets >= 0) & (targets < vocab)).sum()
    offsets = torch.tensor([0, n], device=dev())
    want = bpe.token_logprobs_and_grad(x, targets, -advantages / many)[2].float()
    loss, lp2, got = bpe.policy_loss(x, targets, offsets, lp1, advantages, out=x)
    assert torch.equal(lp2, lp1) and got.data_ptr() == x.data_ptr()
    # (both divide, in another order, and round the gradient once)
    ulp = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype]
    off = want.abs() * (2 * ulp + 4 * 2.0 ** -23) + (2.0 ** -24 if dtype == "f16" else 0.0)
    assert ((got.float() - want).abs() <= off).all()


def test_another_stream_and_a_graph():
    import paper_2507_11941_amd as bpe

    n, vocab = 40, 32256
    x, targets, upstream = some_logits(n, vocab, torch.float16, 1), some_targets(n, vocab, 2), some_upstream(n, 3)
    want = bpe.token_logprobs_and_grad(x, targets, upstream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = bpe.token_logprobs_and_grad(x, targets, upstream, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp, lse = bpe.token_logprobs(x, targets)
        grad = bpe.token_logprobs_grad(x, targets, lse, upstream)
    for seed in (5, 6, 7):
        x.copy_(some_logits(n, vocab, torch.float16, seed))
        grad.fill_(1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = bpe.token_logprobs(x, targets)
        assert torch.equal(eager[0], lp) and torch.equal(eager[1], lse)
        assert torch.equal(bpe.token_logprobs_grad(x, targets, lse, upstream), grad)


def test_refusals():
    import paper_2507_11941_amd as bpe

    x, targets, u = some_logits(4, 10, torch.float32, 1), some_targets(4, 10, 2), some_upstream(4, 3)
    for bad in (lambda: bpe.token_logprobs(x.cpu(), targets), lambda: bpe.token_logprobs(x, targets.long()), lambda: bpe.token_logprobs(x, targets[:3]),
                lambda: bpe.token_logprobs(x.double(), targets), lambda: bpe.token_logprobs(x.t(), some_targets(10, 4, 1)),
                lambda: bpe.token_logprobs(x[:, :0], targets), lambda: bpe.token_logprobs(x[0], targets),
                lambda: bpe.token_logprobs(some_logits(4, 100260, torch.float32, 1), targets, workspace=torch.empty(1, dtype=torch.uint8, device=dev())),
                lambda: bpe.token_logprobs_grad(x, targets, u, u[:3]), lambda: bpe.token_logprobs_grad(x, targets, u.double(), u),
                lambda: bpe.token_logprobs_grad(x, targets, u, u, out=x.half()), lambda: bpe.token_logprobs_and_grad(x, targets, u.cpu()),
                lambda: bpe.token_logprobs_and_grad(x, targets, u, out=torch.empty(4, 11, device=dev())),
                lambda: bpe.token_logprobs_and_grad(x[:, ::2], targets, u)):
        with pytest.raises(ValueError):
            bad()
    torch.cuda.synchronize()


def test_more_rows_than_one_launch_takes():
    """Rows are launched 2^21 at a time (and parts of rows as many): those of the second launch are where they belong."""
    n, vocab = (1 << 21) + 1003, 5
    check_all(some_logits(n, vocab, torch.float16, 4), some_targets(n, vocab, 5), some_upstream(n, 6))
