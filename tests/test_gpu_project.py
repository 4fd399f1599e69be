"""Logits from 8-bit rows and weights against 64 bits: whole numbers are exact, so that only the scales' roundings remain."""
import math

import pytest
import torch

import head_reference as ref
from ops_reference import TYPES, assert_near

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


def bytes_of(rows, columns, seed, spread=0, at=0, fill=None):
    g = torch.Generator().manual_seed(seed)
    room = torch.randint(-128, 128, (rows * (columns + spread) + at,), generator=g, dtype=torch.int8).to(dev())
    view = room[at:].as_strided((rows, columns), (columns + spread, 1))
    if fill is not None:
        view.fill_(fill)
    return view


def scales_of(rows, seed):
    return (torch.rand(rows, generator=torch.Generator().manual_seed(seed)) * 2.0 ** -9).to(dev())


def check(n, vocab, dim, dtype=torch.bfloat16, q_view=(0, 0), weight_view=(0, 0), out=None):
    import paper_2507_11941_amd as bpe

    q, weight = bytes_of(n, dim, 1, *q_view), bytes_of(vocab, dim, 2, *weight_view)
    scales, weight_scales = scales_of(n, 3), scales_of(vocab, 4)
    got = bpe.project_8bit(q, scales, weight, weight_scales, dtype, out)
    want = ref.project(q, scales, weight, weight_scales)
    assert got.shape == (n, vocab) and got.dtype == dtype
    assert_near(got, want, 3 * ref.U * want.abs(), f"{n} x {vocab} x {dim}")


@pytest.mark.parametrize("n", [1, 2, 8, 31, 32, 33, 61, 64, 65, 100, 128, 129, 200, 256, 257, 400, 700])
def test_products(n):
    for vocab, dim in ((1, 16), (5, 1), (127, 129), (129, 128), (257, 387), (300, 1000), (1256, 512), (64, 2064), (130, 15)):
        print(n, vocab, dim, flush=True)
        check(n, vocab, dim)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_types(dtype):
    for n in (3, 50, 100, 300):
        for vocab, dim in ((1000, 256), (259, 97), (1256, 400)):
            check(n, vocab, dim, TYPES[dtype])


@pytest.mark.parametrize("n", [7, 40, 90, 260])
def test_views(n):
    for dim in (64, 100, 144, 387):
        for q_view, weight_view in (((1, 0), (0, 0)), ((0, 3), (0, 0)), ((0, 0), (0, 5)), ((13, 1), (29, 7)), ((16 - dim % 16, 0), (16 - dim % 16, 0)),
                                    ((16 - dim % 16 + 16, 16), (16 - dim % 16, 32))):
            print(n, dim, q_view, weight_view, flush=True)
            check(n, 270, dim, torch.bfloat16, q_view, weight_view)


@pytest.mark.parametrize("dim", [48, 128, 304, 512, 700])
@pytest.mark.parametrize("n", [5, 32, 33, 64, 100, 200, 290, 520])
def test_many_tiles_of_a_workgroup(n, dim):
    """Workgroups go from one tile to the next with stages on their way: every logit, several times, of one, two and more steps."""
    import paper_2507_11941_amd as bpe

    vocab = 100260 if n < 128 else 70001
    q, weight, scales = bytes_of(n, dim, 1), bytes_of(vocab, dim, 2), scales_of(n, 3)
    weight_scales = scales_of(vocab, 4)
    sums = q.double() @ weight.double().t()                  # (whole numbers below 2^53)
    for dtype in (torch.bfloat16, torch.float32):
        # what the kernel rounds: the sum, its products with either scale, the result
        want = (sums.float() * scales[:, None] * weight_scales).to(dtype)
        for _ in range(4):
            assert torch.equal(bpe.project_8bit(q, scales, weight, weight_scales, dtype), want)


@pytest.mark.parametrize("dim", [7, 16, 100, 387, 1029, 2048])
@pytest.mark.parametrize("n", [1, 20, 31, 32])
def test_few_tokens_and_large_vocabularies(n, dim):
    """About the vocabularies from which few tokens have tiles of their own, and with a second tile for some workgroups."""
    import paper_2507_11941_amd as bpe

    for vocab, dtype, spread in ((16384, torch.bfloat16, 0), (16385, torch.float32, 4), (16512, torch.float16, 0), (30001, torch.bfloat16, 3),
                                 (65537, torch.bfloat16, 0)):
        print(n, dim, vocab, flush=True)
        q, weight = bytes_of(n, dim, 1, spread), bytes_of(vocab, dim, 2, spread)
        scales, weight_scales = scales_of(n, 3), scales_of(vocab, 4)
        # (whole numbers below 2^53; what the kernel rounds: the sum, its products with either scale, the result)
        want = ((q.double() @ weight.double().t()).float() * scales[:, None] * weight_scales).to(dtype)
        room = torch.full((n + 2, vocab + 5), 3.0, dtype=dtype, device=dev())
        out = room[1:-1, 2:vocab + 2]
        for _ in range(3):
            assert torch.equal(bpe.project_8bit(q, scales, weight, weight_scales, dtype), want)
            bpe.project_8bit(q, scales, weight, weight_scales, out=out)
            assert torch.equal(out, want)
        out.fill_(3.0)
        assert bool((room == 3.0).all())


@pytest.mark.parametrize("n", [9, 60, 130])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nothing_else_is_written(n, dtype):
    import paper_2507_11941_amd as bpe

    for vocab in (77, 260):
        room = torch.full((n + 2, vocab + 5), 3.0, dtype=dtype, device=dev())
        out = room[1:-1, 2:vocab + 2]
        before = out._version
        check(n, vocab, 160, dtype, out=out)
        assert out._version > before
        out.fill_(3.0)
        assert bool((room == 3.0).all())
    assert bpe.project_8bit(bytes_of(0, 16, 1), scales_of(0, 1), bytes_of(5, 16, 2), scales_of(5, 2)).shape == (0, 5)


def test_the_largest_sums():
    import paper_2507_11941_amd as bpe

    dim = 131071
    for a, b in ((-128, -128), (-128, 127), (127, 127)):
        for n in (1, 70):
            q, weight = bytes_of(n, dim, 1, fill=a), bytes_of(3, dim, 1, fill=b)
            one = torch.ones(n, device=dev())
            got = bpe.project_8bit(q, one, weight, torch.ones(3, device=dev()), torch.float32)
            assert bool((got.cpu().double() == float(torch.tensor(a * b * dim, dtype=torch.float32))).all())


def test_scales_that_are_none():
    import paper_2507_11941_amd as bpe

    q, weight = bytes_of(4, 64, 1), bytes_of(40, 64, 2)
    scales, weight_scales = scales_of(4, 3), scales_of(40, 4)
    scales[1], scales[2], weight_scales[7] = math.nan, 0.0, 0.0
    got = bpe.project_8bit(q, scales, weight, weight_scales, torch.float32)
    assert bool(torch.isnan(got[1]).all()) and not got[2].any() and not got[[0, 2, 3], 7].any()
    assert bool(torch.isfinite(got[[0, 2, 3]]).all())


def test_rows_of_the_norm_and_of_quantised_weights():
    """The output end as it is used, in a graph that is replayed on new hidden states: norm, product, adjustment, log-probabilities."""
    import paper_2507_11941_amd as bpe

    n, dim, vocab = 20, 200, 1256
    g = torch.Generator().manual_seed(1)
    weight, gain = torch.randn(vocab, dim, generator=g).to(dev()), torch.rand(dim, generator=g).to(dev())
    x, residual = torch.randn(n, dim, generator=g).to(dev()), torch.randn(n, dim, generator=g).to(dev())
    head, head_scales = bpe.quantize_rows(weight)
    ids = torch.randint(0, vocab, (100,), generator=g, dtype=torch.int32).to(dev())
    begin, end = torch.arange(n, device=dev()) * 5, torch.arange(n, device=dev()) * 5 + 4
    targets = torch.randint(0, vocab, (n,), generator=g, dtype=torch.int32).to(dev())

    def step():
        q, scales, total = bpe.add_norm_8bit(x, gain, residual, summed=residual)
        logits = bpe.project_8bit(q, scales, head, head_scales, torch.float32)
        adjusted = bpe.adjust_logits(logits, ids, begin, end, (1.25, 0.5, 0.0), out=logits)
        return (q, scales, total, adjusted, *bpe.token_logprobs(adjusted, targets))

    kept = residual.clone()
    want = [t.clone() for t in step()]
    s = kept + x
    rows, factor = ref.rows_8bit(s.cpu().double() * gain.cpu().double(), ref.norm(s, gain, 1e-6)[1])
    assert torch.equal(want[0].cpu(), rows) and torch.equal(want[2], s)
    logits = ref.project(rows, want[1], head, head_scales)
    wanted, off = ref.adjust(logits, ids, begin, end, (1.25, 0.5, 0.0))
    assert_near(want[3], wanted, off + 5 * ref.U * logits.abs(), "adjusted")
    # what the 8 bits lose: half a step of either factor of a product, as a random walk along the row; five of these at most
    exact = ref.norm(s, gain, 1e-6)[0] @ weight.cpu().double().t()
    step_of = (want[1].cpu().double()[:, None] * weight.cpu().double().norm(dim=1) + ref.norm(s, gain, 1e-6)[0].norm(dim=1)[:, None]
               * head_scales.cpu().double()) / math.sqrt(12)
    assert bool(((logits - exact).abs() < 6 * step_of).all())

    residual.copy_(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (None, 5, 6, None):
        residual.copy_(kept)
        if seed is None:
            x.copy_(s - kept)
        else:
            x.normal_(generator=torch.Generator(device=dev()).manual_seed(seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in captured]
        residual.copy_(kept)
        for a, b in zip(replayed, step()):
            assert torch.equal(a, b)
