"""The 8-bit product by every size of tiles, and by two of them where the last round has few: equal to what the kernel rounds."""
import os
import re

import pytest
import torch

from ops_reference import TYPES
from test_gpu_project import bytes_of, dev, scales_of

LARGE, MIDDLE, SMALL, FEW = range(4)


def rule():
    """(tokens, words and workgroups at once of each size; how long its rounds take; what a launch takes), as project.hip has them."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "paper_2507_11941_amd", "csrc", "head", "project.hip")).read()
    sizes = [tuple(map(int, s)) for s in re.findall(r"\{(\d+), (\d+), (\d+)\}", re.search(r"kSizes\[\] = \{(.*)\};", text).group(1))]
    rounds = [float(x) for x in re.search(r"kRound\[\] = \{(.*?)\}", text).group(1).split(",")]
    return sizes, rounds, float(re.search(r"kLaunch = (.*?);", text).group(1))


def plan(n, vocab):
    """The sizes of tiles that a product takes, and the columns of each launch."""
    sizes, rounds, launch = rule()
    tiles = lambda size, v: -(-n // sizes[size][0]) * -(-v // sizes[size][1])
    time = lambda size, v: rounds[size] * -(-tiles(size, v) // sizes[size][2])

    def best(v):
        if n <= 32 and tiles(SMALL, v) > 256:
            return FEW
        return SMALL if n <= 64 else min((LARGE, MIDDLE, SMALL), key=lambda size: time(size, v))

    size = best(vocab)
    whole = tiles(size, vocab) // sizes[size][2] * sizes[size][2] // -(-n // sizes[size][0]) * sizes[size][1]
    if size < SMALL and 0 < whole < vocab:
        rest = best(vocab - whole)
        if rest > size and time(size, whole) + time(rest, vocab - whole) + launch < time(size, vocab):
            return [(rest, vocab - whole), (size, whole)]
    return [(size, vocab)]


# what the products below are to try
CASES = [((257, 22001), [LARGE]), ((385, 17003), [LARGE]), ((513, 14001), [LARGE]), ((1290, 19001), [LARGE]), ((200, 70001), [MIDDLE]),
         ((129, 33001), [LARGE]), ((1025, 14000), [MIDDLE]), ((500, 98500), [SMALL, LARGE]), ((500, 100260), [SMALL, LARGE]), ((1027, 45425), [MIDDLE, LARGE])]


def test_plans():
    for (n, vocab), want in CASES:
        assert [size for size, _ in plan(n, vocab)] == want, (n, vocab)
    assert plan(500, 98500) == [(SMALL, 196), (LARGE, 98304)]
    # (five tiles of tokens: 765 large tiles in three rounds of 256)
    assert plan(1027, 45425) == [(MIDDLE, 45425 - 39168), (LARGE, 39168)]


def check(n, vocab, dim, dtype, q_view=(0, 0), weight_view=(0, 0), times=2):
    import paper_2507_11941_amd as bpe

    q, weight = bytes_of(n, dim, 1, *q_view), bytes_of(vocab, dim, 2, *weight_view)
    scales, weight_scales = scales_of(n, 3), scales_of(vocab, 4)
    # (whole numbers below 2^53; what the kernel rounds: the sum, its products with either scale, the result)
    want = ((q.double() @ weight.double().t()).float() * scales[:, None] * weight_scales).to(dtype)
    room = torch.full((n + 2, vocab + 5), 3.0, dtype=dtype, device=dev())
    out = room[1:-1, 3:vocab + 3]
    for _ in range(times):
        assert torch.equal(bpe.project_8bit(q, scales, weight, weight_scales, dtype), want)
        bpe.project_8bit(q, scales, weight, weight_scales, out=out)
        assert torch.equal(out, want)
    out.fill_(3.0)
    assert bool((room == 3.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_products(case, dtype):
    """Rows that go into shared memory by themselves, of one, two and more steps, whole and not."""
    (n, vocab), _ = CASES[case]
    for dim in (16, 100, 128, 304, 1040):
        print(dim, flush=True)
        check(n, vocab, dim, TYPES[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_products_of_rows_of_any_width_and_alignment(case, dtype):
    """Rows that go through registers; rows that begin at multiples of 4 bytes, with room behind them."""
    (n, vocab), _ = CASES[case]
    for dim, q_view, weight_view in ((387, (0, 0), (0, 0)), (1029, (3, 0), (11, 0)), (128, (0, 1), (0, 0)), (256, (0, 0), (0, 3)), (7, (0, 0), (2, 1)),
                                     (260, (13, 1), (29, 7)), (144, (4, 4), (12, 8))):
        print(dim, q_view, weight_view, flush=True)
        check(n, vocab, dim, TYPES[dtype], q_view, weight_view, 1)


@pytest.mark.gpu
def test_tiles_that_many_workgroups_go_through():
    """Thousands of tokens: several large tiles a workgroup, one after another, and bands of tokens of which the last has fewer tiles."""
    for n, vocab, dim in ((2500, 33000, 128), (2049, 40003, 300), (4100, 20001, 144)):
        assert plan(n, vocab)[-1][0] == LARGE
        check(n, vocab, dim, torch.bfloat16)
